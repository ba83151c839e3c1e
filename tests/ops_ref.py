"""The operators of mts_ops.h in 64 bits, straight from their definitions, on
the CPU, and the inputs of their tests."""
import math

import torch

# unit roundoff of the 16-bit types (half a unit in the last place)
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}


def make_batch(lens, news, bt, Hkv, D, dtype, seed=0, spare=3, layout="bhtd", poison=True):
    """A pool whose requests' blocks lie in random order, and its tables; what
    no request's slots cover is NaN.  layout: bhtd contiguous, bthd token-major,
    kv keys and values of a block side by side."""
    g = torch.Generator().manual_seed(seed)
    n = len(lens)
    nb = [-(-L // bt) for L in lens]
    blocks = sum(nb) + spare
    perm = torch.randperm(blocks, generator=g)
    width = max(nb + [1]) + 1
    table = torch.full((n, width), -7, dtype=torch.int32)
    at = 0
    for r, m in enumerate(nb):
        table[r, :m] = perm[at:at + m].int()
        at += m
    shape = {"bhtd": (blocks, Hkv, bt, D), "bthd": (blocks, bt, Hkv, D), "kv": (blocks, 2, Hkv, bt, D)}[layout]
    if layout == "kv":
        both = torch.randn(shape, generator=g).to(dtype)
        k, v = both[:, 0], both[:, 1]
    else:
        k, v = torch.randn(shape, generator=g).to(dtype), torch.randn(shape, generator=g).to(dtype)
        if layout == "bthd":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
    if poison:
        used = torch.zeros(blocks, bt, dtype=torch.bool)
        for r, L in enumerate(lens):
            j = torch.arange(L)
            used[table[r].long()[j // bt], j % bt] = True
        free = ~used[:, None, :, None].expand(blocks, Hkv, bt, D)
        k.masked_fill_(free, math.nan)
        v.masked_fill_(free, math.nan)
    q_start = torch.tensor([sum(news[:r]) for r in range(n + 1)], dtype=torch.int32)
    return dict(k=k, v=v, table=table, lens=torch.tensor(lens, dtype=torch.int32), q_start=q_start, bt=bt, max_q=max(news + [1]), g=g)


def random_tree(news, g, words=None):
    """Ancestor bits [tokens][words] of random trees (a token sees itself)."""
    words = words or -(-max(news + [1]) // 64)
    rows = []
    for T in news:
        bits = []
        for j in range(T):
            parent = int(torch.randint(0, j + 1, (1,), generator=g)) - 1
            bits.append((bits[parent] if parent >= 0 else 0) | 1 << j)
        rows += bits
    out = torch.zeros(len(rows), words, dtype=torch.int64)
    for i, b in enumerate(rows):
        for w in range(words):
            x = (b >> 64 * w) & (1 << 64) - 1
            out[i, w] = x - (1 << 64) if x >> 63 else x
    return out


def sees(b, r, t, j, tree):
    """Whether new token t of request r attends slot j."""
    T = int(b["q_start"][r + 1] - b["q_start"][r])
    rel = j - (int(b["lens"][r]) - T)
    if rel < 0:
        return True
    if tree is None:
        return rel <= t
    row = tree[int(b["q_start"][r]) + t]
    return rel < 64 * row.numel() and bool((int(row[rel // 64]) >> (rel % 64)) & 1)


def mask_of(b, r, tree):
    """[T, L] of sees()."""
    L, a = int(b["lens"][r]), int(b["q_start"][r])
    T = int(b["q_start"][r + 1]) - a
    see = torch.ones(T, L, dtype=torch.bool)
    for t in range(T):
        for j in range(max(0, L - T), L):
            see[t, j] = sees(b, r, t, j, tree)
    return see


def rows_of(b, r, x, h):
    """The slots of request r in order, and which of them lie in the pool."""
    L, bt = int(b["lens"][r]), b["bt"]
    j = torch.arange(L)
    blk = b["table"][r].long()[j // bt]
    ok = (blk >= 0) & (blk < x.shape[0])
    return x[blk.clamp(0, x.shape[0] - 1), h, j % bt], ok


def attend(b, q, scale=None, tree=None):
    """(out, lse, bound on the error of out, bound on that of lse)."""
    N, Hq, D = q.shape
    Hkv = b["k"].shape[1]
    G = Hq // Hkv
    u = ROUND[q.dtype]
    scale = D ** -0.5 if scale is None else scale
    out = torch.zeros(N, Hq, D, dtype=torch.float64)
    lse = torch.full((N, Hq), -math.inf, dtype=torch.float64)
    spread = torch.zeros(N, Hq, D, dtype=torch.float64)
    size = torch.zeros(N, Hq, dtype=torch.float64)
    for r in range(len(b["lens"])):
        a, z = int(b["q_start"][r]), int(b["q_start"][r + 1])
        if a == z:
            continue
        see = mask_of(b, r, tree)
        for h in range(Hq):
            k, ok = rows_of(b, r, b["k"], h // G)
            v, _ = rows_of(b, r, b["v"], h // G)
            for t in range(z - a):
                on = see[t] & ok
                if not on.any():
                    continue
                kk, vv, qq = k[on].double(), v[on].double(), q[a + t, h].double()
                x = (kk @ qq) * scale
                m = x.max()
                p = torch.exp(x - m)
                out[a + t, h] = (p / p.sum()) @ vv
                lse[a + t, h] = m + torch.log(p.sum())
                spread[a + t, h] = (p / p.sum()) @ vv.abs()
                size[a + t, h] = (kk.abs() @ qq.abs()).max() * abs(scale)
    # a score is a sum of D exact products in 32 bits, two roundings when it is scaled and shifted, one or two units of
    # the power of two: the weights' relative error, on the output and on lse; then the weights rounded to the type for
    # the product with the values, and the output rounded once
    e32 = 2.0 ** -24
    weight = (D + 16) * e32 * (size + 1)
    # below the 16-bit type's normal range a weight's rounding is absolute
    tiny = 2.0 ** -24 if q.dtype == torch.float16 else 0.0
    vmax = b["v"].double().nan_to_num(0, 0, 0).abs().max()
    bound = u * out.abs() + (u + 2 * weight[..., None] + 1e-5) * spread + tiny * b["lens"].max().item() * vmax
    return out, lse, bound * 1.02, weight * 2 + 8 * e32 * (1 + lse.abs().nan_to_num(0, 0, 0))


def weigh(b, q, lse, score, decay, scale=None, tree=None):
    """(score, bound on its error)."""
    N, Hq, D = q.shape
    Hkv = b["k"].shape[1]
    G = Hq // Hkv
    scale = D ** -0.5 if scale is None else scale
    out, err = score.double().clone(), torch.zeros(score.shape, dtype=torch.float64)
    e32 = 2.0 ** -24
    for r in range(len(b["lens"])):
        a, z, L = int(b["q_start"][r]), int(b["q_start"][r + 1]), int(b["lens"][r])
        if a == z:
            continue
        see = mask_of(b, r, tree)
        for hk in range(Hkv):
            k, ok = rows_of(b, r, b["k"], hk)
            w = torch.zeros(L, dtype=torch.float64)
            e = torch.zeros(L, dtype=torch.float64)
            for t in range(z - a):
                on = see[t] & ok
                for h in range(hk * G, hk * G + G):
                    if lse[a + t, h] == -math.inf:
                        continue
                    kk, qq = k[on].double(), q[a + t, h].double()
                    p = torch.exp((kk @ qq) * scale - lse[a + t, h].double())
                    w[on] += p
                    e[on] += p * ((D + 16) * e32 * ((kk.abs() @ qq.abs()) * abs(scale) + 1) + 4 * e32 * lse[a + t, h].abs().double())
            for j in range(L):
                if not ok[j]:
                    continue
                at = (int(b["table"][r, j // b["bt"]]), hk, j % b["bt"])
                old = 0.0 if decay == 0.0 or j >= L - (z - a) else decay * float(score[at])
                out[at] = old + w[j]
                err[at] = 2 * e[j] + (z - a) * G * e32 * w[j] + 4 * e32 * (abs(old) + w[j])
    return out, err


def evict(b, score, pos, next_pos, budget, recent, sink):
    """(k, v, score, pos, lens) after an eviction in place."""
    k, v, s, ps = b["k"].clone(), b["v"].clone(), score.clone(), pos.clone()
    bt, lens = b["bt"], []
    for r, L in enumerate(b["lens"].tolist()):
        lens.append(min(L, budget))
        if L <= budget:
            continue
        at = [(int(b["table"][r, j // bt]), j % bt) for j in range(L)]
        for h in range(k.shape[1]):
            def rank(j):
                blk, off = at[j]
                if not 0 <= blk < k.shape[0]:
                    return (2, 0.0, j)
                p = int(pos[blk, h, off])
                if p < sink or p >= int(next_pos[r]) - recent:
                    return (0, 0.0, j)
                x = float(score[blk, h, off])
                return (1, math.inf if x != x else -x, j)
            keep = set(sorted(range(L), key=rank)[:budget])
            holes = [j for j in range(budget) if j not in keep]
            come = [j for j in sorted(keep) if j >= budget]
            assert len(holes) == len(come)
            for to, frm in zip(holes, come):
                (tb, to_), (fb, fo) = at[to], at[frm]
                if not (0 <= tb < k.shape[0] and 0 <= fb < k.shape[0]):
                    continue
                k[tb, h, to_], v[tb, h, to_] = b["k"][fb, h, fo], b["v"][fb, h, fo]
                s[tb, h, to_], ps[tb, h, to_] = score[fb, h, fo], pos[fb, h, fo]
    return k, v, s, ps, torch.tensor(lens, dtype=torch.int32)


def kept_weights(x, temperature, top_k, top_p, min_p):
    """A row's weights in vocabulary order, zero where not kept; None for a row without a logit above -inf."""
    x = x.double()
    x = torch.where(torch.isnan(x), -math.inf, x) + 0.0
    top = x.max()
    if top == -math.inf:
        return None
    w = torch.where(x == top, 1.0, torch.exp((x - top) / temperature))
    order = torch.sort(x, descending=True, stable=True)[1]
    if top_k > 0:
        order = order[:top_k]
    c = torch.cumsum(w[order], 0)
    if top_p < 1:
        before = c - w[order]
        keep = before < top_p * c[-1]
        keep[0] = True
        order = order[keep]
    order = order[w[order] >= min(min_p, 1.0)]
    out = torch.zeros_like(w)
    out[order] = w[order]
    return out


def rope(x, positions, freqs, layout, mscale=1.0, inverse=False):
    rot = 2 * freqs.numel()
    a = positions.double()[:, None, None] * freqs.double()
    c, s = torch.cos(a) * mscale, torch.sin(a) * mscale * (-1 if inverse else 1)
    y = x.double().clone()
    at = (slice(0, rot, 2), slice(1, rot, 2)) if layout == "interleaved" else (slice(0, rot // 2), slice(rot // 2, rot))
    p, q = x[..., at[0]].double(), x[..., at[1]].double()
    y[..., at[0]], y[..., at[1]] = p * c - q * s, p * s + q * c
    return y
