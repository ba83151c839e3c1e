"""Timed cases of the operators that one serving instance runs in a tick.

The scheduler counts an instance's KV blocks and its requests' tokens; these
operators are what the instance computes on them: rotary positions and the
append to the paged cache, attention of single tokens, drafted trees and
prompt chunks over it, the attention weight its slots accumulate, the eviction
of the least attended ones, and the draw of the next token.

Request lengths follow the workload presets (log-normal prompts, 16-token
blocks); they are the distribution's quantiles, so a case reads the same
number of tokens for every seed while the order, the blocks and the values
change.
"""
import math
import statistics

import torch

own = False

DEV = "cuda"
_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}


def listed():
    return [
        # the tick's tokens of one instance: a row a request, written to its block
        dict(name="rope_token", op="rope_append", n=150, Hq=32, Hkv=8, D=128, rot=128, type="bf16", layout="half",
             scaling="none", span=8192),
        # the prompts of a batch: pairs interleaved, half of the head, positions of a stretched context
        dict(name="rope_prompt", op="rope_append", n=16384, Hq=32, Hkv=8, D=128, rot=64, type="fp16", layout="interleaved",
             scaling="parts", span=131072),
        # one request of the tiny preset decoding alone: latency
        dict(name="attend_token", op="attend", n=1, mu=0.0, sigma=0.0, lo=1024, hi=1024, T=1, Tmin=1, tree=False, Hq=32, Hkv=8,
             D=128, type="bf16", bt=16),
        # an instance of the enterprise preset decoding its running requests
        dict(name="attend_decode", op="attend", n=150, mu=6.2, sigma=0.8, lo=32, hi=8192, T=1, Tmin=1, tree=False, Hq=32, Hkv=8,
             D=128, type="bf16", bt=16),
        # drafted trees of 1 to 48 tokens verified over the wide preset's contexts; five query heads a KV head
        dict(name="attend_tree", op="attend", n=24, mu=8.0, sigma=1.2, lo=32, hi=32768, T=48, Tmin=1, tree=True, Hq=40, Hkv=8,
             D=128, type="fp16", bt=16),
        # chunks of long prompts, their earlier part already in the cache
        dict(name="attend_chunk", op="attend", n=3, mu=8.7, sigma=0.8, lo=2048, hi=16384, T=2048, Tmin=1500, tree=False, Hq=32,
             Hkv=8, D=128, type="bf16", bt=16),
        # the decode step's weights, accumulated with a decay
        dict(name="weigh_decode", op="weigh", n=150, mu=6.2, sigma=0.8, lo=32, hi=8192, T=1, Tmin=1, tree=False, Hq=32, Hkv=8,
             D=128, type="bf16", bt=16, decay=0.98),
        # the weights that the last tokens of long prompts give, before their first eviction
        dict(name="weigh_window", op="weigh", n=6, mu=9.2, sigma=0.5, lo=1024, hi=32768, T=64, Tmin=64, tree=False, Hq=32, Hkv=8,
             D=64, type="fp16", bt=16, decay=0.0),
        # two requests brought down to their budgets between ticks
        dict(name="evict_few", op="evict", n=2, mu=7.6, sigma=0.3, lo=1024, hi=4096, Hkv=8, D=128, type="bf16", bt=16, budget=1024,
             recent=64, sink=4),
        # an instance out of blocks: every long request of the wide preset shrinks
        dict(name="evict_pressure", op="evict", n=64, mu=7.0, sigma=1.2, lo=32, hi=32768, Hkv=8, D=128, type="bf16", bt=16,
             budget=1000, recent=128, sink=4),
        # one request's token from a small vocabulary
        dict(name="sample_one", op="sample", B=1, V=32768, type="fp32", mix="nucleus"),
        # a slot of every kind of request: a vocabulary of odd size, greedy, top-k, top-p, min-p and unrestricted rows mixed
        dict(name="sample_batch", op="sample", B=512, V=100003, type="bf16", mix="all"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    op = rng.choice(["rope", "rope_append", "attend", "attend", "attend", "weigh", "evict", "sample", "sample"])
    if op == "sample":
        B = int(_log(rng, 1, 512.99))
        return dict(op=op, B=B, V=int(min(_log(rng, 1000, 131073), 512 * 100003 // B)), type=rng.choice(["fp32", "bf16", "bf16", "fp16"]),
                    mix=rng.choice(["all", "nucleus", "topk", "minp", "plain"]))
    Hkv = rng.choice([1, 2, 4, 8, 8, 8])
    G = rng.choice([1, 2, 4, 4, 5, 7, 8])
    D = rng.choice([64, 96, 128, 128, 128, 256])
    kind = rng.choice(["bf16", "bf16", "fp16"])
    if op in ("rope", "rope_append"):
        rot = rng.choice([D, D, D // 2])
        most = 16384 * 48 * 128 // ((G + 2) * Hkv * D)
        return dict(op=op, n=int(_log(rng, 1, max(2, min(16384, most)))), Hq=G * Hkv, Hkv=Hkv, D=D, rot=rot,
                    type=rng.choice([kind, kind, "fp32"]) if op == "rope" else kind, layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "parts"]), span=rng.choice([2048, 32768, 131072, 1000000]),
                    inverse=op == "rope" and rng.random() < 0.5)
    c = dict(op=op, mu=round(rng.uniform(6.2, 7.5), 2), sigma=round(rng.uniform(0.3, 1.2), 2), lo=32, hi=rng.choice([4096, 8192, 16384, 32768]),
             Hkv=Hkv, D=D, type=kind, bt=rng.choice([16, 16, 16, 8, 32, 64]))
    n = int(_log(rng, 1, 150.99))
    if op == "evict":
        n = min(n, 64)
        c.update(budget=int(_log(rng, 100, 2048)), recent=rng.choice([0, 16, 64]), sink=rng.choice([0, 1, 4]))
    else:
        shape = rng.choice(["token", "token", "tree", "chunk"] if op == "attend" else ["token", "token", "window"])
        T = {"token": 1, "tree": rng.randint(2, 64), "chunk": int(_log(rng, 65, 2048)), "window": rng.randint(2, 64)}[shape]
        c.update(Hq=G * Hkv, T=T, Tmin=rng.randint(max(1, T // 4), T), tree=shape == "tree")
        if op == "weigh":
            c.update(decay=rng.choice([0.0, 0.9, 1.0]))
        if shape == "chunk":
            n = min(n, 4)
            c.update(hi=min(c["hi"], 16384))
    # no more cache than the listed cases read
    while n > 1 and sum(_lengths(dict(c, n=n))) * Hkv * D > 105000 * 8 * 128:
        n = n * 3 // 4
    while n > 1 and n * max(_lengths(dict(c, n=n))) * Hkv * D > 150 * 8192 * 8 * 128:
        n = n * 3 // 4
    c["n"] = n
    # no more scores than the listed chunks have
    while c.get("T", 1) > 1 and c["T"] * n * max(_lengths(c)) * c["Hq"] * max(D, 128) > 2048 * 3 * 13000 * 32 * 128:
        c["T"] = max(1, c["T"] * 3 // 4)
        c["Tmin"] = min(c["Tmin"], c["T"])
    return c


# ---------------------------------------------------------------- inputs


def _lengths(c):
    """The quantiles of the case's log-normal lengths, clipped."""
    N = statistics.NormalDist()
    q = [N.inv_cdf((i + 0.5) / c["n"]) for i in range(c["n"])]
    return [int(min(c["hi"], max(c["lo"], round(math.exp(c["mu"] + c["sigma"] * z))))) for z in q]


def _drafts(c):
    """New tokens of every request, spread over [Tmin, T]; a prompt is never shorter than its chunk."""
    lo, hi, n = c["Tmin"], c["T"], c["n"]
    T = [lo + (hi - lo) * (i + 1) // n if n > 1 else hi for i in range(n)]
    return [min(t, L) for t, L in zip(T, _lengths(c))]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape, type=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32 if type == torch.float32 else type)


def _freqs(rot, scaling, span):
    """Radians a position turns each pair by, and the factor on the rotated values: plain, positions divided by a factor,
    or fast pairs kept and slow ones divided with a ramp between."""
    f = torch.tensor([10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64)
    factor = max(1.0, span / 4096)
    if scaling == "linear":
        f = f / factor
    if scaling == "parts":
        turns = 4096 * f / (2 * math.pi)
        keep = ((turns - 1.0) / 31.0).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
        return f.to(DEV), 0.1 * math.log(factor) + 1.0
    return f.to(DEV), 1.0


def _cache(c, g, lens):
    """A pool a little larger than the requests need and the tables of their blocks, in random order."""
    bt = c["bt"]
    nb = [-(-L // bt) for L in lens]
    blocks = sum(nb) + 7
    perm = torch.randperm(blocks, generator=g, device=DEV).to(torch.int32)
    width = max(nb)
    take = torch.full((c["n"], width), -1, dtype=torch.int64)
    at = 0
    for r, m in enumerate(nb):
        take[r, :m] = torch.arange(at, at + m)
        at += m
    take = take.to(DEV)
    table = torch.where(take >= 0, perm[take.clamp(min=0)], -1)
    t = _TYPES[c["type"]]
    shape = (blocks, c["Hkv"], bt, c["D"])
    # a few channels of the keys carry a common offset, as rotated keys do
    k = _randn(g, *shape, type=t)
    k += (_randn(g, c["D"]) * (torch.rand(c["D"], generator=g, device=DEV) < 0.06) * 2.0).to(t)
    v = _randn(g, *shape, type=t)
    return k, v, table


def _tree(g, drafts):
    """Ancestor bits of random drafted trees: token j hangs below the request's last token or an earlier drafted one."""
    top = max(drafts)
    words = -(-top // 64)
    r = torch.rand(sum(drafts), generator=g, device=DEV).tolist()
    rows, at = [], 0
    for T in drafts:
        bits = []
        for j in range(T):
            parent = int(r[at + j] * (j + 1)) - 1
            bits.append((bits[parent] if parent >= 0 else 0) | 1 << j)
        rows += bits
        at += T
    signed = [[((b >> 64 * w) & (1 << 64) - 1) for w in range(words)] for b in rows]
    return torch.tensor([[x - (1 << 64) if x >> 63 else x for x in row] for row in signed], dtype=torch.int64, device=DEV)


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed)
    t = _TYPES[c["type"]]
    s = dict(c=c)
    if c["op"] == "sample":
        B, V = c["B"], c["V"]
        x = _randn(g, B, V) * 2.0
        # a handful of likely tokens a row
        x.scatter_add_(1, torch.randint(0, V, (B, 24), generator=g, device=DEV), torch.rand(B, 24, generator=g, device=DEV) * 10.0)
        s["logits"] = x.to(t)
        s["u"] = torch.rand(B, generator=g, device=DEV)
        kind = {"all": torch.arange(B, device=DEV) % 6, "nucleus": 1, "topk": 2, "minp": 3, "plain": 4}[c["mix"]]
        kind = kind if torch.is_tensor(kind) else torch.full((B,), kind, device=DEV)
        r = torch.rand(B, generator=g, device=DEV)
        # 0 greedy, 1 top-p, 2 top-k, 3 min-p, 4 unrestricted, 5 all three
        s["temperature"] = torch.where(kind == 0, 0.0, 0.6 + 0.6 * r)
        s["top_k"] = torch.where((kind == 2) | (kind == 5), (20 + 180 * r).long(), 0).to(torch.int32)
        s["top_p"] = torch.where((kind == 1) | (kind == 5), 0.85 + 0.13 * r, 1.0)
        s["min_p"] = torch.where((kind == 3) | (kind == 5), 0.02 + 0.08 * r, 0.0)
        return s
    if c["op"] in ("rope", "rope_append"):
        n, Hq, Hkv, D = c["n"], c["Hq"], c["Hkv"], c["D"]
        # one fused projection's rows, as a model's layer hands them over
        qkv = _randn(g, n, (Hq + 2 * Hkv) * D, type=t)
        s["q"] = qkv[:, :Hq * D].view(n, Hq, D)
        s["k"] = qkv[:, Hq * D:(Hq + Hkv) * D].view(n, Hkv, D)
        s["v"] = qkv[:, (Hq + Hkv) * D:].view(n, Hkv, D)
        s["positions"] = torch.randint(0, c["span"], (n,), generator=g, device=DEV).to(torch.int32)
        s["freqs"], s["mscale"] = _freqs(c["rot"], c["scaling"], c["span"])
        if c["op"] == "rope_append":
            bt = 16
            blocks = -(-n // bt) + 5
            s["slots"] = torch.randperm(blocks * bt, generator=g, device=DEV)[:n].contiguous()
            s["k_cache"] = torch.zeros(blocks, Hkv, bt, D, dtype=t, device=DEV)
            s["v_cache"] = torch.zeros_like(s["k_cache"])
            s["pos"] = torch.zeros(blocks, Hkv, bt, dtype=torch.int32, device=DEV)
        return s
    order = torch.randperm(c["n"], generator=g, device=DEV).tolist()
    lens = _lengths(c)
    drafts = _drafts(c) if c["op"] != "evict" else [1] * c["n"]
    lens, drafts = [lens[i] for i in order], [drafts[i] for i in order]
    s["k_cache"], s["v_cache"], s["table"] = _cache(c, g, lens)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    if c["op"] == "evict":
        shape = s["k_cache"].shape[:3]
        s["score"] = torch.exp(1.5 * _randn(g, *shape))
        width = s["table"].shape[1]
        where = torch.arange(width * c["bt"], dtype=torch.int32, device=DEV).view(width, 1, c["bt"]).expand(width, c["Hkv"], c["bt"])
        s["pos"] = torch.zeros(shape, dtype=torch.int32, device=DEV)
        used = s["table"] >= 0
        s["pos"][s["table"][used].long()] = where.expand(c["n"], *where.shape)[used]
        s["next_pos"] = s["lens"].clone()
        s["score_out"], s["pos_out"] = torch.zeros_like(s["score"]), torch.zeros_like(s["pos"])
        return s
    s["max_q"] = max(drafts)
    s["q_start"] = torch.tensor([sum(drafts[:r]) for r in range(c["n"] + 1)], dtype=torch.int32, device=DEV)
    # queries that pick out some keys: scores spread over a few units
    s["q"] = (_randn(g, sum(drafts), c["Hq"], c["D"]) * 1.7).to(t)
    s["tree"] = _tree(g, drafts) if c["tree"] else None
    if c["op"] == "weigh":
        s["score"] = torch.exp(_randn(g, *s["k_cache"].shape[:3]))
        s["lse"] = _attend(s)[1]
    return s


# ---------------------------------------------------------------- plain forms


def _rotate(x, cos, sin, rot, layout):
    f = x.float()
    a, b = (f[..., 0:rot:2], f[..., 1:rot:2]) if layout == "interleaved" else (f[..., :rot // 2], f[..., rot // 2:rot])
    ra, rb = a * cos - b * sin, a * sin + b * cos
    r = torch.stack((ra, rb), -1).flatten(-2) if layout == "interleaved" else torch.cat((ra, rb), -1)
    return torch.cat((r, f[..., rot:]), -1).to(x.dtype)


def _rope(s):
    c = s["c"]
    # a position times a frequency has more digits than 32 bits hold: the angle is formed in 64
    angle = s["positions"].double()[:, None, None] * s["freqs"]
    m = s["mscale"]
    cos, sin = (angle.cos() * m).float(), (angle.sin() * m).float()
    if c.get("inverse"):
        sin = -sin
    q, k = (_rotate(s[x], cos, sin, c["rot"], c["layout"]) for x in "qk")
    if c["op"] == "rope":
        return q, k
    bt = s["k_cache"].shape[2]
    at = (s["slots"] // bt, slice(None), s["slots"] % bt)
    s["k_cache"][at] = k
    s["v_cache"][at] = s["v"]
    s["pos"][at] = s["positions"][:, None].expand(-1, c["Hkv"])
    return q, s["k_cache"], s["v_cache"], s["pos"]


def _visible(s, T, L):
    """[n, T, L]: which slots each new token attends."""
    t = torch.arange(T, device=DEV)
    row = (s["q_start"][:-1, None] + t).clamp(max=s["q"].shape[0] - 1).long()
    new = (s["q_start"][1:] - s["q_start"][:-1]).long()
    j = torch.arange(L, device=DEV)
    rel = (j - (s["lens"].long() - new)[:, None])[:, None, :]
    if s["tree"] is None:
        see = rel <= t[None, :, None]
    else:
        at = rel.clamp(0, 64 * s["tree"].shape[1] - 1)
        bits = torch.gather(s["tree"][row], 2, (at // 64).expand(-1, T, -1))
        see = (rel < 0) | ((bits >> (at % 64)) & 1).bool()
    return see & (j < s["lens"][:, None])[:, None, :] & (t < new[:, None])[:, :, None], row, t < new[:, None]


def _keys(s, x):
    """A request's rows of a pool in slot order, heads first: [n, Hkv, L, ...]."""
    y = x[s["table"].clamp(min=0).long()].transpose(1, 2)
    return y.reshape(y.shape[0], y.shape[1], -1, *y.shape[4:])


def _scores(s):
    c = s["c"]
    n, Hkv, D, T = c["n"], c["Hkv"], c["D"], s["max_q"]
    G = c["Hq"] // Hkv
    k = _keys(s, s["k_cache"]).float()
    see, row, real = _visible(s, T, k.shape[2])
    q = s["q"][row].float().view(n, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(n, Hkv, T * G, D)
    x = torch.matmul(q * D ** -0.5, k.transpose(-1, -2).contiguous())
    see = see[:, None, :, None, :].expand(n, Hkv, T, G, -1).reshape(n, Hkv, T * G, -1)
    return x, see, row, real


def _attend(s):
    c = s["c"]
    n, Hkv, D, T = c["n"], c["Hkv"], c["D"], s["max_q"]
    G = c["Hq"] // Hkv
    x, see, row, real = _scores(s)
    x = x.masked_fill_(~see, -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p = x.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    v = _keys(s, s["v_cache"]).float()
    o = torch.matmul(p, v) / torch.where(z == 0, 1.0, z)
    lse = torch.log(z) + m
    back = lambda y: y.view(n, Hkv, T, G, -1).permute(0, 2, 1, 3, 4).reshape(n, T, Hkv * G, -1)[real]  # noqa: E731
    return back(o).to(s["q"].dtype), back(lse).squeeze(-1)


def _weigh(s):
    c = s["c"]
    n, Hkv, T = c["n"], c["Hkv"], s["max_q"]
    G = c["Hq"] // Hkv
    x, see, row, _ = _scores(s)
    lse = s["lse"][row].view(n, T, Hkv, G).permute(0, 2, 1, 3).reshape(n, Hkv, T * G, 1)
    w = torch.where(see, torch.exp(x - lse), 0.0).sum(2)
    bt, L = c["bt"], w.shape[2]
    j = torch.arange(L, device=DEV)
    new = (s["q_start"][1:] - s["q_start"][:-1])[:, None]
    old = _keys(s, s["score"])
    first = (j >= s["lens"][:, None] - new)[:, None] | (c["decay"] == 0.0)
    w = torch.where(first, w, c["decay"] * old + w)
    r, at = torch.nonzero(j < s["lens"][:, None], as_tuple=True)
    s["score"][s["table"][r, at // bt].long(), :, at % bt] = w[r, :, at]
    return s["score"]


def _evict(s):
    c = s["c"]
    bt, B = c["bt"], c["budget"]
    score, pos = _keys(s, s["score"]), _keys(s, s["pos"])
    L = score.shape[2]
    j = torch.arange(L, device=DEV)
    live = (j < s["lens"][:, None])[:, None]
    kept_first = (pos < c["sink"]) | (pos >= (s["next_pos"] - c["recent"])[:, None, None])
    key = torch.where(kept_first, math.inf, torch.where(score != score, -math.inf, score))
    key = torch.where(live, key, -math.inf)
    order = torch.argsort(key, dim=-1, descending=True, stable=True)
    rank = torch.empty_like(order).scatter_(-1, order, j.expand_as(order).contiguous())
    keep = (rank < B) & live
    r, h, src = torch.nonzero(keep & (j >= B), as_tuple=True)
    _, _, dst = torch.nonzero(~keep & (j < B) & live, as_tuple=True)
    block = lambda r, at: s["table"][r, at // bt].long()  # noqa: E731
    # what stays below the budget, then what moves into the holes
    r0, h0, at0 = torch.nonzero(keep & (j < B), as_tuple=True)
    here = (block(r0, at0), h0, at0 % bt)
    a, b = (block(r, src), h, src % bt), (block(r, dst), h, dst % bt)
    s["score_out"][here], s["pos_out"][here] = s["score"][here], s["pos"][here]
    s["score_out"][b], s["pos_out"][b] = s["score"][a], s["pos"][a]
    s["k_cache"][b], s["v_cache"][b] = s["k_cache"][a], s["v_cache"][a]
    return s["k_cache"], s["v_cache"], s["score_out"], s["pos_out"], s["lens"].clamp(max=B)


def _sample(s):
    x = s["logits"].float()
    x = torch.where(x != x, -math.inf, x) + 0.0
    V = x.shape[1]
    t, k, p, mp = (s[n][:, None] for n in ("temperature", "top_k", "top_p", "min_p"))
    xs, idx = torch.sort(x, dim=1, descending=True, stable=True)
    top = xs[:, :1]
    w = torch.where(xs == top, 1.0, torch.exp((xs - top) * (1.0 / t)))
    ranked = torch.arange(V, device=DEV) < torch.where(k > 0, k, V)
    # the token is a whole number that sums decide: they are carried in 64 bits
    w = torch.where(ranked, w, 0.0).double()
    below = w.cumsum(1) - w
    keep = ranked & ((p >= 1.0) | (below < p.double() * w.sum(1, keepdim=True))) & (w >= mp)
    w = torch.zeros_like(w).scatter_(1, idx, torch.where(keep, w, 0.0))
    c = w.cumsum(1)
    W = c[:, -1:]
    token = (c <= s["u"].double()[:, None] * W).sum(1, keepdim=True).clamp(max=V - 1)
    logp = (torch.gather(w, 1, token) / W).log().float()
    greedy, dead = t <= 0, top == -math.inf
    token = torch.where(dead, -1, torch.where(greedy, idx[:, :1], token))
    logp = torch.where(dead, -math.inf, torch.where(greedy, 0.0, logp))
    return token[:, 0].to(torch.int32), logp[:, 0]


# ---------------------------------------------------------------- one pass


def run(state):
    s = state
    c = s["c"]
    op = c["op"]
    if not own:
        return {"rope": _rope, "rope_append": _rope, "attend": _attend, "weigh": _weigh, "evict": _evict, "sample": _sample}[op](s)
    from paper_2608_16336_amd import ops
    if op == "rope":
        return ops.rope(s["q"], s["k"], s["positions"], s["freqs"], layout=c["layout"], mscale=s["mscale"], inverse=c["inverse"])
    if op == "rope_append":
        q = ops.rope_append(s["q"], s["k"], s["v"], s["positions"], s["slots"], s["freqs"], s["k_cache"], s["v_cache"], s["pos"],
                            layout=c["layout"], mscale=s["mscale"])
        return q, s["k_cache"], s["v_cache"], s["pos"]
    if op == "sample":
        return ops.sample(s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"])
    if op == "attend":
        return ops.attend(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["q_start"], s["max_q"], tree=s["tree"])
    if op == "weigh":
        return ops.weigh(s["q"], s["lse"], s["k_cache"], s["table"], s["lens"], s["q_start"], s["max_q"], s["score"],
                         decay=c["decay"], tree=s["tree"])
    lens = ops.evict(s["k_cache"], s["v_cache"], s["score"], s["pos"], s["table"], s["lens"], s["next_pos"], c["budget"],
                     recent=c["recent"], sink=c["sink"], score_out=s["score_out"], pos_out=s["pos_out"])
    return s["k_cache"], s["v_cache"], s["score_out"], s["pos_out"], lens


def work(case):
    c = case
    e = _BYTES[c["type"]]
    if c["op"] == "sample":
        return dict(bytes=c["B"] * (c["V"] * e + 28), flops=4.0 * c["B"] * c["V"])
    if c["op"] in ("rope", "rope_append"):
        heads = c["Hq"] + c["Hkv"]
        extra = 2 * c["Hkv"] * c["D"] * e + 12 + 4 * c["Hkv"] if c["op"] == "rope_append" else 4
        return dict(bytes=c["n"] * (2 * heads * c["D"] * e + extra), flops=3.0 * c["n"] * heads * c["rot"])
    lens, Hkv, D = _lengths(c), c["Hkv"], c["D"]
    row = Hkv * D * e
    if c["op"] == "evict":
        B, moved, kept = c["budget"], 0.0, 0
        for L in lens:
            kept += min(L, B)
            if L > B:
                # the recent ones above the budget move; of the others' places below it, as many as scores in random order leave
                recent = min(c["recent"], L - B, B)
                rest = max(0, B - min(c["recent"], B) - c["sink"])
                pool = L - c["recent"] - c["sink"]
                moved += recent + (rest * max(0, L - B - c["recent"]) / pool if pool > 0 else 0)
        return dict(bytes=sum(lens) * Hkv * 8 + kept * Hkv * 8 + moved * 4 * row, flops=0.0)
    drafts = _drafts(c)
    # a drafted token sees about half of its tree or chunk
    seen = sum(T * (L - T) + T * (T + 1) / 2 for T, L in zip(drafts, lens))
    rows = sum(drafts) * c["Hq"]
    if c["op"] == "attend":
        return dict(bytes=2 * sum(lens) * row + rows * (2 * D * e + 4), flops=4.0 * c["Hq"] * D * seen)
    return dict(bytes=sum(lens) * (row + Hkv * (8 if c["decay"] else 4)) + rows * (D * e + 4), flops=2.0 * c["Hq"] * D * seen)


# ---------------------------------------------------------------- 64 bits


def _exact_rope(s, c):
    f = s["freqs"] * (-1.0 if c.get("inverse") else 1.0)
    turn = torch.polar(torch.full((c["n"], 1, f.numel()), float(s["mscale"]), dtype=torch.float64, device=DEV),
                       (s["positions"].double()[:, None] * f)[:, None])
    outs = []
    for x in (s["q"], s["k"]):
        y = x.double().clone()
        half = c["rot"] // 2
        at = (slice(0, c["rot"], 2), slice(1, c["rot"], 2)) if c["layout"] == "interleaved" else (slice(0, half), slice(half, 2 * half))
        z = torch.complex(y[..., at[0]], y[..., at[1]]) * turn
        y[..., at[0]], y[..., at[1]] = z.real, z.imag
        outs.append(y)
    if c["op"] == "rope":
        return tuple(outs)
    kc, vc, pos = s["k_cache"].double(), s["v_cache"].double(), s["pos"].clone()
    blk, off = torch.div(s["slots"], 16, rounding_mode="floor"), s["slots"].remainder(16)
    for h in range(c["Hkv"]):
        kc[blk, h, off], vc[blk, h, off], pos[blk, h, off] = outs[1][:, h], s["v"][:, h].double(), s["positions"]
    return outs[0], kc, vc, pos


def _exact_attention(s, c, weights):
    """One request and KV head at a time, straight from the definition."""
    G, D, bt = c["Hq"] // c["Hkv"], c["D"], c["bt"]
    start, lens = s["q_start"].tolist(), s["lens"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEV)
    score = s["score"].double() if weights else None
    for r in range(c["n"]):
        a, b, L = start[r], start[r + 1], lens[r]
        T = b - a
        blocks = s["table"][r, :-(-L // bt)].long()
        see = torch.ones(T, L, dtype=torch.bool, device=DEV)
        if s["tree"] is None:
            see[:, L - T:] = torch.ones(T, T, dtype=torch.bool, device=DEV).tril()
        else:
            one = torch.arange(64, device=DEV)
            see[:, L - T:] = (((s["tree"][a:b, :, None] >> one) & 1) == 1).flatten(1)[:, :T]
        for h in range(c["Hkv"]):
            k = s["k_cache"][blocks, h].reshape(-1, D)[:L].double()
            q = s["q"][a:b, h * G:(h + 1) * G].double()
            x = (torch.matmul(q.reshape(T * G, D), k.t().contiguous()) / math.sqrt(D)).view(T, G, L)
            x = x.masked_fill(~see[:, None], -math.inf)
            if weights:
                w = torch.exp(x - s["lse"][a:b, h * G:(h + 1) * G, None].double()).sum((0, 1))
                at = torch.arange(L, device=DEV)
                old = score[blocks[at // bt], h, at % bt] * c["decay"]
                old[L - T:] = 0
                score[blocks[at // bt], h, at % bt] = old + w
                continue
            v = s["v_cache"][blocks, h].reshape(-1, D)[:L].double()
            y = torch.logsumexp(x, -1)
            lse[a:b, h * G:(h + 1) * G] = y
            p = torch.exp(x - y[..., None]).view(T * G, L)
            out[a:b, h * G:(h + 1) * G] = torch.matmul(p, v).view(T, G, D)
    return score if weights else (out, lse)


def _exact_evict(s, c):
    bt, B = c["bt"], c["budget"]
    k, v, so, po = s["k_cache"].double(), s["v_cache"].double(), s["score_out"].double(), s["pos_out"].clone()
    lens, nxt = s["lens"].tolist(), s["next_pos"].tolist()
    for r, L in enumerate(lens):
        at = torch.arange(L, device=DEV)
        blk, off = s["table"][r].long()[at // bt], at % bt
        for h in range(c["Hkv"]):
            sc, ps = s["score"][blk, h, off], s["pos"][blk, h, off]
            must = (ps < c["sink"]) | (ps >= nxt[r] - c["recent"])
            kept = torch.cat((at[must], at[~must][torch.sort(sc[~must], descending=True, stable=True)[1]]))[:B].sort()[0]
            stay, come = kept[kept < B], kept[kept >= B]
            hole = torch.ones(min(L, B), dtype=torch.bool, device=DEV)
            hole[stay] = False
            to = torch.cat((stay, torch.nonzero(hole)[:, 0]))
            frm = torch.cat((stay, come))
            so[blk[to], h, off[to]], po[blk[to], h, off[to]] = sc[frm].double(), ps[frm]
            k[blk[to], h, off[to]], v[blk[to], h, off[to]] = k[blk[frm], h, off[frm]], v[blk[frm], h, off[frm]]
    return k, v, so, po, None


def _exact_sample(s, c):
    logp = []
    par = zip(s["u"].tolist(), s["temperature"].tolist(), s["top_k"].tolist(), s["top_p"].tolist(), s["min_p"].tolist())
    for b, (u, t, k, p, mp) in enumerate(par):
        if t <= 0:
            logp.append(0.0)
            continue
        x = s["logits"][b].double()
        w = torch.softmax((x - x.max()) / t, 0)
        w = w / w.max()
        order = torch.sort(x, descending=True, stable=True)[1]
        order = order[:k] if k else order
        c2 = torch.cumsum(w[order], 0)
        if p < 1:
            order = order[:1 + int((c2[:-1] < p * c2[-1]).sum())]
        order = order[w[order] >= mp].sort()[0]
        c2 = torch.cumsum(w[order], 0)
        at = min(int((c2 <= u * c2[-1]).sum()), order.numel() - 1)
        logp.append(float(torch.log(w[order[at]] / c2[-1])))
    return None, torch.tensor(logp, dtype=torch.float64, device=DEV)


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["op"] in ("rope", "rope_append"):
        return _exact_rope(s, c)
    if c["op"] in ("attend", "weigh"):
        return _exact_attention(s, c, c["op"] == "weigh")
    return _exact_evict(s, c) if c["op"] == "evict" else _exact_sample(s, c)
