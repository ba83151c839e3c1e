"""The operators of mts_ops.h against their definitions in 64 bits: sizes,
layouts, masks and contents at which they can go wrong.  Tolerances follow from
the roundings the header names (ops_ref.py)."""
import math

import pytest

torch = pytest.importorskip("torch")

import ops_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU-only hosts, never run there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_16336_amd import ops  # noqa: E402
from paper_2608_16336_amd.mts import MtsError  # noqa: E402

BF, HF, FL = torch.bfloat16, torch.float16, torch.float32


def cuda(b):
    """The batch on the GPU, with the strides it has."""
    out = dict(b)
    for x in ("k", "v"):
        s = b[x].stride()
        size = 1 + sum((d - 1) * t for d, t in zip(b[x].shape, s))
        flat = torch.empty(size, dtype=b[x].dtype, device="cuda")
        out[x] = flat.as_strided(b[x].shape, s)
        out[x].copy_(b[x])
    for x in ("table", "lens", "q_start"):
        out[x] = b[x].cuda()
    return out


def query(b, Hq, D, dtype, seed=1):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(int(b["q_start"][-1]), Hq, D, generator=g) * 1.5).to(dtype)


def run_attend(b, q, tree=None, **kw):
    c = cuda(b)
    out, lse = ops.attend(q.cuda(), c["k"], c["v"], c["table"], c["lens"], c["q_start"], b["max_q"],
                          tree=None if tree is None else tree.cuda(), **kw)
    return out.cpu(), lse.cpu()


def check_attend(b, q, tree=None, scale=None):
    out, lse = run_attend(b, q, tree, scale=scale)
    want, wlse, bound, lbound = ref.attend(b, q, scale, tree)
    assert torch.equal(torch.isneginf(lse), torch.isneginf(wlse))
    on = ~torch.isneginf(wlse)
    assert ((lse.double() - wlse).abs()[on] <= lbound[on]).all()
    err = (out.double() - want).abs()
    assert (err <= bound).all(), (err - bound).max()
    return out, lse


# ---------------------------------------------------------------- attend

SHAPES = [
    # lens, new tokens, block_tokens, kv heads, group, head dim, type
    ([1], [1], 16, 1, 1, 64, BF),
    ([2, 31, 32, 33], [1, 1, 1, 1], 16, 2, 4, 128, BF),
    ([127, 128, 129, 5], [1, 2, 3, 4], 16, 1, 4, 128, HF),
    ([40, 0, 17, 300], [1, 0, 1, 1], 8, 2, 7, 96, BF),
    ([65, 64, 63], [1, 1, 1], 64, 1, 5, 256, HF),
    ([9, 70, 200], [9, 16, 33], 1, 2, 1, 64, HF),
    ([50, 260], [3, 20], 2, 1, 8, 128, BF),
    ([150, 90], [64, 41], 32, 1, 4, 96, HF),
    ([130, 40], [70, 40], 16, 1, 2, 256, BF),
]


@pytest.mark.parametrize("lens,news,bt,Hkv,G,D,dtype", SHAPES)
@pytest.mark.parametrize("shape", ["chain", "tree"])
def test_attend(lens, news, bt, Hkv, G, D, dtype, shape):
    b = ref.make_batch(lens, news, bt, Hkv, D, dtype, seed=len(lens) + bt)
    tree = ref.random_tree(news, b["g"]) if shape == "tree" else None
    check_attend(b, query(b, Hkv * G, D, dtype), tree)


@pytest.mark.parametrize("lens,news,G,D", [([5000], [1], 4, 128), ([4097, 3000], [1, 2], 3, 64), ([2500], [12], 4, 128),
                                           ([1700, 40], [140, 40], 2, 64)])
def test_attend_long_split(lens, news, G, D):
    """Keys of one request over many workgroups, joined again."""
    b = ref.make_batch(lens, news, 16, 1, D, BF, seed=3)
    check_attend(b, query(b, G, D, BF))


def test_attend_many_requests():
    """More requests than one workgroup looks over at once, some without slots or without new tokens."""
    lens = [(7 * r) % 41 for r in range(531)]
    news = [0 if r % 13 == 0 else min(lens[r], 1 + r % 3) for r in range(531)]
    b = ref.make_batch(lens, news, 16, 1, 64, HF, seed=4)
    check_attend(b, query(b, 2, 64, HF))


def test_attend_sees_nothing():
    """Rows whose mask leaves nothing: no slot before them and no bit of their own."""
    news = [3, 5, 2]
    b = ref.make_batch([3, 5, 40], news, 16, 2, 64, BF, seed=5)
    tree = ref.random_tree(news, b["g"])
    tree[1] = 0
    tree[4] = 0
    tree[9] = 0  # has its request's earlier slots
    out, lse = check_attend(b, query(b, 4, 64, BF), tree)
    assert (out[[1, 4]] == 0).all() and torch.isneginf(lse[[1, 4]]).all()


def test_attend_fewer_slots_than_new_tokens():
    """lens counts the new tokens; where it is smaller, the first of them have no slot."""
    b = ref.make_batch([2, 0, 1], [4, 3, 1], 16, 1, 64, BF, seed=6)
    out, lse = check_attend(b, query(b, 2, 64, BF))
    assert (out[:2] == 0).all() and (out[4:7] == 0).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("news,G,D", [([6, 7], 2, 64), ([40, 33], 4, 128), ([3, 2], 3, 256)])
def test_attend_masked_values_do_not_leak(bad, news, G, D):
    """What a drafted token holds reaches only the rows that see it."""
    b = ref.make_batch([60, 45], news, 16, 2, D, BF, seed=7)
    tree = ref.random_tree(news, b["g"])
    # the last drafted token of each request is nobody's ancestor: a row of its own
    clean, _ = run_attend(b, query(b, 2 * G, D, BF), tree)
    rows = torch.ones(sum(news), dtype=torch.bool)
    for r, T in enumerate(news):
        j = int(b["lens"][r]) - 1
        blk = int(b["table"][r, j // 16])
        b["v"][blk, 1, j % 16, 5] = bad
        b["k"][blk, 1, j % 16, 3] = bad
        rows[int(b["q_start"][r + 1]) - 1] = False
    out, lse = run_attend(b, query(b, 2 * G, D, BF), tree)
    want, _, bound, _ = ref.attend(b, query(b, 2 * G, D, BF), None, tree)
    assert torch.isfinite(out[rows].float()).all() and torch.isfinite(lse[rows]).all()
    err = (out.double() - want).abs()[rows]
    assert (err <= bound[rows]).all()
    # the other KV head saw nothing of it
    assert torch.equal(out[:, :G], clean[:, :G])


def test_attend_seen_infinity_arrives():
    """An infinite value that a row does see is in its output."""
    b = ref.make_batch([20], [3], 16, 1, 64, HF, seed=8)
    j = 18  # the second new token
    b["v"][int(b["table"][0, 1]), 0, j % 16, 7] = math.inf
    out, _ = run_attend(b, query(b, 2, 64, HF))
    assert torch.isfinite(out[0].float()).all()
    assert torch.isposinf(out[1:, :, 7]).all() and torch.isfinite(out[1:, :, 8:].float()).all()


def test_attend_large_scores():
    """Scores far beyond what exp takes without its maximum, of both signs."""
    b = ref.make_batch([90, 33], [2, 1], 16, 1, 64, BF, seed=9)
    check_attend(b, query(b, 4, 64, BF) * 60)
    check_attend(b, query(b, 4, 64, BF), scale=-0.3)
    check_attend(b, query(b, 4, 64, BF), scale=0.0)


@pytest.mark.parametrize("layout", ["bthd", "kv"])
@pytest.mark.parametrize("news", [[1, 1, 1], [17, 40, 25]])
def test_attend_strided(layout, news):
    """Token-major pools, keys and values side by side, queries and outputs that are slices."""
    D, G = 128, 4
    b = ref.make_batch([100, 47, 333], news, 16, 2, D, BF, seed=10, layout=layout)
    N = sum(news)
    wide = torch.randn(N, 3, 2 * G, D + 8, generator=b["g"]).to(BF)
    q = wide[:, 1, :, 8:]
    big = torch.zeros(2 * G, N, D, dtype=BF, device="cuda")
    c = cuda(b)
    gq = wide.cuda()[:, 1, :, 8:]
    out, lse = ops.attend(gq, c["k"], c["v"], c["table"], c["lens"], c["q_start"], b["max_q"], out=big.transpose(0, 1))
    want, wlse, bound, lbound = ref.attend(b, q)
    assert ((out.cpu().double() - want).abs() <= bound).all()
    assert ((lse.cpu().double() - wlse).abs() <= lbound).all()


def test_attend_holes_in_the_table():
    """Block ids outside the pool leave their slots unseen."""
    b = ref.make_batch([100, 60], [2, 1], 16, 1, 64, BF, seed=11)
    b["table"][0, 2] = -1
    b["table"][0, 5] = b["k"].shape[0]
    b["table"][1, :4] = 1 << 30
    check_attend(b, query(b, 2, 64, BF))


def test_attend_lens_past_the_table():
    """Lengths are clamped to what the table holds."""
    b = ref.make_batch([64], [1], 16, 1, 64, BF, seed=12)
    b["table"] = b["table"][:, :4].contiguous()
    q = query(b, 2, 64, BF)
    want, _ = run_attend(b, q)
    b["lens"] += 1000
    out, _ = run_attend(b, q)
    assert torch.equal(out, want)


def test_attend_offsets_past_32_bits():
    """A pool whose blocks lie more than 2^32 bytes apart."""
    D, bt, stride = 64, 16, 3 * 2 ** 28
    flat = torch.empty(8 * stride, dtype=BF, device="cuda")
    shape = (8, 1, bt, D)
    k = flat.as_strided(shape, (stride, bt * D, D, 1))
    v = flat.as_strided(shape, (stride, bt * D, D, 1), stride // 2)
    b = ref.make_batch([70, 30], [1, 1], bt, 1, D, BF, seed=13, spare=1)
    assert b["k"].shape[0] == 8
    k.copy_(b["k"])
    v.copy_(b["v"])
    c = cuda(b)
    q = query(b, 4, D, BF)
    out, _ = ops.attend(q.cuda(), k, v, c["table"], c["lens"], c["q_start"], 1)
    want, _, bound, _ = ref.attend(b, q)
    assert ((out.cpu().double() - want).abs() <= bound).all()


def test_attend_twice_the_same_and_on_another_stream():
    """Splits are joined in their own order: repeated calls agree bit for bit, also beside another stream's."""
    b = ref.make_batch([3000, 700, 1500], [1, 4, 2], 16, 2, 128, BF, seed=14)
    c, q = cuda(b), query(b, 8, 128, BF).cuda()
    call = lambda: ops.attend(q, c["k"], c["v"], c["table"], c["lens"], c["q_start"], 4)  # noqa: E731
    first, lse = call()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    outs = []
    for _ in range(10):
        outs.append(call())
        with torch.cuda.stream(s):
            outs.append(call())
    torch.cuda.synchronize()
    for o, l in outs:
        assert torch.equal(o, first) and torch.equal(l, lse)


def test_attend_workspace_serves_calls_of_other_sizes():
    """One workspace for large and small calls in turn."""
    big = ref.make_batch([2000] * 6, [12] * 6, 16, 2, 64, BF, seed=15)
    small = ref.make_batch([900], [1], 16, 2, 64, BF, seed=16)
    ws = torch.full((ops.attend_workspace(6, 72, 12, 8, 2, 64),), 255, dtype=torch.uint8, device="cuda")
    qb, qs = query(big, 8, 64, BF), query(small, 8, 64, BF)
    want_b, want_s = run_attend(big, qb)[0], run_attend(small, qs)[0]
    for _ in range(3):
        assert torch.equal(run_attend(big, qb, workspace=ws)[0], want_b)
        assert torch.equal(run_attend(small, qs, workspace=ws)[0], want_s)


def test_attend_in_a_graph():
    """Captured and replayed with other contents, lengths and tables, against the eager call."""
    b = ref.make_batch([700, 90], [1, 3], 16, 2, 64, BF, seed=17)
    c, q = cuda(b), query(b, 8, 64, BF).cuda()
    score = torch.zeros(b["k"].shape[:3], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        ops.attend(q, c["k"], c["v"], c["table"], c["lens"], c["q_start"], 3)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = ops.attend(q, c["k"], c["v"], c["table"], c["lens"], c["q_start"], 3)
        ops.weigh(q, lse, c["k"], c["table"], c["lens"], c["q_start"], 3, score, decay=0.0)
    for turn in range(4):
        q.copy_(query(b, 8, 64, BF, seed=20 + turn))
        c["lens"].copy_(torch.tensor([700 - 151 * turn, 90 - 20 * turn], dtype=torch.int32))
        score.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        eager, elo = ops.attend(q, c["k"], c["v"], c["table"], c["lens"], c["q_start"], 3)
        again = ops.weigh(q, elo, c["k"], c["table"], c["lens"], c["q_start"], 3, torch.full_like(score, 7.0), decay=0.0)
        assert torch.equal(out, eager) and torch.equal(lse, elo) and torch.equal(score, again)


# ---------------------------------------------------------------- weigh


@pytest.mark.parametrize("lens,news,bt,Hkv,G,D,dtype", SHAPES)
@pytest.mark.parametrize("decay,shape", [(0.9, "chain"), (0.0, "tree"), (1.0, "tree")])
def test_weigh(lens, news, bt, Hkv, G, D, dtype, decay, shape):
    b = ref.make_batch(lens, news, bt, Hkv, D, dtype, seed=30 + bt)
    tree = ref.random_tree(news, b["g"]) if shape == "tree" else None
    q = query(b, Hkv * G, D, dtype)
    score = torch.rand(b["k"].shape[:3], generator=b["g"])
    if decay == 0.0:
        score[:] = math.nan  # not read
    lse = ref.attend(b, q, None, tree)[1].float()
    c = cuda(b)
    got = ops.weigh(q.cuda(), lse.cuda(), c["k"], c["table"], c["lens"], c["q_start"], b["max_q"], score.cuda(),
                    decay=decay, tree=None if tree is None else tree.cuda()).cpu()
    want, err = ref.weigh(b, q, lse, score, decay, None, tree)
    same = err == 0
    assert torch.equal(got[same].nan_to_num(-1.0), score[same].nan_to_num(-1.0))
    assert ((got.double() - want).abs()[~same] <= err[~same]).all()


def test_weigh_sums_to_the_rows():
    """The weights of a row sum to one: a request's new weight is its number of rows."""
    b = ref.make_batch([700, 33], [5, 2], 16, 2, 128, BF, seed=40)
    c, q = cuda(b), query(b, 8, 128, BF).cuda()
    lse = ops.attend(q, c["k"], c["v"], c["table"], c["lens"], c["q_start"], 5)[1]
    score = ops.weigh(q, lse, c["k"], c["table"], c["lens"], c["q_start"], 5, torch.zeros(b["k"].shape[:3], device="cuda")).cpu()
    for r, rows in ((0, 5 * 4), (1, 2 * 4)):
        for h in range(2):
            x, _ = ref.rows_of(b, r, score[..., None], h)
            assert abs(float(x.double().sum()) - rows) < 1e-4 * rows


def test_weigh_empty_rows_and_nan_slots():
    """Rows that saw nothing add nothing; a masked slot's NaN key reaches no other slot."""
    news = [3, 4]
    b = ref.make_batch([3, 50], news, 16, 1, 64, BF, seed=41)
    tree = ref.random_tree(news, b["g"])
    tree[1] = 0
    q = query(b, 2, 64, BF)
    lse = ref.attend(b, q, None, tree)[1].float()
    j = 49
    b["k"][int(b["table"][1, j // 16]), 0, j % 16, 0] = math.nan
    score = torch.zeros(b["k"].shape[:3])
    c = cuda(b)
    got = ops.weigh(q.cuda(), lse.cuda(), c["k"], c["table"], c["lens"], c["q_start"], 4, score.cuda(), tree=tree.cuda()).cpu()
    x, _ = ref.rows_of(b, 1, got[..., None], 0)
    assert torch.isfinite(x[:49]).all()
    x0, _ = ref.rows_of(b, 0, got[..., None], 0)
    assert torch.isfinite(x0).all()


# ---------------------------------------------------------------- evict


def evict_inputs(b, seed, kind="random"):
    g = torch.Generator().manual_seed(seed)
    shape = b["k"].shape[:3]
    score = torch.randn(shape, generator=g)
    if kind == "ties":
        score = (score * 2).round() / 2  # also -0 and 0
    if kind == "special":
        pick = torch.randint(0, 6, shape, generator=g)
        for i, x in enumerate((math.nan, math.inf, -math.inf, 0.0, -0.0)):
            score[pick == i] = x
    pos = torch.zeros(shape, dtype=torch.int32)
    nxt = []
    for r, L in enumerate(b["lens"].tolist()):
        order = torch.randperm(L + 10, generator=g)[:L].int()  # an earlier eviction left gaps and another order
        j = torch.arange(L)
        ok = b["table"][r].long()[j // b["bt"]].clamp(0, b["k"].shape[0] - 1)
        pos[ok, :, j % b["bt"]] = order[:, None]
        nxt.append(L + 10)
    return score, pos, torch.tensor(nxt, dtype=torch.int32)


@pytest.mark.parametrize("lens,budget,recent,sink,bt,Hkv,D,dtype,kind", [
    ([1, 2, 3], 1, 0, 0, 16, 1, 64, BF, "random"),
    ([40, 64, 65, 0, 200], 64, 8, 2, 16, 2, 128, BF, "random"),
    ([300, 17, 129], 33, 5, 1, 8, 3, 96, HF, "ties"),
    ([500, 100], 64, 0, 0, 32, 1, 64, BF, "ties"),
    ([257, 90], 80, 16, 4, 64, 2, 256, HF, "special"),
    ([90, 91], 20, 60, 3, 1, 1, 64, BF, "random"),       # more kept first than the budget
    ([90, 91], 89, 200, 0, 4, 1, 64, BF, "random"),      # all kept first: the lowest slots
    ([2500, 2100], 1100, 32, 4, 16, 1, 64, BF, "special"),
    ([4200], 17, 3, 1, 16, 1, 64, BF, "random"),
])
@pytest.mark.parametrize("in_place", [True, False])
def test_evict(lens, budget, recent, sink, bt, Hkv, D, dtype, kind, in_place):
    b = ref.make_batch(lens, [0] * len(lens), bt, Hkv, D, dtype, seed=50 + budget)
    score, pos, nxt = evict_inputs(b, 60, kind)
    k, v, s, ps, want_lens = ref.evict(b, score, pos, nxt, budget, recent, sink)
    c = cuda(b)
    gs, gp = score.cuda(), pos.cuda()
    so, po = (gs, gp) if in_place else (torch.full_like(gs, 9.0), torch.full_like(gp, -9))
    got = ops.evict(c["k"], c["v"], gs, gp, c["table"], c["lens"], nxt.cuda(), budget, recent=recent, sink=sink,
                    score_out=so, pos_out=po)
    assert torch.equal(got.cpu(), want_lens)
    bits = lambda t: t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)  # noqa: E731
    assert torch.equal(bits(c["k"].cpu()), bits(k)) and torch.equal(bits(c["v"].cpu()), bits(v))
    so, po = so.cpu(), po.cpu()
    for r in range(len(lens)):
        for h in range(Hkv):
            cut = dict(b, lens=want_lens)
            for a, z in ((so, s), (po, ps)):
                assert torch.equal(bits(ref.rows_of(cut, r, a[..., None], h)[0]), bits(ref.rows_of(cut, r, z[..., None], h)[0]))
    if in_place:
        assert torch.equal(bits(so), bits(s)) and torch.equal(po, ps)
    else:
        assert torch.equal(bits(gs.cpu()), bits(score)) and torch.equal(gp.cpu(), pos)


def test_evict_holes_in_the_table():
    """Slots outside the pool are given up first and nothing is copied to them."""
    b = ref.make_batch([100], [0], 16, 2, 64, BF, seed=70)
    score, pos, nxt = evict_inputs(b, 71)
    b["table"][0, 1] = -1
    b["table"][0, 4] = b["k"].shape[0] + 5
    k, v, s, ps, lens = ref.evict(b, score, pos, nxt, 40, 4, 1)
    c, gs, gp = cuda(b), score.cuda(), pos.cuda()
    got = ops.evict(c["k"], c["v"], gs, gp, c["table"], c["lens"], nxt.cuda(), 40, recent=4, sink=1)
    assert torch.equal(got.cpu(), lens)
    assert torch.equal(c["k"].cpu().view(torch.int16), k.view(torch.int16)) and torch.equal(gs.cpu(), s) and torch.equal(gp.cpu(), ps)


def test_evict_token_major_pool():
    b = ref.make_batch([120, 77], [0, 0], 16, 2, 64, HF, seed=72, layout="bthd")
    score, pos, nxt = evict_inputs(b, 73)
    k, v, s, ps, lens = ref.evict(b, score, pos, nxt, 50, 4, 1)
    c, gs, gp = cuda(b), score.cuda(), pos.cuda()
    ops.evict(c["k"], c["v"], gs, gp, c["table"], c["lens"], nxt.cuda(), 50, recent=4, sink=1)
    for a, z in ((c["k"], k), (c["v"], v)):
        assert torch.equal(a.cpu().contiguous().view(torch.int16), z.contiguous().view(torch.int16))
    assert torch.equal(gs.cpu(), s) and torch.equal(gp.cpu(), ps)


def test_attention_after_eviction_is_that_of_the_kept():
    """Attending the compacted slots equals attending the kept ones where they were."""
    b = ref.make_batch([200], [1], 16, 1, 64, HF, seed=74, poison=False)
    score, pos, nxt = evict_inputs(b, 75)
    pos = torch.zeros_like(pos)
    j = torch.arange(200)
    pos[b["table"][0].long()[j // 16], :, j % 16] = j.int()[:, None]
    nxt[:] = 200
    q = query(b, 4, 64, HF)
    c = cuda(b)
    gs = score.cuda()
    lens = ops.evict(c["k"], c["v"], gs, pos.cuda(), c["table"], c["lens"], nxt.cuda(), 90, recent=8, sink=2)
    out, _ = ops.attend(q.cuda(), c["k"], c["v"], c["table"], lens, c["q_start"], 1)
    kk, _ = ref.rows_of(b, 0, b["k"], 0)
    vv, _ = ref.rows_of(b, 0, b["v"], 0)
    ss, _ = ref.rows_of(b, 0, score[..., None], 0)
    first = (j < 2) | (j >= 192)
    rest = j[~first][torch.sort(ss[~first, 0], descending=True, stable=True)[1]]
    keep = torch.cat((j[first], rest))[:90]
    kept = dict(k=kk[keep].view(1, 1, 90, 64), v=vv[keep].view(1, 1, 90, 64), table=torch.zeros(1, 1, dtype=torch.int32),
                lens=torch.tensor([90], dtype=torch.int32), q_start=b["q_start"], bt=90)
    # the newest slot need not be the last one after the eviction: the one new token sees every slot either way
    want, _, bound, _ = ref.attend(kept, q)
    assert ((out.cpu().double() - want).abs() <= bound).all()


# ---------------------------------------------------------------- sample


def draw_u(w, g):
    """A uniform number in the middle of a kept token's share, and that token."""
    c = torch.cumsum(w, 0)
    at = int(torch.multinomial(w, 1, generator=g))
    return float((c[at] - w[at] / 2) / c[-1]), at


@pytest.mark.parametrize("V,dtype", [(1, FL), (2, BF), (7, HF), (63, FL), (1000, BF), (1025, HF), (4099, FL), (20011, BF), (70001, FL)])
@pytest.mark.parametrize("rule", ["all", "k", "p", "min_p", "kp", "kpm"])
def test_sample(V, dtype, rule):
    g = torch.Generator().manual_seed(V + len(rule))
    rows = 12
    x = (torch.randn(rows, V, generator=g) * 2).to(dtype)
    x[:, torch.randint(0, V, (min(V, 9),), generator=g)] += 6
    T = (0.5 + torch.rand(rows, generator=g)).float()
    k = torch.randint(1, max(2, min(V, 300)), (rows,), generator=g) if "k" in rule else torch.zeros(rows, dtype=torch.int64)
    p = (0.3 + 0.65 * torch.rand(rows, generator=g)) if "p" in rule and rule != "min_p" else torch.ones(rows)
    m = 0.3 * torch.rand(rows, generator=g) if rule in ("min_p", "kpm") else torch.zeros(rows)
    u, want, logp = [], [], []
    for r in range(rows):
        # the limit of top_p in the middle between two ranks' sums: the kept set does not hang on the last digit
        w = ref.kept_weights(x[r], float(T[r]), int(k[r]), 1.0, 0.0)
        s = torch.cumsum(torch.sort(w[w > 0], descending=True)[0], 0) / w.sum()
        if p[r] < 1:
            i = int((s < float(p[r])).sum())
            lo = float(s[i - 1]) if i else 0.0
            p[r] = 0.5 * (lo + float(s[i])) if i < s.numel() else 0.5 * lo
        w = ref.kept_weights(x[r], float(T[r]), int(k[r]), float(p[r]), 0.0)
        if m[r] > 0:
            v = torch.unique(w[w > 0])
            i = int((v < float(m[r])).sum())
            m[r] = 0.5 * ((float(v[i - 1]) if i else 0.0) + float(v[i]))
        w = ref.kept_weights(x[r], float(T[r]), int(k[r]), float(p[r]), float(m[r]))
        ur, at = draw_u(w, g)
        u.append(ur)
        want.append(at)
        logp.append(float(torch.log(w[at] / w.sum())))
    tok, lp = ops.sample(x.cuda(), torch.tensor(u).cuda(), T.cuda(), k.int().cuda(), p.float().cuda(), m.float().cuda())
    assert tok.tolist() == want
    # weights in 32 bits (argument and exponential: a few units of arguments up to 60), the rest in 64
    assert (lp.cpu().double() - torch.tensor(logp, dtype=torch.float64)).abs().max() <= 2e-5


def params(rows, T=1.0, k=0, p=1.0, m=0.0, u=0.5):
    f = lambda v: torch.full((rows,), float(v), device="cuda")  # noqa: E731
    return f(u), f(T), torch.full((rows,), int(k), dtype=torch.int32, device="cuda"), f(p), f(m)


def test_sample_greedy_and_ties():
    """Temperature 0 takes the lowest index of the largest logit; top-k cuts equal logits by index, -0 equals 0."""
    x = torch.zeros(3, 500)
    x[0, [123, 77, 400]] = 5.0
    x[1, 10] = -0.0
    x[2] = -3.0
    u, T, k, p, m = params(3, T=0.0)
    tok, lp = ops.sample(x.cuda(), u, T, k, p, m)
    assert tok.tolist() == [77, 0, 0] and lp.tolist() == [0.0, 0.0, 0.0]
    # of 500 equal logits the first 10 are kept, or the first ones up to a share
    for kw, n in ((dict(k=10), 10), (dict(p=0.101), 51), (dict(k=40, p=0.5), 20), (dict(k=40, p=0.26), 11)):
        for i in (0, n // 2, n - 1):
            u, T, k, p, m = params(3, u=(i + 0.5) / n, **kw)
            tok, lp = ops.sample(x[2:].expand(3, 500).cuda().contiguous(), u, T, k, p, m)
            assert tok.tolist() == [i] * 3
            assert (lp.cpu() + math.log(n)).abs().max() < 1e-6


def test_sample_special_logits():
    """NaN and -inf are never drawn, +inf takes all, a row of nothing gives -1."""
    V = 3001
    x = torch.full((6, V), -math.inf)
    x[0] = math.nan
    x[2, 7] = 1.0
    x[3, [5, 2000]] = math.inf
    x[3, 100:900] = 4.0
    x[4] = torch.randn(V, generator=torch.Generator().manual_seed(1))
    x[4, ::2] = math.nan
    x[5, 1234] = -3.0e38
    for kw in (dict(), dict(k=3), dict(p=0.9), dict(m=0.5), dict(k=2000, p=0.5, m=0.1)):
        for u in (0.0, 0.25, 0.75, 1.0 - 2.0 ** -24):
            tok, lp = ops.sample(x.cuda(), *params(6, u=u, **kw))
            tok, lp = tok.tolist(), lp.tolist()
            assert tok[0] == tok[1] == -1 and lp[0] == lp[1] == -math.inf
            assert tok[2] == 7 and lp[2] == 0.0 and tok[5] == 1234
            want = 5 if kw.get("p", 1) < 0.51 or u < 0.5 else 2000
            assert tok[3] == want, (kw, u)
            assert tok[4] % 2 == 1 and 0 <= tok[4] < V


def test_sample_out_of_range_parameters():
    """Parameters past their ends count as the ends: the kept set is never empty and a token is always written."""
    V = 1000
    x = torch.randn(4, V, generator=torch.Generator().manual_seed(2))
    best = x.argmax(1).tolist()
    for kw in (dict(p=0.0), dict(p=-1.0), dict(m=1.0), dict(m=7.0), dict(k=1), dict(T=1e-30), dict(T=-2.0), dict(T=math.nan)):
        tok, _ = ops.sample(x.cuda(), *params(4, u=0.9, **kw))
        assert tok.tolist() == best, kw
    for kw in (dict(u=1.0), dict(u=5.0), dict(u=-3.0), dict(u=math.nan), dict(p=math.nan), dict(m=math.nan), dict(m=-1.0), dict(k=-5),
               dict(k=V), dict(k=V + 1), dict(p=2.0)):
        tok, lp = ops.sample(x.cuda(), *params(4, **kw))
        assert all(0 <= t < V for t in tok.tolist()), kw
        assert torch.isfinite(lp).all()


def test_sample_strided_rows_and_shares():
    """Rows of a larger matrix at odd offsets; frequencies over a grid of u are the kept shares."""
    base = torch.randn(5, 1013, generator=torch.Generator().manual_seed(3)).to(BF)
    big = base.cuda()
    x = big[:, 3:604]
    n = 5
    tok, _ = ops.sample(x, *params(n, T=0.0))
    assert tok.tolist() == base[:, 3:604].float().argmax(1).tolist()
    row = torch.tensor([0.0, 1.0, 2.0, 3.0, -1.0])
    grid = 4000
    u = (torch.arange(grid) + 0.5) / grid
    tok, _ = ops.sample(row.expand(grid, 5).contiguous().cuda(), u.cuda(), *params(grid, k=4)[1:])
    share = torch.bincount(tok.cpu().long(), minlength=5) / grid
    assert (share - torch.tensor([*torch.softmax(row[:4], 0).tolist(), 0.0])).abs().max() <= 1.0 / grid
    assert (tok.cpu().diff() >= 0).all()


# ---------------------------------------------------------------- rope


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("D,rot,dtype", [(64, 64, BF), (128, 64, HF), (128, 128, FL), (96, 10, BF), (96, 30, FL), (64, 2, HF), (256, 256, BF),
                                         (80, 48, HF)])
def test_rope(layout, D, rot, dtype):
    g = torch.Generator().manual_seed(D + rot)
    n, Hq, Hkv = 37, 5, 2
    q, k = (torch.randn(n, h, D, generator=g).to(dtype) for h in (Hq, Hkv))
    pos = torch.randint(0, 1 << 20, (n,), generator=g).int()
    pos[0], pos[1] = 0, (1 << 31) - 1
    f = ops.rope_freqs(rot, base=10000.0, scaling="parts", factor=8.0)
    for inverse in (False, True):
        oq, ok = ops.rope(q.cuda(), k.cuda(), pos.cuda(), f, layout=layout, mscale=1.25, inverse=inverse)
        for got, x in ((oq, q), (ok, k)):
            want = ref.rope(x, pos, f.cpu(), layout, 1.25, inverse)
            # sine and cosine to a few units of 32 bits, two products and a sum, the result rounded to the type; 64-bit
            # angles of 2^31 turns keep 2^-22
            size = 1.25 * x.double().abs().amax(-1, keepdim=True) * 2
            bound = ref.ROUND[dtype] * want.abs() + 2.0 ** -20 * size
            assert ((got.cpu().double() - want).abs() <= bound).all()
            assert torch.equal(got.cpu()[..., rot:], x[..., rot:])


def test_rope_in_place_alone_and_back():
    g = torch.Generator().manual_seed(5)
    q = torch.randn(9, 3, 64, generator=g).cuda()
    pos = torch.arange(9, dtype=torch.int32, device="cuda") * 1000
    f = ops.rope_freqs(64)
    want, none = ops.rope(q, None, pos, f)
    assert none is None
    x = q.clone()
    got, _ = ops.rope(x, None, pos, f, q_out=x)
    assert got is x and torch.equal(x, want)
    _, kk = ops.rope(None, q, pos, f)
    assert torch.equal(kk, want)
    back, _ = ops.rope(want, None, pos, f, inverse=True)
    assert (back - q).abs().max() <= 2.0 ** -20 * 8


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_gradient(layout):
    """The inverse rotation is the gradient: against the formula's transposed product and against differences."""
    g = torch.Generator().manual_seed(6)
    x, d, w = (torch.randn(4, 2, 32, generator=g, dtype=torch.float64) for _ in range(3))
    pos = torch.tensor([0, 3, 500, 70000], dtype=torch.int32)
    f = ops.rope_freqs(24)
    grad, _ = ops.rope(w.float().cuda(), None, pos.cuda(), f, layout=layout, mscale=1.1, inverse=True)
    xx = x.clone().requires_grad_(True)
    (ref.rope(xx, pos, f.cpu(), layout, 1.1) * w).sum().backward()
    assert (grad.cpu().double() - xx.grad).abs().max() <= 2.0 ** -19 * 8
    up, down = (ref.rope(x + e * d, pos, f.cpu(), layout, 1.1) for e in (1e-4, -1e-4))
    slope = float(((up - down) * w).sum()) / 2e-4
    assert abs(float((grad.cpu().double() * d).sum()) - slope) <= 1e-4 * float((w.abs() * d.abs()).sum())


@pytest.mark.parametrize("bt,dtype", [(16, BF), (1, HF), (64, BF)])
def test_rope_append(bt, dtype):
    g = torch.Generator().manual_seed(7)
    n, Hq, Hkv, D = 41, 6, 3, 64
    qkv = torch.randn(n, (Hq + 2 * Hkv) * D, generator=g).to(dtype)
    gq = qkv.cuda()
    cut = lambda t: (t[:, :Hq * D].view(n, Hq, D), t[:, Hq * D:(Hq + Hkv) * D].view(n, Hkv, D), t[:, (Hq + Hkv) * D:].view(n, Hkv, D))  # noqa: E731
    blocks = -(-n // bt) + 2
    slots = torch.randperm(blocks * bt, generator=g)[:n]
    slots[5], slots[6], slots[7] = -1, blocks * bt, 1 << 40
    pos = torch.randint(0, 5000, (n,), generator=g).int()
    f = ops.rope_freqs(D)
    kc, vc = (torch.full((blocks, Hkv, bt, D), 3.0, dtype=dtype, device="cuda") for _ in range(2))
    pc = torch.full((blocks, Hkv, bt), -5, dtype=torch.int32, device="cuda")
    out = ops.rope_append(*cut(gq), pos.cuda(), slots.cuda(), f, kc, vc, pc)
    wq, wk = ops.rope(cut(gq)[0], cut(gq)[1], pos.cuda(), f)
    assert torch.equal(out, wq)
    ek, ev, ep = (torch.full_like(kc, 3.0), torch.full_like(vc, 3.0), torch.full_like(pc, -5))
    for t in range(n):
        s = int(slots[t])
        if 0 <= s < blocks * bt:
            ek[s // bt, :, s % bt], ev[s // bt, :, s % bt], ep[s // bt, :, s % bt] = wk[t], cut(gq)[2][t], pos[t]
    assert torch.equal(kc, ek) and torch.equal(vc, ev) and torch.equal(pc, ep)


# ---------------------------------------------------------------- refusals


def test_refusals():
    b = ref.make_batch([20], [1], 16, 1, 64, BF)
    c, q = cuda(b), query(b, 2, 64, BF).cuda()
    ok = (q, c["k"], c["v"], c["table"], c["lens"], c["q_start"], 1)
    ops.attend(*ok)
    change = lambda i, x: ok[:i] + (x,) + ok[i + 1:]  # noqa: E731
    for bad in (change(0, q.half()), change(0, q.cpu()), change(0, q[..., :32]), change(1, c["k"].float()), change(2, c["v"][:1]),
                change(3, c["table"].long()), change(4, c["lens"].long()), change(5, c["q_start"][:1]), change(0, q.transpose(1, 2))):
        with pytest.raises((ValueError, MtsError)):
            ops.attend(*bad)
    odd = torch.zeros(2000, dtype=BF, device="cuda")[1:129].view(1, 2, 64)
    for bad in (change(0, odd), change(6, 0), change(0, torch.zeros(1, 3, 64, dtype=BF, device="cuda")[:, :0])):
        with pytest.raises(MtsError) as e:
            ops.attend(*bad)
        assert e.value.code == -1
    with pytest.raises(MtsError):
        ops.attend(*ok, scale=math.nan)
    with pytest.raises(MtsError) as e:
        ops.attend(*ok, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == -2
    with pytest.raises(ValueError):
        ops.attend(*ok, tree=torch.zeros(2, 1, dtype=torch.int64, device="cuda"))
    score, pos = torch.zeros(c["k"].shape[:3], device="cuda"), torch.zeros(c["k"].shape[:3], dtype=torch.int32, device="cuda")
    with pytest.raises(MtsError):
        ops.evict(c["k"], c["v"], score, pos, c["table"], c["lens"], c["lens"], 4, lens_out=c["lens"])
    with pytest.raises(MtsError):
        ops.evict(c["k"], c["v"], score, pos, c["table"], c["lens"], c["lens"], 0)
    with pytest.raises(ValueError):
        ops.evict(c["k"], c["v"], score[:1], pos, c["table"], c["lens"], c["lens"], 4)
    with pytest.raises(MtsError):
        ops.weigh(q, torch.zeros(1, 2, device="cuda"), c["k"], c["table"], c["lens"], c["q_start"], 1, score, decay=2.0)
    x = torch.zeros(2, 8, device="cuda")
    with pytest.raises(ValueError):
        ops.sample(x, *params(3))
    with pytest.raises(ValueError):
        ops.sample(x.t(), *params(8))
    with pytest.raises(ValueError):
        ops.rope(q, None, c["lens"].long(), ops.rope_freqs(64))
    with pytest.raises(MtsError):
        ops.rope(q, None, c["lens"], torch.zeros(33, dtype=torch.float64, device="cuda"))
    with pytest.raises(KeyError):
        ops.rope(q, None, c["lens"], ops.rope_freqs(64), layout="other")


def test_nothing_to_do():
    """Calls without requests, tokens or rows do nothing."""
    k = torch.zeros(2, 1, 16, 64, dtype=BF, device="cuda")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.zeros(0, 2, 64, dtype=BF, device="cuda")
    out, lse = ops.attend(q, k, k, i32(0, 1), i32(0), i32(1), 1)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
    score = torch.ones(2, 1, 16, device="cuda")
    ops.weigh(q, lse, k, i32(0, 1), i32(0), i32(1), 1, score, decay=0.5)
    assert (score == 1).all()
    assert ops.evict(k, k, score, i32(2, 1, 16), i32(0, 1), i32(0), i32(0), 4).shape == (0,)
    tok, _ = ops.sample(torch.zeros(0, 10, device="cuda"), *params(0))
    assert tok.shape == (0,)
    f = ops.rope_freqs(64)
    a, b = ops.rope(q, q[:, :1], i32(0), f)
    assert a.shape == q.shape
