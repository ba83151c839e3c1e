"""Sizes at which the operators take another of their ways through the work:
more query rows than are staged at once, more rows of logits than compute
units, kept sets too large to be listed, requests whose lengths differ by far.
Against the same definitions in 64 bits, with the same tolerances (ops_ref.py)."""
import math

import pytest

torch = pytest.importorskip("torch")

import ops_ref as ref  # noqa: E402

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU-only hosts, never run there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_16336_amd import ops  # noqa: E402
from test_gpu_ops import BF, FL, HF, check_attend, cuda, draw_u, query  # noqa: E402


@pytest.mark.parametrize("D,G,dtype", [(64, 4, BF), (96, 3, HF), (128, 5, BF), (256, 2, HF)])
@pytest.mark.parametrize("decay,shape", [(0.0, "chain"), (0.9, "tree"), (1.0, "chain")])
def test_weigh_rows_in_several_passes(D, G, dtype, decay, shape):
    """Up to 90 new tokens a request: 270 query rows and more where 64 to 256 are staged at once; the first pass applies the
    decay, the later ones add."""
    lens, news = [700, 90, 400, 33], [90, 90, 64, 1]
    b = ref.make_batch(lens, news, 16, 2, D, dtype, seed=50 + D)
    tree = ref.random_tree(news, b["g"]) if shape == "tree" else None
    q = query(b, 2 * G, D, dtype)
    score = torch.rand(b["k"].shape[:3], generator=b["g"])
    if decay == 0.0:
        score[:] = math.nan  # not read
    lse = ref.attend(b, q, None, tree)[1].float()
    c = cuda(b)
    got = ops.weigh(q.cuda(), lse.cuda(), c["k"], c["table"], c["lens"], c["q_start"], b["max_q"], score.cuda(), decay=decay,
                    tree=None if tree is None else tree.cuda()).cpu()
    want, err = ref.weigh(b, q, lse, score, decay, None, tree)
    same = err == 0
    assert torch.equal(got[same].nan_to_num(-1.0), score[same].nan_to_num(-1.0))
    assert ((got.double() - want).abs()[~same] <= err[~same]).all()


@pytest.mark.parametrize("news", [[1] * 9, [30, 1, 48, 7, 26, 2, 40, 13, 48]])
def test_attend_lengths_that_differ_by_far(news):
    """One request has most of the slots: its keys are shared by many jobs, the others' by one or two."""
    lens = [9000, 40, 700, 64, 26, 3000, 129, 13, 1500]
    b = ref.make_batch(lens, news, 16, 2, 128, BF, seed=61)
    check_attend(b, query(b, 10, 128, BF), ref.random_tree(news, b["g"]) if max(news) > 1 else None)


@pytest.mark.parametrize("rows,V,dtype", [(300, 2003, BF), (257, 777, FL), (3, 30011, HF)])
def test_sample_large_kept_sets(rows, V, dtype):
    """Every mixture of the rules, on more and on fewer rows than compute units; flat rows whose kept sets pass what is
    listed, and rows of few distinct logits."""
    g = torch.Generator().manual_seed(V)
    x = (torch.randn(rows, V, generator=g) * torch.tensor([0.3, 1.0, 3.0])[torch.arange(rows) % 3, None]).to(dtype)
    x[1::7] = (x[1::7].float() * 2).round().to(dtype) / 2
    T = (0.5 + torch.rand(rows, generator=g)).float()
    kind = torch.arange(rows) % 5
    k = torch.where((kind == 1) | (kind == 4), torch.randint(1, V, (rows,), generator=g), 0)
    p = torch.where((kind == 2) | (kind == 4), 0.5 + 0.49 * torch.rand(rows, generator=g), 1.0)
    m = torch.where((kind == 3) | (kind == 4), 0.2 * torch.rand(rows, generator=g), 0.0)
    u, want, logp = [], [], []
    for r in range(rows):
        # limits in the middle between two ranks' sums, or two weights: the kept set does not hang on the last digit
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
    # as in test_sample: weights in 32 bits, the rest in 64
    assert (lp.cpu().double() - torch.tensor(logp, dtype=torch.float64)).abs().max() <= 2e-5


def test_sample_ends_of_the_range():
    """u = 0 draws the first kept token, u past every sum the last one, whichever way the row takes."""
    V = 5000
    g = torch.Generator().manual_seed(9)
    x = torch.randn(V, generator=g).float()
    rules = [(0, 1.0, 0.0), (40, 1.0, 0.0), (3000, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.05), (3000, 0.9, 0.01)]
    for k, p, m in rules:
        w = ref.kept_weights(x, 1.0, k, p, m)
        kept = torch.nonzero(w)[:, 0]
        for u, token in ((0.0, int(kept[0])), (1.0, int(kept[-1]))):
            one = lambda v, t=torch.float32: torch.tensor([v], dtype=t, device="cuda")  # noqa: E731
            tok, _ = ops.sample(x[None].cuda(), one(u), one(1.0), one(k, torch.int32), one(p), one(m))
            assert tok.item() == token, (k, p, m, u)
