"""The operators together, as one instance runs them: tick by tick against the
whole layer computed from the token sequence, without a cache, in 64 bits."""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on CPU-only hosts, never run there
    pytest.skip("needs a GPU", allow_module_level=True)

from paper_2608_16336_amd.instance import Instance, main  # noqa: E402


def logits_of(inst, tokens):
    """The layer over a whole sequence: logits after every token."""
    x = inst.embed[torch.tensor(tokens, device="cuda")].double()
    n, D = len(tokens), inst.D
    q, k, v = (x @ inst.wqkv.double().t()).split([inst.Hq * D, inst.Hkv * D, inst.Hkv * D], dim=1)
    a = torch.arange(n, device="cuda").double()[:, None, None] * inst.freqs
    c, s = torch.cos(a), torch.sin(a)

    def turn(y):
        y = y.view(n, -1, D)
        p, r = y[..., :D // 2], y[..., D // 2:]
        return torch.cat((p * c - r * s, p * s + r * c), -1)
    q, k, v = turn(q), turn(k), v.view(n, -1, D)
    G = inst.Hq // inst.Hkv
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    w = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0).contiguous()) / math.sqrt(D)
    w = w.masked_fill(~torch.ones(n, n, dtype=torch.bool, device="cuda").tril(), -math.inf).softmax(-1)
    o = torch.matmul(w, v.transpose(0, 1).contiguous()).transpose(0, 1).reshape(n, -1)
    return (x + o @ inst.wo.double().t()) @ inst.embed.double().t()


def prompts(lens, vocab, seed=3):
    g = torch.Generator().manual_seed(seed)
    return [torch.randint(0, vocab, (n,), generator=g).tolist() for n in lens]


@pytest.mark.parametrize("branches,depth", [(0, 1), (1, 4), (3, 2)])
def test_greedy_decode_is_the_layers_argmax(branches, depth):
    inst = Instance(64, vocab=256, branches=branches, depth=depth, seed=5, dtype=torch.float16)
    start = prompts([1, 17, 40, 100], 256)
    assert inst.admit(start)
    for _ in range(6):
        inst.tick()
    for p, r in zip(start, inst.requests):
        assert r["tokens"][:len(p)] == p and len(r["tokens"]) >= len(p) + 6
        assert r["len"] == r["next_pos"] == len(r["tokens"]) - 1
        assert len(r["blocks"]) == -(-r["len"] // inst.bt)
        z = logits_of(inst, r["tokens"][:-1])
        got = torch.tensor(r["tokens"][len(p):], device="cuda")
        z = z[len(p) - 1:]
        # a token is the largest logit but for the 16-bit rounding of activations and logits: of sums over 512 products
        short = z.max(1)[0] - z.gather(1, got[:, None])[:, 0]
        assert (short <= 2.0 ** -8 * z.abs().amax(1) + 0.05).all()
    assert len(inst.free) + inst.blocks_in_use() == 64


def test_weights_are_those_of_all_ticks():
    """Every row of attention hands out one unit of weight a head; the slots hold what their own passes gave them."""
    inst = Instance(32, vocab=128, seed=6)
    inst.admit(prompts([30, 7], 128))
    for _ in range(4):
        inst.tick()
    for r, n in zip(inst.requests, (30, 7)):
        j = torch.arange(r["len"], device="cuda")
        blk = torch.tensor(r["blocks"], device="cuda")[j // inst.bt]
        for h in range(inst.Hkv):
            total = float(inst.score[blk, h, j % inst.bt].double().sum())
            rows = (n - 1 + 4) * inst.Hq // inst.Hkv
            assert abs(total - rows) <= 1e-4 * rows


def test_eviction_makes_room():
    inst = Instance(30, vocab=128, seed=7, budget=48, recent=8, sink=2, temperature=0.9, top_k=20, top_p=0.9, min_p=0.01)
    assert inst.admit(prompts([100, 90, 120, 100], 128))
    assert not inst.admit(prompts([200], 128)) and len(inst.requests) == 4
    for _ in range(130):
        out = inst.tick()
        assert all(len(t) == 1 and 0 <= t[0] < 128 for t in out)
        assert inst.blocks_in_use() + len(inst.free) == 30
    assert inst.evictions >= 2
    for r in inst.requests:
        assert r["len"] <= r["next_pos"] and len(r["tokens"]) >= 150
        j = torch.arange(r["len"], device="cuda")
        blk = torch.tensor(r["blocks"], device="cuda")[j // inst.bt]
        for h in range(inst.Hkv):
            pos = inst.pos[blk, h, j % inst.bt].tolist()
            # positions stay distinct, the first and the last ones are there
            assert len(set(pos)) == len(pos) and {0, 1} <= set(pos)
            assert set(range(r["next_pos"] - 8, r["next_pos"])) <= set(pos)


def test_command(capsys):
    main(["--ticks", "4", "--branches", "2", "--depth", "2"])
    out = capsys.readouterr().out
    assert "running requests" in out and "4 ticks" in out
