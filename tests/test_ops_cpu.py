"""Host-side checks of the operators (no GPU): exported symbols, rotary
frequencies, workspace sizes, refusals that are made before anything is
launched, and the references the GPU tests use."""
import ctypes
import math
import os
import re

import pytest

torch = pytest.importorskip("torch")

import ops_ref as ref  # noqa: E402
from paper_2608_16336_amd import mts, ops  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "mts_ops.h")).read(), flags=re.S)


def test_library_exports_every_declared_operator():
    names = set(re.findall(r"\b(mts_[a-z_]+)\s*\(", header()))
    assert names == set(ops.EXPORTED)
    for n in names:
        assert hasattr(mts.load_library(), n), n


def test_structures_match_the_header(tmp_path):
    """Sizes and offsets as the C compiler sees them."""
    types = ["mts_pool", "mts_batch", "mts_rope_args", "mts_attend_args", "mts_weigh_args", "mts_evict_args", "mts_sample_args"]
    lines = []
    for t in types:
        lines.append('printf("%s %%zu\\n", sizeof(%s));' % (t, t))
        for f, _ in getattr(ops, t)._fields_:
            lines.append('printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (t, f, t, f))
    src = tmp_path / "s.c"
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include <stdint.h>\n#define __HIP_PLATFORM_AMD__ 1\n#include \"mts_ops.h\"\n"
                   "int main(void){%s return 0;}\n" % "\n".join(lines))
    exe = tmp_path / "s"
    import subprocess
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include", "-o", str(exe), str(src)], check=True)
    for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines():
        what, n = line.split()
        t, _, f = what.partition(".")
        s = getattr(ops, t)
        assert int(n) == (getattr(s, f).offset if f else ctypes.sizeof(s)), what


def test_rope_freqs():
    f = ops.rope_freqs(64, base=500.0, device="cpu")
    assert torch.allclose(f, torch.tensor([500.0 ** (-2.0 * i / 64) for i in range(32)], dtype=torch.float64), rtol=1e-15)
    assert torch.allclose(ops.rope_freqs(64, base=500.0, scaling="linear", factor=8.0, device="cpu"), f / 8, rtol=1e-15)
    b = ops.rope_freqs(64, base=500.0, scaling="base", factor=8.0, device="cpu")
    assert b[0] == f[0] and abs(b[-1] / f[-1] - 1 / 8) < 1e-12
    p = ops.rope_freqs(64, base=10000.0, scaling="parts", factor=16.0, trained=2048.0, fast=32.0, slow=1.0, device="cpu")
    g = ops.rope_freqs(64, device="cpu")
    turns = 2048 * g / (2 * math.pi)
    assert torch.equal(p[turns >= 32], g[turns >= 32]) and torch.allclose(p[turns <= 1], g[turns <= 1] / 16, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    keep = (turns[mid] - 1) / 31
    assert mid.any() and torch.allclose(p[mid], g[mid] * (keep + (1 - keep) / 16), rtol=1e-14)


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=7), dict(rot=514), dict(base=0.0), dict(base=math.nan), dict(scaling="linear", factor=0.5),
                                dict(scaling="base", factor=2.0, rot=2), dict(scaling="parts", factor=2.0, fast=1.0, slow=2.0),
                                dict(scaling="parts", factor=2.0, trained=0.0), dict(scaling="linear", factor=math.inf)])
def test_rope_freqs_refuses(kw):
    a = dict(rot=64)
    a.update(kw)
    with pytest.raises(mts.MtsError) as e:
        ops.rope_freqs(device="cpu", **a)
    assert e.value.code == -1


def test_attend_workspace():
    last = 0
    for n in (0, 1, 2, 100, 1000):
        b = ops.attend_workspace(n, n, 1, 32, 8, 128)
        assert b > last or n == 0
        last = b
    for bad in ((1, 1, 0, 4, 2, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 1, 2, 64), (1, 1, 1, 4, 0, 64), (1, 1, 1, 4, 2, 80)):
        with pytest.raises(mts.MtsError):
            ops.attend_workspace(*bad)


FAKE = 1 << 20  # a 256-byte aligned address that no call below may reach


def _pool(**kw):
    p = ops.mts_pool(k=FAKE, v=FAKE, k_block=1024, k_head=1024, k_token=64, v_block=1024, v_head=1024, v_token=64, n_blocks=4,
                     block_tokens=16, kv_heads=1, head_dim=64, type=0, reserved=0)
    for k, v in kw.items():
        setattr(p, k, v)
    return p


def _batch(**kw):
    b = ops.mts_batch(table=FAKE, lens=FAKE, q_start=FAKE, tree=None, n=1, table_width=4, n_tokens=1, max_q=1, tree_words=0, reserved=0)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


POOLS = [dict(k=None), dict(k=FAKE + 8), dict(k_token=60), dict(k_block=-8), dict(n_blocks=0), dict(n_blocks=1 << 31), dict(block_tokens=12),
         dict(block_tokens=128), dict(block_tokens=0), dict(kv_heads=0), dict(head_dim=80), dict(head_dim=0), dict(type=2), dict(type=9),
         dict(reserved=1)]
BATCHES = [dict(table=None), dict(lens=None), dict(q_start=None), dict(table_width=0), dict(table_width=1 << 27), dict(max_q=0),
           dict(tree_words=1), dict(tree=FAKE), dict(tree=FAKE, tree_words=2000), dict(n_tokens=1 << 31), dict(reserved=1)]


def _attend(pool=None, batch=None, **kw):
    a = ops.mts_attend_args(pool=pool or _pool(), batch=batch or _batch(), q=FAKE, out=FAKE, lse=None, q_token=64, q_head=64, out_token=64,
                            out_head=64, q_heads=2, scale=1.0, workspace=FAKE, workspace_bytes=1 << 40)
    for k, v in kw.items():
        setattr(a, k, v)
    return ops._library().mts_attend(ctypes.byref(a), None)


def test_attend_refuses():
    for p in POOLS + [dict(v=None), dict(v_head=4)]:
        assert _attend(pool=_pool(**p)) == -1, p
    for b in BATCHES:
        assert _attend(batch=_batch(**b)) == -1, b
    for kw in (dict(q=None), dict(q=FAKE + 2), dict(out=FAKE + 8), dict(q_token=4), dict(out_head=-8), dict(q_heads=0), dict(q_heads=70000),
               dict(scale=math.nan), dict(workspace=None), dict(workspace=FAKE + 16)):
        assert _attend(**kw) == -1, kw
    assert _attend(pool=_pool(kv_heads=2), q_heads=3) == -1
    assert _attend(workspace_bytes=1000) == -2
    assert ops._library().mts_attend(None, None) == -1
    assert _attend(batch=_batch(n=0)) == 0 and _attend(batch=_batch(n_tokens=0)) == 0


def test_weigh_refuses():
    def call(pool=None, batch=None, **kw):
        a = ops.mts_weigh_args(pool=pool or _pool(v=None), batch=batch or _batch(), q=FAKE, lse=FAKE, q_token=64, q_head=64, score=FAKE,
                               q_heads=2, scale=1.0, decay=0.5)
        for k, v in kw.items():
            setattr(a, k, v)
        return ops._library().mts_weigh(ctypes.byref(a), None)
    for p in POOLS:
        assert call(pool=_pool(**p)) == -1, p
    for b in BATCHES:
        assert call(batch=_batch(**b)) == -1, b
    for kw in (dict(q=None), dict(lse=None), dict(score=None), dict(score=FAKE + 1), dict(decay=-0.1), dict(decay=1.5), dict(decay=math.nan),
               dict(scale=math.nan), dict(q_heads=0), dict(q_head=3)):
        assert call(**kw) == -1, kw
    assert call(batch=_batch(n=0)) == 0


def test_evict_refuses():
    def call(pool=None, batch=None, **kw):
        a = ops.mts_evict_args(pool=pool or _pool(), batch=batch or _batch(q_start=None), score=FAKE, pos=FAKE, next_pos=FAKE, score_out=FAKE,
                               pos_out=FAKE, lens_out=FAKE + 64, budget=8, recent=0, sink=0, reserved=0, workspace=FAKE, workspace_bytes=1 << 40)
        for k, v in kw.items():
            setattr(a, k, v)
        return ops._library().mts_evict(ctypes.byref(a), None)
    for p in [x for x in POOLS if x.get("head_dim") != 80] + [dict(v=None), dict(head_dim=4), dict(head_dim=12)]:
        assert call(pool=_pool(**p)) == -1, p
    for b in (dict(table=None), dict(lens=None), dict(table_width=0)):
        assert call(batch=_batch(**b)) == -1, b
    for kw in (dict(score=None), dict(pos=None), dict(next_pos=None), dict(score_out=None), dict(pos_out=None), dict(lens_out=None),
               dict(lens_out=FAKE), dict(budget=0), dict(budget=1 << 31), dict(recent=1 << 31), dict(sink=1 << 31), dict(reserved=1),
               dict(workspace=None)):
        assert call(**kw) == -1, kw
    assert call(workspace_bytes=100) == -2
    assert call(batch=_batch(n=0)) == 0
    n = ctypes.c_size_t(0)
    assert ops._library().mts_evict_workspace(4, 8, 100, 16, 0, ctypes.byref(n)) == -1
    assert ops._library().mts_evict_workspace(4, 8, 100, 16, 500, None) == -1


def test_rope_refuses():
    def call(pool=None, **kw):
        a = ops.mts_rope_args(q=FAKE, k=FAKE, v=FAKE, q_out=FAKE, k_out=None, q_token=128, q_head=64, k_token=64, k_head=64, v_token=64,
                              v_head=64, qo_token=128, qo_head=64, ko_token=64, ko_head=64, positions=FAKE, freqs=FAKE, slots=FAKE, pos=FAKE,
                              pool=pool or _pool(), n_tokens=1, q_heads=2, rot=64, layout=0, inverse=0, mscale=1.0)
        for k, v in kw.items():
            setattr(a, k, v)
        return ops._library().mts_rope(ctypes.byref(a), None)
    for p in (dict(k=None), dict(v=None), dict(k=FAKE + 8), dict(n_blocks=0), dict(block_tokens=12), dict(kv_heads=0), dict(head_dim=60),
              dict(head_dim=1024), dict(type=2), dict(type=3), dict(reserved=1)):
        assert call(pool=_pool(**p)) == -1, p
    for kw in (dict(q=None), dict(q_out=None), dict(k=None), dict(v=FAKE + 4), dict(rot=0), dict(rot=63), dict(rot=66), dict(layout=2),
               dict(inverse=2), dict(mscale=math.nan), dict(positions=None), dict(freqs=None), dict(q_head=4), dict(n_tokens=1 << 31),
               dict(slots=None), dict(q_heads=70000)):
        assert call(**kw) == -1, kw
    assert call(n_tokens=0) == 0


def test_sample_refuses():
    def call(**kw):
        a = ops.mts_sample_args(logits=FAKE, row_stride=100, u=FAKE, temperature=FAKE, top_k=FAKE, top_p=FAKE, min_p=FAKE, token=FAKE,
                                logprob=None, rows=2, vocab=100, type=0, reserved=0)
        for k, v in kw.items():
            setattr(a, k, v)
        return ops._library().mts_sample(ctypes.byref(a), None)
    for kw in (dict(logits=None), dict(logits=FAKE + 1), dict(row_stride=99), dict(row_stride=-100), dict(u=None), dict(temperature=None),
               dict(top_k=None), dict(top_p=None), dict(min_p=None), dict(token=None), dict(token=FAKE + 2), dict(logprob=FAKE + 1),
               dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(type=3), dict(reserved=1), dict(rows=1 << 31)):
        assert call(**kw) == -1, kw
    assert call(rows=0) == 0


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 8)
    f = torch.zeros(2)
    with pytest.raises(ValueError):
        ops.sample(x, f, f, torch.zeros(2, dtype=torch.int32), f, f)


# ---------------------------------------------------------------- the references themselves


def test_reference_attention_is_torchs_softmax():
    b = ref.make_batch([21, 9], [5, 9], 4, 2, 16, torch.float16, poison=False)
    q = torch.randn(14, 4, 16).half()
    out, lse, _, _ = ref.attend(b, q)
    for r, (a, z, L) in enumerate(((0, 5, 21), (5, 14, 9))):
        for h in range(4):
            k, v = (ref.rows_of(b, r, b[x], h // 2)[0].double() for x in "kv")
            s = q[a:z, h].double() @ k.t() / 4.0
            s = s.masked_fill(~torch.ones(z - a, L).tril(L - (z - a)).bool(), -math.inf)
            assert torch.allclose(out[a:z, h], torch.softmax(s, -1) @ v, rtol=1e-12, atol=1e-13)
            assert torch.allclose(lse[a:z, h], torch.logsumexp(s, -1), rtol=1e-12, atol=1e-13)


def test_reference_kept_weights():
    x = torch.tensor([0.0, 3.0, 1.0, 3.0, 2.0])
    w = ref.kept_weights(x, 1.0, 0, 1.0, 0.0)
    assert torch.allclose(w / w.sum(), torch.softmax(x.double(), 0))
    assert torch.nonzero(ref.kept_weights(x, 1.0, 3, 1.0, 0.0))[:, 0].tolist() == [1, 3, 4]
    assert torch.nonzero(ref.kept_weights(x, 1.0, 1, 1.0, 0.0))[:, 0].tolist() == [1]
    assert torch.nonzero(ref.kept_weights(x, 1.0, 0, 0.0, 0.0))[:, 0].tolist() == [1]
    assert torch.nonzero(ref.kept_weights(x, 1.0, 0, 1.0, 0.3))[:, 0].tolist() == [1, 3, 4]
    assert ref.kept_weights(torch.tensor([math.nan, -math.inf]), 1.0, 0, 1.0, 0.0) is None
