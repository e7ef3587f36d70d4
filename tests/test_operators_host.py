"""The attention operators' host side: bounds, frequencies, workspace sizes, and every
refusal, which comes before any device work (the pointers here are made up)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import positions

binding = pytest.importorskip("paper_2606_07881_amd.binding",
                              reason="libpaci_stage.so not built (python -m paper_2606_07881_amd.build)")
lib, INVAL, UNSUP, NOMEM = binding.lib, binding.E_INVAL, binding.E_UNSUPPORTED, binding.E_NOMEM
A = 1 << 20   # addresses of made-up buffers, 16-byte aligned


@pytest.mark.parametrize("n_buckets", [2, 3, 7, 8, 32, 33, 64, 255, 256])
def test_rel_bounds_match_whole_number_arithmetic(n_buckets):
    for md in sorted({n_buckets // 2 + 1, 129, 130, 137, 192, 256, 320, 384, 511, 512}):
        if md > n_buckets // 2:
            assert binding.rel_bounds(n_buckets, md).tolist() == positions.bounds(n_buckets, md), md


def test_rel_bounds_and_freqs_refuse():
    b = (ctypes.c_int32 * 300)()
    for n, md, code in [(1, 10, INVAL), (0, 10, INVAL), (32, 16, INVAL), (32, 0, INVAL), (257, 400, UNSUP), (32, 513, UNSUP)]:
        assert lib.paci_rel_bounds(n, md, b) == code, (n, md)
    assert lib.paci_rel_bounds(32, 128, None) == INVAL
    f = (ctypes.c_double * 64)()
    for theta, R in [(0.0, 8), (-1.0, 8), (float("inf"), 8), (float("nan"), 8), (1e4, 7), (1e4, 0), (1e4, -2)]:
        assert lib.paci_rope_freqs(theta, R, f) == INVAL
    assert lib.paci_rope_freqs(1e4, 8, None) == INVAL
    np.testing.assert_allclose(binding.rope_freqs(500000.0, 64), positions.freqs(500000.0, 64), rtol=1e-15)


QK = dict(dtype=1, tokens=4, seq=4, q_heads=2, k_heads=2, head_dim=64, norm=1, eps=1e-5, rope_dims=64, rope_pairs=0)
QK_BAD = [
    (dict(tokens=-1), INVAL), (dict(seq=0), INVAL), (dict(q_heads=-1), INVAL), (dict(q_heads=0, k_heads=0), INVAL),
    (dict(head_dim=0), INVAL), (dict(head_dim=-16), INVAL), (dict(norm=2), INVAL), (dict(norm=0, rope_dims=0), INVAL),
    (dict(eps=-1.0), INVAL), (dict(eps=float("nan")), INVAL), (dict(eps=float("inf")), INVAL), (dict(rope_dims=-16), INVAL),
    (dict(rope_dims=80), INVAL), (dict(rope_pairs=2), INVAL), (dict(rope_pairs=-1), INVAL), (dict(dtype=2), UNSUP),
    (dict(head_dim=24, rope_dims=16), UNSUP), (dict(head_dim=272), UNSUP), (dict(rope_dims=24), UNSUP),
    (dict(q_heads=16384, k_heads=1), UNSUP), (dict(q_heads=2 ** 31 - 1, k_heads=2 ** 31 - 1), UNSUP),
    (dict(tokens=2 ** 30 + 1), UNSUP),
]


def qk_fwd(s, **over):
    p = dict(x=A, ldx=256, gq=A, gk=A, pos=None, freq=A, y=2 * A, ldy=256)
    p.update(over)
    return lib.paci_qk_norm_rope_forward(ctypes.byref(s), p["x"], p["ldx"], p["gq"], p["gk"], p["pos"], p["freq"], p["y"],
                                         p["ldy"], None)


def qk_bwd(s, **over):
    p = dict(x=A, ldx=256, dy=3 * A, lddy=256, gq=A, gk=A, pos=None, freq=A, dx=2 * A, lddx=256, wq=A, wk=A + 256,
             wb=A + 512, ws=A, n=1 << 40)
    p.update(over)
    return lib.paci_qk_norm_rope_backward(ctypes.byref(s), p["x"], p["ldx"], p["dy"], p["lddy"], p["gq"], p["gk"], p["pos"],
                                          p["freq"], p["dx"], p["lddx"], p["wq"], p["wk"], p["wb"], p["ws"], p["n"], None)


@pytest.mark.parametrize("over,code", QK_BAD, ids=str)
def test_qk_shapes_are_refused(over, code):
    s = binding.PaciQkShapes(**dict(QK, **over))
    n = ctypes.c_size_t(0)
    assert qk_fwd(s) == code and qk_bwd(s) == code
    assert lib.paci_qk_norm_rope_workspace(ctypes.byref(s), ctypes.byref(n)) == code


def test_qk_buffers_are_refused():
    s = binding.PaciQkShapes(**QK)
    for over in [dict(x=None), dict(x=A + 8), dict(ldx=255), dict(ldx=252), dict(ldx=248), dict(ldx=-256), dict(gq=None),
                 dict(gk=None), dict(gq=A + 2), dict(pos=A + 2), dict(freq=None), dict(freq=A + 4), dict(ldx=2 ** 45)]:
        assert qk_fwd(s, **over) == INVAL, over
        assert qk_bwd(s, **over) == INVAL, over
    for over in [dict(y=None), dict(y=2 * A + 4), dict(ldy=128), dict(y=A, ldy=264)]:
        assert qk_fwd(s, **over) == INVAL, over
    for over in [dict(dy=None), dict(dy=3 * A + 8), dict(lddy=128), dict(dx=None), dict(dx=2 * A + 8), dict(lddx=128),
                 dict(dx=3 * A, lddx=264), dict(dx=A), dict(wq=A + 2), dict(wb=A + 1), dict(ws=None), dict(ws=A + 4)]:
        assert qk_bwd(s, **over) == INVAL, over
    # parameter gradients that share elements: 64 of a gain each, 256 column sums
    for over in [dict(wk=A), dict(wk=A + 252), dict(wk=A - 252), dict(wb=A), dict(wb=A + 256), dict(wb=A + 508),
                 dict(wb=A - 1020), dict(wq=None, wb=A + 256)]:
        assert qk_bwd(s, **over) == INVAL, over
    n = ctypes.c_size_t(0)
    assert lib.paci_qk_norm_rope_workspace(ctypes.byref(s), ctypes.byref(n)) == 0 and n.value > 0
    assert qk_bwd(s, n=n.value - 1) == NOMEM
    assert lib.paci_qk_norm_rope_workspace(ctypes.byref(s), None) == INVAL
    assert lib.paci_qk_norm_rope_workspace(None, ctypes.byref(n)) == INVAL
    assert qk_bwd(binding.PaciQkShapes(**dict(QK, norm=0))) == INVAL    # gain gradients without a norm
    assert qk_fwd(binding.PaciQkShapes(**dict(QK, tokens=0)), x=None, y=None) == 0


ATTN = dict(dtype=1, batch=2, seq=64, n_heads=2, head_dim=64, n_buckets=8, max_distance=32)
ATTN_BAD = [
    (dict(batch=-1), INVAL), (dict(seq=-1), INVAL), (dict(n_heads=0), INVAL), (dict(head_dim=0), INVAL),
    (dict(n_buckets=-1), INVAL), (dict(n_buckets=1), INVAL), (dict(max_distance=0), INVAL), (dict(dtype=2), UNSUP),
    (dict(head_dim=48), UNSUP), (dict(head_dim=128, dtype=0), UNSUP), (dict(n_buckets=257), UNSUP),
    (dict(max_distance=513), UNSUP), (dict(batch=32768, n_heads=2), UNSUP), (dict(seq=2 ** 20 + 1), UNSUP),
    (dict(batch=2048, seq=2 ** 20, n_heads=1), UNSUP), (dict(batch=256, seq=2 ** 20, n_heads=1), UNSUP), (dict(batch=2 ** 31 - 1, n_heads=2 ** 31 - 1), UNSUP),
]


def attn_fwd(s, **over):
    p = dict(q=A, ldq=128, k=A, ldk=128, v=A, ldv=128, table=A, bounds=A, o=2 * A, lse2=A)
    p.update(over)
    return lib.paci_attn_forward(ctypes.byref(s), p["q"], p["ldq"], p["k"], p["ldk"], p["v"], p["ldv"], p["table"],
                                 p["bounds"], p["o"], p["lse2"], None)


def attn_bwd(s, **over):
    p = dict(q=A, ldq=128, k=A, ldk=128, v=A, ldv=128, table=A, bounds=A, o=3 * A, lse2=A, do=5 * A, dq=2 * A, lddq=128,
             dk=4 * A, lddk=128, dv=6 * A, lddv=128, gt=A, ws=A, n=1 << 40)
    p.update(over)
    return lib.paci_attn_backward(ctypes.byref(s), p["q"], p["ldq"], p["k"], p["ldk"], p["v"], p["ldv"], p["table"],
                                  p["bounds"], p["o"], p["lse2"], p["do"], p["dq"], p["lddq"], p["dk"], p["lddk"], p["dv"],
                                  p["lddv"], p["gt"], p["ws"], p["n"], None)


@pytest.mark.parametrize("over,code", ATTN_BAD, ids=str)
def test_attention_shapes_are_refused(over, code):
    s = binding.PaciAttnShapes(**dict(ATTN, **over))
    n = ctypes.c_size_t(0)
    assert attn_fwd(s) == code and attn_bwd(s) == code
    assert lib.paci_attn_workspace(ctypes.byref(s), ctypes.byref(n)) == code


def test_attention_buffers_are_refused():
    s = binding.PaciAttnShapes(**ATTN)
    both = [dict(zip((n, "ld" + n), bad)) for n in "qkv" for bad in ((None, 128), (A + 8, 128), (A, 120), (A, 132), (A, -128))]
    both += [dict(table=None), dict(bounds=None), dict(table=A + 2), dict(bounds=A + 2), dict(o=None), dict(o=A + 8),
             dict(lse2=None), dict(lse2=A + 2), dict(q=A, ldq=2 ** 41)]
    for over in both:
        assert attn_fwd(s, **over) == INVAL, over
        assert attn_bwd(s, **over) == INVAL, over
    assert attn_fwd(s, o=A) == INVAL   # an operand
    for over in [dict(do=None), dict(do=A + 8), dict(dq=None), dict(dk=None), dict(dv=None), dict(lddq=64), dict(lddk=64),
                 dict(lddv=132), dict(dq=A), dict(dk=A), dict(dv=A), dict(dv=3 * A), dict(dq=5 * A), dict(dq=4 * A), dict(dv=2 * A), dict(dk=6 * A), dict(gt=A + 2), dict(ws=None),
                 dict(ws=A + 8)]:
        assert attn_bwd(s, **over) == INVAL, over
    n = ctypes.c_size_t(0)
    assert lib.paci_attn_workspace(ctypes.byref(s), ctypes.byref(n)) == 0 and n.value > 0
    assert attn_bwd(s, n=n.value - 1) == NOMEM
    assert lib.paci_attn_workspace(ctypes.byref(s), None) == INVAL
    plain = binding.PaciAttnShapes(**dict(ATTN, n_buckets=0))
    assert attn_fwd(plain) == INVAL and attn_bwd(plain) == INVAL          # a table without buckets
    assert attn_bwd(plain, table=None, bounds=None) == INVAL              # a table gradient without a table
    empty = binding.PaciAttnShapes(**dict(ATTN, batch=0))
    assert attn_fwd(empty, q=None, o=None) == 0 and attn_bwd(empty, q=None, ws=None) == 0


def test_binding_refuses_what_it_cannot_pass_on():
    x = torch.zeros(4, 128)
    for call in (lambda: binding.qk_norm_rope(x, x, 1, 1, q_gain=torch.ones(64), k_gain=torch.ones(64)),
                 lambda: binding.attention(x, x, x, x, torch.zeros(2, 4), 1, 2)):
        with pytest.raises(binding.PaciError) as e:
            call()
        assert e.value.code == INVAL   # host tensors


class Shape:
    """A matrix on a device as far as sizes go."""
    is_cuda, dtype = True, torch.bfloat16

    def __init__(self, *shape):
        self.shape = shape

    def dim(self):
        return len(self.shape)


def test_binding_refuses_sizes_beyond_the_c_types():
    """Sizes are 32-bit in the C structures: one that does not fit is refused, not cut to its low bits."""
    big = 2 ** 32
    for call in (lambda: binding.qk_norm_rope_workspace(Shape(big + 4, 128), 1, 1),
                 lambda: binding.qk_norm_rope_workspace(Shape(4, 128), 1, 1, seq=big + 4),
                 lambda: binding.qk_norm_rope_workspace(Shape(4, 128), big + 2, -big),
                 lambda: binding.attention_workspace(Shape(big + 4, 128), 1, 2),
                 lambda: binding.attention_workspace(Shape(big + 4, 128), big + 4, 2),
                 lambda: binding.attention_workspace(Shape(4, 128), 1, 2, table=torch.zeros(8, 2), max_distance=big + 32)):
        with pytest.raises(binding.PaciError):
            call()
    assert binding.qk_norm_rope_workspace(Shape(4, 128), 1, 1, seq=4) > 0
    assert binding.attention_workspace(Shape(4, 128), 1, 2, table=torch.zeros(8, 2), max_distance=32) > 0


# ---- the same as options of a stage -------------------------------------------------------
def test_stage_options_are_checked_and_listed():
    from oracle import stage as ostage
    from paper_2606_07881_amd import configs, inputs
    c = configs.get("gpt2m_mid_bf16", qk_norm=1, rope_dims=64, rel_buckets=32, rel_max_distance=128)
    out = ctypes.c_size_t(0)

    def arena(**over):
        s = binding.shapes(dict(c, **{k: v for k, v in over.items() if k != "raw"}))
        for k, v in over.get("raw", {}).items():
            setattr(s, k, v)
        return lib.paci_stage_arena_bytes(ctypes.byref(s), 8, 3, ctypes.byref(out))
    assert arena() == 0
    with_options = out.value
    for over, code in [(dict(raw=dict(qk_norm=2)), INVAL), (dict(rope_dims=-16), INVAL), (dict(rope_dims=80), INVAL),
                       (dict(rope_dims=8), UNSUP), (dict(rope_theta=0.0), INVAL), (dict(rope_theta=float("nan")), INVAL),
                       (dict(raw=dict(rope_pairs=2)), INVAL), (dict(rel_buckets=-8), INVAL), (dict(rel_buckets=12), UNSUP),
                       (dict(rel_max_distance=16), INVAL), (dict(rel_max_distance=513), UNSUP),
                       (dict(rel_buckets=264, rel_max_distance=512), UNSUP)]:
        assert arena(**over) == code, over
    table = binding.param_table(c)
    specs = inputs.param_specs(c)
    assert [t["name"] for t in table] == [n for n, _, _ in specs] == [n for n, _ in ostage.param_shapes(c)]
    names = [t["name"] for t in table][:8]
    assert names == ["h0.ln1_g", "h0.ln1_b", "h0.w_qkv", "h0.b_qkv", "h0.q_g", "h0.k_g", "h0.rel", "h0.w_o"]
    off = 0
    for t, (n, shape, _) in zip(table, specs):
        assert t["offset"] == off and t["numel"] == int(np.prod(shape)) and t["decay"] == ostage.decayed(n)
        off += t["numel"]
    # the normalised q and k of every block and micro-batch in flight, and little else
    T, d = 8192, 1024
    assert arena(qk_norm=0, rope_dims=0, rel_buckets=0) == 0
    extra = with_options - out.value
    assert 4 * 6 * T * 2 * d * 2 <= extra <= 4 * 6 * T * 2 * d * 2 + (24 << 20)


def test_binding_refuses_negative_sizes_beyond_the_c_types():
    """The low 32 bits of these are sizes that the C calls take."""
    big = 2 ** 32
    for call in (lambda: binding.qk_norm_rope_workspace(Shape(4, 128), 1, 1, seq=4 - big),
                 lambda: binding.attention_workspace(Shape(4, 128), 1, 2, table=torch.zeros(8, 2), max_distance=32 - big)):
        with pytest.raises(binding.PaciError) as e:
            call()
        assert e.value.code == INVAL


def test_host_calls_refuse_sizes_beyond_the_c_types():
    """The C calls would see 64 dimensions and 32 buckets, and fill arrays made for the sizes given."""
    big = 2 ** 32
    for call in (lambda: binding.rope_freqs(1e4, 64 - big), lambda: binding.rope_freqs(1e4, 64 + big),
                 lambda: binding.rel_bounds(32 - big, 128), lambda: binding.rel_bounds(32 + big, 128),
                 lambda: binding.rel_bounds(32, 128 + big), lambda: binding.rel_bounds(32, 128 - big)):
        with pytest.raises(binding.PaciError) as e:
            call()
        assert e.value.code == INVAL


# ---- the binding's import -----------------------------------------------------------------
def test_the_binding_needs_no_private_name_of_torch(root):
    """A torch without device support lacks the raw stream call: the module's host calls still work."""
    import subprocess
    import sys
    code = """
import sys
sys.path.insert(0, {root!r})
import torch
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    del torch._C._cuda_getCurrentRawStream
from paper_2606_07881_amd import binding
print(len(binding.rel_bounds(32, 128)), binding._raw_stream is binding._stream_handle)
""".format(root=root)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["32", "True"], r.stdout + r.stderr
