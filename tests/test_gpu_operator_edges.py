"""The attention operators where their results are known: queries that see one key."""
import numpy as np
import pytest

from test_gpu_operators import Attn, check, dev, half_step, host

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def binding():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2606_07881_amd import binding as b
    return b


def run(binding, c):
    """Forward and backward of an Attn case: o, lse2, dq, dk, dv and the table's gradient (from zeros), as float64."""
    import torch
    (q, k, v), kw = c.device()
    o, lse2 = torch.empty(c.T, c.d, device="cuda", dtype=q.dtype), torch.empty(c.B * c.H, c.S, device="cuda")
    binding.attention(q, k, v, o, lse2, **kw)
    grads = [torch.empty_like(o) for _ in range(3)]
    g_table = torch.zeros(c.nb, c.H, device="cuda")
    binding.attention_backward(q, k, v, o, lse2, dev(c.do, c.dtype), *grads, g_table=g_table, **kw)
    return [host(t) for t in (o, lse2, *grads, g_table)]


# (batch, seq, heads, head_dim): few and many (sequence, head) pairs
ONE_KEY = [(1, 1, 1, 32), (3, 1, 25, 64), (600, 1, 3, 32), (700, 1, 2, 64), (2, 150, 3, 64), (3, 70, 2, 32), (9, 200, 16, 64),
           (8, 130, 24, 32)]


@pytest.mark.parametrize("shape,dtype", [(s, t) for t in ("bf16", "fp32") for s in ONE_KEY] +
                         [(s, "bf16") for s in ((1, 1, 2, 128), (5, 90, 3, 128), (9, 200, 16, 128))], ids=str)
def test_a_query_that_sees_one_key_has_no_score_gradient(binding, shape, dtype):
    """P is one and o is that key's value, so dS = P (dO v - dO o) is zero: the two sums have the same terms, and taken
    in the same order they are the same float. Sequences of one token, and tables that leave one distance."""
    B, S, H, dh = shape
    far = 0 if S == 1 else 3
    c = Attn((B, S, H, dh, 8, 7, ""), dtype, 11)
    c.bounds = np.arange(8, dtype=np.int32)   # a bucket per distance
    if S > 1:
        c.table[:] = -np.inf
        c.table[far] = np.float32(np.random.default_rng(12).standard_normal(H))
    o, lse2, dq, dk, dv, g_table = run(binding, c)
    val, do = c.split(c.v), c.split(c.do)
    assert np.array_equal(c.split(o)[:, :, far:], val[:, :, :S - far])
    assert np.isneginf(lse2.reshape(B, H, S)[:, :, :far]).all()
    for name, g in (("dq", dq), ("dk", dk), ("g_table", g_table)):
        assert not g.any(), f"{name}: {np.count_nonzero(g)} of {g.size} not zero, up to {np.abs(g).max()}"
    # dv is do, P = 2^(score - lse2) a rounding of the score (below 64, times log2 e) off one, and the output's rounding
    want = np.zeros_like(do)
    want[:, :, :S - far] = do[:, :, far:]
    check(c.split(dv), want, (half_step(dtype) + 128 * U32) * np.abs(want), "dv")
