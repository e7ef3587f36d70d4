"""The attention operators where their results are known: queries that see one key, and table entries at and
beyond the largest that count."""
import numpy as np
import pytest

from oracle import model, positions
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


def run(binding, c, do=None):
    """Forward and backward (of c.do) of an Attn case: o, lse2, dq, dk, dv and the table's gradient (from zeros), as
    float64."""
    import torch
    (q, k, v), kw = c.device()
    o, lse2 = torch.empty(c.T, c.d, device="cuda", dtype=q.dtype), torch.empty(c.B * c.H, c.S, device="cuda")
    binding.attention(q, k, v, o, lse2, **kw)
    grads = [torch.empty_like(o) for _ in range(3)]
    g_table = torch.zeros(c.nb, c.H, device="cuda")
    binding.attention_backward(q, k, v, o, lse2, dev(c.do if do is None else do, c.dtype), *grads, g_table=g_table, **kw)
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


@pytest.mark.parametrize("entry", [-3e4, 3e4])
@pytest.mark.parametrize("shape,dtype", [((700, 1, 2, 64), "bf16"), ((600, 1, 3, 32), "fp32"), ((2, 150, 3, 64), "fp32"),
                                         ((9, 200, 16, 64), "bf16"), ((5, 90, 3, 128), "bf16")], ids=str)
def test_nor_at_the_largest_entries(binding, shape, dtype, entry):
    """There the forward's probability can be off one by 2^-9, and the sum it is divided by with it."""
    B, S, H, dh = shape
    far = 0 if S == 1 else 3
    c = Attn((B, S, H, dh, 8, 7, ""), dtype, 18)
    c.bounds = np.arange(8, dtype=np.int32)
    c.table[:] = -np.inf
    c.table[far] = np.float32(entry + np.random.default_rng(19).standard_normal(H))
    o, _, dq, dk, _, g_table = run(binding, c)
    assert np.array_equal(c.split(o)[:, :, far:], c.split(c.v)[:, :, :S - far])
    for name, g in (("dq", dq), ("dk", dk), ("g_table", g_table)):
        assert not g.any(), name


# ---- large entries ----------------------------------------------------------------------------
def _with_table(shape, dtype, table):
    """An Attn case with a bucket per distance (7 and more share the last) and this table."""
    c = Attn((*shape, 8, 7, ""), dtype, 13)
    c.bounds = np.arange(8, dtype=np.int32)
    c.table = np.float32(table)
    c.bias = positions.bias_by_distance(c.table, c.bounds, c.md, c.S)
    c.o, lse = model.attention_fwd(c.qkv, c.B, c.S, c.H, c.dh, bias=c.bias)
    c.lse2 = lse / np.log(2.0)
    return c


def _check_probabilities(binding, c):
    """Forward and backward against the oracle's own probabilities (not those that the saved statistic gives).

    A score takes dh + 4 roundings of sum |q k| / sqrt(dh), and the bias as many in bf16, where the products start from
    it, and 2 in fp32; both directions form it alike. An error e of the scores moves a probability P_j by the relative
    (1 - P_j) e_j + sum of P_i e_i over the other keys. Its distance from the statistic, one float, takes 4 roundings of
    the larger of both: their product with a scale in each direction, the statistic's and the difference's."""
    u, r = half_step(c.dtype), half_step(c.dtype) if c.dtype == "bf16" else 0.0
    Q, K, V, dO = (c.split(a) for a in (c.q, c.k, c.v, c.do))
    sc, i = 1 / np.sqrt(c.dh), np.arange(c.S)
    dist = i[:, None] - i
    bias = c.bias[:, np.maximum(dist, 0)]
    s = np.where(dist < 0, -np.inf, Q @ K.transpose(0, 1, 3, 2) * sc + bias)
    l = c.lse2.reshape(c.B, c.H, c.S, 1) * np.log(2.0)
    P = np.exp(s - np.where(l == -np.inf, np.inf, l))
    size = np.abs(np.where(np.isfinite(bias), bias, 0.0))
    e = (c.dh + 4) * U32 * (np.abs(Q) @ np.abs(K).transpose(0, 1, 3, 2)) * sc + (c.dh + 4 if c.dtype == "bf16" else 2) * U32 * size
    e = np.where(P > 0, e, 0.0)
    both = (P * e).sum(-1, keepdims=True)
    stat = 4 * U32 * np.maximum(np.abs(np.where(np.isfinite(l), l, 0.0)), np.where(P > 0, np.abs(np.where(P > 0, s, 0.0)), 0.0))
    rel = (1 - P) * e + (both - P * e) + stat + (c.S + 16) * U32
    o, lse2, dq, dk, dv, g_table = run(binding, c)
    fwd = rel.max(-1, keepdims=True)
    check(c.split(o), c.split(c.o), (r + fwd) * (P @ np.abs(V)) + 1.01 * u * np.abs(c.split(c.o)), "o")
    want = c.lse2.reshape(c.B * c.H, c.S)
    top = np.where(np.isfinite(want), np.abs(want), 0.0)
    check(lse2, want, (e.max(-1).reshape(want.shape) + (c.S + 16) * U32) / np.log(2.0) + 4 * U32 * top, "lse2")
    O = c.split(o)
    dS = P * (dO @ V.transpose(0, 1, 3, 2) - (dO * O).sum(-1, keepdims=True))
    mass = np.abs(dO) @ np.abs(V).transpose(0, 1, 3, 2) + (np.abs(dO) * np.abs(O)).sum(-1, keepdims=True)
    absd, acc = np.abs(dS), (c.S + 8) * U32
    e_s = P * mass * (c.dh + 8) * U32 + absd * (rel + 8 * U32)
    flip = lambda a: a.transpose(0, 1, 3, 2)  # noqa: E731
    both_ways = (r + acc) * absd + e_s
    for name, got, ref, tol in (("dq", dq, dS @ K * sc, both_ways @ np.abs(K) * sc),
                                ("dk", dk, flip(dS) @ Q * sc, flip(both_ways) @ np.abs(Q) * sc),
                                ("dv", dv, flip(P) @ dO, flip((r + acc + rel + 8 * U32) * P) @ np.abs(dO))):
        check(c.split(got), ref, tol + 1.01 * u * np.abs(ref) + 1e-37, name)
    g = positions.table_grad(dS.sum(0), c.bounds, c.md)
    check(g_table, g, positions.table_grad((e_s + 64 * U32 * absd).sum(0), c.bounds, c.md) + U32 * np.abs(g), "g_table")
    # of output gradients of one, dv adds up to the probabilities' sums: one for every query with a key
    ones = run(binding, c, np.ones_like(c.do))[4]
    rows = np.isfinite(l[..., 0])
    total = c.split(ones).sum(2)
    room = ((stat * P).sum(-1) + ((c.S + 16) * U32 + r) * rows).sum(-1, keepdims=True)
    check(total, np.broadcast_to(rows.sum(-1)[..., None], total.shape).astype(np.float64),
          room + u * c.split(ones).sum(2), "sum of the probabilities")


LIMIT_SHAPES = [((2, 140, 2, 64), "bf16"), ((2, 140, 2, 64), "fp32"), ((1, 90, 3, 32), "bf16"), ((1, 90, 3, 32), "fp32"),
                ((2, 75, 2, 128), "bf16"), ((9, 200, 16, 64), "bf16")]


@pytest.mark.parametrize("entry", [1e4, 3e4, 32768.0, 1e5, 1e6, 1e8, 3e38], ids="{:g}".format)
@pytest.mark.parametrize("shape,dtype", LIMIT_SHAPES, ids=str)
def test_an_entry_above_every_score_leaves_one_key(binding, shape, dtype, entry):
    """Entries above 2^15 count as it. From query 3 on, one key has P = 1."""
    table = np.random.default_rng(14).standard_normal((8, shape[2]))
    table[3] = entry
    _check_probabilities(binding, _with_table(shape, dtype, table))


@pytest.mark.parametrize("entry", [1e4, 3e4, 32700.0], ids="{:g}".format)
@pytest.mark.parametrize("shape,dtype", LIMIT_SHAPES, ids=str)
def test_low_entries_that_a_row_shares_cancel(binding, shape, dtype, entry):
    """Every visible key at a low entry that still counts: the softmax of what the scores differ in."""
    table = np.random.default_rng(15).standard_normal((8, shape[2])) - entry
    _check_probabilities(binding, _with_table(shape, dtype, table))


@pytest.mark.parametrize("entry", [32768.0, 65504.0, 1e8, 9e8, 3e38], ids="{:g}".format)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_entries_at_or_below_the_lowest_hide(binding, dtype, entry):
    """A head at the entry sees nothing; in the other one, distances 0 and 2 are hidden."""
    table = np.random.default_rng(16).standard_normal((8, 2))
    table[:, 0] = -entry
    table[[0, 2], 1] = -entry
    c = _with_table((2, 100, 2, 64), dtype, table)
    assert np.isneginf(c.lse2.reshape(2, 2, 100)[:, 0]).all()
    _check_probabilities(binding, c)


# ---- layouts ----------------------------------------------------------------------------------
@pytest.mark.parametrize("buckets", [0, 8])
@pytest.mark.parametrize("shape,dtype", [((2, 140, 2, 64), "bf16"), ((2, 140, 2, 64), "fp32"), ((1, 90, 3, 32), "bf16"),
                                         ((1, 90, 3, 32), "fp32"), ((2, 75, 2, 128), "bf16"), ((9, 200, 16, 64), "bf16")], ids=str)
def test_the_operands_layout_does_not_matter(binding, shape, dtype, buckets):
    """The thirds of a fused projection (and of its gradient) against buffers of their own with wider rows, other orders and
    NaN around them: the same bits, with a bias and without."""
    import torch
    c = Attn((*shape, buckets, 7, ""), dtype, 17)
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    kw = dict(batch=c.B, n_heads=c.H)
    if buckets:
        kw.update(table=dev(c.table), bounds=torch.from_numpy(c.bounds).cuda(), max_distance=c.md)

    def chain(operands, grads):
        o, lse2 = torch.empty(c.T, c.d, device="cuda", dtype=act), torch.empty(c.B * c.H, c.S, device="cuda")
        g_table = torch.zeros(buckets, c.H, device="cuda") if buckets else None
        binding.attention(*operands, o, lse2, **kw)
        binding.attention_backward(*operands, o, lse2, dev(c.do, dtype), *grads, g_table=g_table, **kw)
        return [o, lse2, *grads] + ([g_table] if buckets else [])

    def apart(pads):
        return [torch.full((c.T, c.d + p), float("nan"), device="cuda", dtype=act)[:, 8:8 + c.d] for p in pads]
    qkv = dev(c.qkv, dtype)
    fused = chain(qkv.split(c.d, 1), torch.empty_like(qkv).split(c.d, 1))
    operands = apart((8, 40, 24))
    for t, a in zip(operands, (c.q, c.k, c.v)):
        t.copy_(dev(a, dtype))
    other = chain(operands, apart((56, 8, 16)))
    vk = torch.empty(c.T, 2 * c.d, device="cuda", dtype=act)   # v before k, q alone
    vk[:, :c.d], vk[:, c.d:] = dev(c.v, dtype), dev(c.k, dtype)
    dkv = torch.empty_like(vk)
    third = chain([dev(c.q, dtype), vk[:, c.d:], vk[:, :c.d]], [torch.empty(c.T, c.d, device="cuda", dtype=act), dkv[:, c.d:], dkv[:, :c.d]])
    for i, (x, y, z) in enumerate(zip(fused, other, third)):
        assert torch.isfinite(x).all() and torch.equal(x, y) and torch.equal(x, z), i


# ---- streams ----------------------------------------------------------------------------------
def test_both_ways_to_the_current_stream_agree(binding):
    import torch
    dev_index = torch.cuda.current_device()
    for st in (torch.cuda.current_stream(), torch.cuda.Stream()):
        with torch.cuda.stream(st):
            assert binding._raw_stream(dev_index) == binding._stream_handle(dev_index) == st.cuda_stream
