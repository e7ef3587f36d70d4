"""The attention operators on the GPU against the oracle in 64 bits, through the binding.

Inputs are rounded to the operator's type before both sides read them. u is the
half step of a type (bf16 2^-8, fp32 2^-24). Every tolerance is elementwise and
counts, from the oracle's own arrays:
* the rounding of an output: u |y|;
* bf16 attention: the probabilities and dS are rounded once before their
  products (u times the product of absolute values);
* fp32 arithmetic: a bound c * 2^-24 of the sum of absolute values of the terms,
  with c at least the number of roundings a term passes through (derived at each
  test).
"""
import numpy as np
import pytest

from oracle import model, positions
from paper_2606_07881_amd import inputs

pytestmark = pytest.mark.gpu
U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def binding():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2606_07881_amd import binding as b
    return b


def half_step(dtype):
    return 2.0 ** -8 if dtype == "bf16" else U32


def rounded(a, dtype):
    """The values of a in the operator's type, as float64."""
    a = np.asarray(a, np.float32)
    return (inputs.bf16_round(a) if dtype == "bf16" else a).astype(np.float64)


def dev(a, dtype=None):
    """float64 values on the GPU in the operator's type (None: float32)."""
    import torch
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def check(got, want, tol, what):
    assert got.shape == want.shape
    same = np.where(np.isfinite(want), np.abs(got - np.where(np.isfinite(want), want, 0.0)) <= tol, got == want)
    if not same.all():
        i = np.unravel_index(np.argmin(same), same.shape)
        raise AssertionError(f"{what}: {np.count_nonzero(~same)} of {same.size} outside, first at {i}: "
                             f"{got[i]} for {want[i]}, tolerance {np.broadcast_to(tol, want.shape)[i]}")


# ---- norms and rotation -----------------------------------------------------------------------
# (tokens, q heads, k heads, head_dim, rope_dims, pairs, norm, positions)
ROTARY = [
    (1, 1, 0, 16, 16, "half", True, "given"), (1, 12, 12, 64, 64, "half", True, "far"),
    (3, 2, 2, 32, 32, "adjacent", True, "seq"), (5, 0, 3, 48, 16, "half", True, "given"),
    (37, 4, 2, 64, 32, "half", False, "seq"), (64, 4, 4, 32, 32, "half", True, "seq"),
    (129, 5, 1, 96, 96, "adjacent", True, "far"), (257, 3, 3, 128, 128, "half", True, "given"),
    (200, 7, 7, 128, 48, "half", True, "seq"), (65, 17, 2, 256, 256, "half", True, "seq"),
    (66, 9, 9, 256, 64, "adjacent", True, "given"), (300, 2, 1, 80, 0, "half", True, "seq"),
    (700, 1, 1, 16, 16, "adjacent", True, "seq"), (90, 40, 8, 112, 112, "half", True, "given"),
    (2100, 16, 16, 64, 64, "half", True, "seq"), (2100, 16, 4, 128, 128, "half", True, "seq"), (1025, 12, 12, 64, 64, "half", False, "far"),
    (70, 80, 17, 128, 128, "half", True, "seq"), (33, 75, 75, 256, 128, "adjacent", True, "given"),
]


class Rotary:
    """Inputs of one case: x and dy are column ranges of wider rows (row stride wider than the heads)."""

    def __init__(self, case, dtype, seed):
        T, qh, kh, dh, R, self.pairs, norm, where = case
        self.T, self.qh, self.kh, self.dh, self.dtype = T, qh, kh, dh, dtype
        g = np.random.default_rng(seed)
        self.n, self.eps, self.seq = (qh + kh) * dh, 1e-5, max(1, T // 2 + 3)
        self.x = rounded(g.standard_normal((T, self.n)) * np.exp(g.standard_normal((T, 1))), dtype)
        self.dy = rounded(g.standard_normal((T, self.n)) * 1e-2, dtype)
        self.gq, self.gk = (np.float32(1 + 0.3 * g.standard_normal(dh)) if norm else None for _ in range(2))
        self.freq = positions.freqs(10000.0, R)
        self.pos = None
        if where == "given":
            self.pos = g.integers(-50, 5000, T).astype(np.int32)
        elif where == "far":
            self.pos = g.integers(2 ** 30, 2 ** 31 - 1, T).astype(np.int32)
        self.at = np.arange(T) % self.seq if self.pos is None else self.pos
        self.gain = None
        if norm:
            self.gain = np.concatenate([np.tile(self.gq, (qh, 1)), np.tile(self.gk, (kh, 1))]).astype(np.float64)
            if not qh:
                self.gq = None
            if not kh:
                self.gk = None

    def heads(self, a):
        return a.reshape(self.T, self.qh + self.kh, self.dh)

    def wide(self, a, pad=24):
        """a as the left columns of wider device rows whose other columns are NaN."""
        import torch
        t = torch.full((self.T, self.n + pad), float("nan"), device="cuda",
                       dtype=torch.bfloat16 if self.dtype == "bf16" else torch.float32)
        t[:, :self.n] = dev(a, self.dtype)
        return t

    def args(self):
        import torch
        return dict(q_heads=self.qh, k_heads=self.kh, seq=self.seq, eps=self.eps, pairs=self.pairs,
                    q_gain=None if self.gq is None else dev(self.gq), k_gain=None if self.gk is None else dev(self.gk),
                    freq=torch.from_numpy(self.freq).cuda() if len(self.freq) else None,
                    pos=None if self.pos is None else torch.from_numpy(self.pos).cuda())

    def fwd(self):
        """(y, tolerance): per element at most dh / 16 + 8 additions of squares (halved by the root), the
        root, two products, the angle (4 units of its sine and cosine) and the turn's product and sum: below
        64 roundings of a head's largest member."""
        y = positions.norm_rope_fwd(self.heads(self.x), self.gain, self.at, self.freq, self.pairs, self.eps)
        n = positions.norm_rope_fwd(self.heads(self.x), self.gain, self.at, np.zeros(0), self.pairs, self.eps)
        big = np.abs(n).max(-1, keepdims=True) * 2
        return y.reshape(self.T, -1), (half_step(self.dtype) * np.abs(y) + 64 * U32 * big).reshape(self.T, -1)

    def bwd(self):
        """(dx, tolerance, dgain, tolerance, column sums, tolerance): as the forward, with the mean of e xh and
        its product; the sums over T tokens add 16 + T / (a workgroup's share) roundings, bounded by T + 64."""
        x, dy = self.heads(self.x), self.heads(self.dy)
        dx, dgain = positions.norm_rope_bwd(dy, x, self.gain, self.at, self.freq, self.pairs, self.eps)
        big = np.abs(dy).max(-1, keepdims=True) * 2
        if self.gain is not None:
            r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + self.eps)
            dn = positions.rotate(dy, self.at, self.freq, self.pairs, -1) if len(self.freq) else dy
            e = np.abs(big * self.gain)
            xh = np.abs(x * r)
            t_g = (64 + self.T) * U32 * (big * xh).sum(0)
            big = r * (e + xh * (e * xh).mean(-1, keepdims=True))
            del dn
        else:
            t_g = None
        t_dx = half_step(self.dtype) * np.abs(dx) + 96 * U32 * big
        t_b = (96 + self.T) * U32 * np.broadcast_to(big, dx.shape).sum(0)
        flat = lambda a: a.reshape(self.T, -1)  # noqa: E731
        if self.gain is None:
            g = gt = None
        else:
            g = [p.sum(0) for p in np.split(dgain, [self.qh])]
            gt = [p.sum(0) for p in np.split(t_g, [self.qh])]
        return flat(dx), flat(t_dx), g, gt, dx.sum(0).reshape(-1), t_b.reshape(-1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", ROTARY, ids=lambda c: "-".join(map(str, c)))
def test_rotary(binding, case, dtype):
    import torch
    c = Rotary(case, dtype, 1)
    print(f"rotary {case} {dtype}", flush=True)
    kw = c.args()
    x = c.wide(c.x)
    want, tol = c.fwd()
    y = c.wide(np.zeros_like(c.x), pad=8)
    binding.qk_norm_rope(x[:, :c.n], y[:, :c.n], **kw)
    check(host(y[:, :c.n]), want, tol, "y")
    assert torch.isnan(y[:, c.n:]).all(), "columns behind the heads were written"
    inplace = x.clone()
    binding.qk_norm_rope(inplace[:, :c.n], inplace[:, :c.n], **kw)
    assert torch.equal(inplace[:, :c.n], y[:, :c.n]) and torch.isnan(inplace[:, c.n:]).all()

    dx, t_dx, g, gt, gb, tb = c.bwd()
    start = np.float32(np.random.default_rng(2).standard_normal(c.n))   # gradients are added to
    got_b, got_q, got_k = dev(start), dev(start[:c.dh]), dev(start[:c.dh])
    dy, out = c.wide(c.dy), c.wide(np.zeros_like(c.x), pad=16)
    gains = dict(g_q_gain=got_q, g_k_gain=got_k) if c.gain is not None else {}
    binding.qk_norm_rope_backward(x[:, :c.n], dy[:, :c.n], out[:, :c.n], g_bias=got_b, **gains, **kw)
    check(host(out[:, :c.n]), dx, t_dx, "dx")
    assert torch.isnan(out[:, c.n:]).all()
    check(host(got_b), gb + start, tb + U32 * np.abs(gb + start), "g_bias")
    if c.gain is not None:
        for name, got, want, tol in zip("qk", (got_q, got_k), g, gt):
            check(host(got), want + start[:c.dh], tol + U32 * np.abs(want + start[:c.dh]), f"g_{name}_gain")
    # in place, without the sums, and again: the same bits
    binding.qk_norm_rope_backward(x[:, :c.n], dy[:, :c.n], dy[:, :c.n], **kw)
    assert torch.equal(dy[:, :c.n], out[:, :c.n])
    again, dy2 = dev(start), c.wide(c.dy)
    binding.qk_norm_rope_backward(x[:, :c.n], dy2[:, :c.n], out[:, :c.n], g_bias=again, **kw)
    assert torch.equal(again, got_b), "two runs differ"


def test_rotary_without_tokens(binding):
    import torch
    x = torch.empty(0, 64, device="cuda")
    g = torch.ones(32, device="cuda")
    binding.qk_norm_rope(x, x, 1, 1, q_gain=g, k_gain=g)
    gb = torch.ones(64, device="cuda")
    binding.qk_norm_rope_backward(x, x, x, 1, 1, q_gain=g, k_gain=g, g_bias=gb)
    assert (gb == 1).all()


# ---- attention --------------------------------------------------------------------------------
# (batch, seq, heads, head_dim, buckets, max_distance, hidden)
ATTN = [
    (1, 1, 1, 32, 8, 16, ""), (2, 2, 3, 64, 32, 128, ""), (1, 17, 2, 64, 8, 5, ""), (3, 63, 1, 32, 16, 40, "far"),
    (2, 64, 2, 64, 32, 128, ""), (1, 65, 3, 64, 2, 2, ""), (2, 100, 2, 32, 16, 33, "first"), (1, 129, 2, 64, 8, 64, "all"),
    (2, 200, 3, 64, 32, 128, "some"), (1, 300, 2, 32, 64, 200, "lowest"), (1, 333, 1, 64, 4, 3, "far"),
    (1, 700, 1, 64, 32, 512, ""), (1, 4500, 1, 64, 32, 128, ""), (1, 520, 2, 32, 8, 100, "big"), (1, 200, 2, 64, 0, 0, ""),
]
# enough (sequence, head) pairs for the larger workgroups
ATTN_MANY = [(8, 260, 16, 64, 32, 128, ""), (3, 250, 47, 32, 16, 30, "some"), (11, 193, 16, 64, 8, 300, "far"),
             (19, 129, 16, 32, 32, 128, "")]
ATTN128 = [(9, 200, 16, 128, 32, 60, ""), (1, 1, 2, 128, 8, 16, ""), (2, 77, 2, 128, 32, 128, "some"), (1, 400, 1, 128, 16, 50, ""),
           (1, 600, 1, 128, 256, 512, "first"), (1, 150, 2, 128, 0, 0, "")]


class Attn:
    """q and k in one buffer, v in another (the stage's layout under a rotation), strided rows."""

    def __init__(self, case, dtype, seed):
        self.B, self.S, self.H, self.dh, nb, md, hidden = case
        self.dtype, self.nb, self.md = dtype, nb, md
        self.d, self.T = self.H * self.dh, self.B * self.S
        g = np.random.default_rng(seed)
        self.q, self.k, self.v = (rounded(g.standard_normal((self.T, self.d)), dtype) for _ in range(3))
        self.do = rounded(g.standard_normal((self.T, self.d)), dtype)
        self.table = self.bounds = self.bias = None
        if nb:
            self.table = np.float32(g.standard_normal((nb, self.H)) * (2000 if hidden == "big" else 1))
            self.bounds = np.array(positions.bounds(nb, md) if md > nb // 2 else range(nb), np.int32)
            t = self.table
            if hidden == "far":
                t[-1] = -np.inf
            elif hidden == "first":    # no query sees itself; the first of a sequence sees nothing
                t[0] = -np.inf
            elif hidden == "all":      # a head that sees nothing
                t[:, 0] = -np.inf
            elif hidden == "some":
                t[g.random(t.shape) < 0.3] = -np.inf
            elif hidden == "lowest":
                t[g.random(t.shape) < 0.5] = np.finfo(np.float32).min
                t[g.random(t.shape) < 0.2] = -1e9
            self.bias = positions.bias_by_distance(t, self.bounds, md, self.S)
        qkv = np.concatenate([self.q, self.k, self.v], 1)
        self.o, lse = model.attention_fwd(qkv, self.B, self.S, self.H, self.dh, bias=self.bias)
        self.lse2 = lse / np.log(2.0)
        self.qkv = qkv

    def device(self):
        import torch
        tab = {}
        if self.nb:
            tab = dict(table=dev(self.table), bounds=torch.from_numpy(self.bounds).cuda(), max_distance=self.md)
        qk = torch.full((self.T, 2 * self.d + 8), float("nan"), device="cuda").to(dev(self.q[:1], self.dtype).dtype)
        vv = torch.full((self.T, self.d + 40), float("nan"), device="cuda").to(qk.dtype)
        qk[:, :self.d], qk[:, self.d:2 * self.d], vv[:, 32:32 + self.d] = (dev(t, self.dtype) for t in (self.q, self.k, self.v))
        return (qk[:, :self.d], qk[:, self.d:2 * self.d], vv[:, 32:32 + self.d]), dict(batch=self.B, n_heads=self.H, **tab)

    def split(self, a):
        return a.reshape(self.B, self.S, self.H, self.dh).transpose(0, 2, 1, 3)

    def merge(self, a):
        return a.transpose(0, 2, 1, 3).reshape(self.T, self.d)

    def probs(self, lse2):
        """P and the fp32 error of a score: dh + 4 roundings of sum |q k| / sqrt(dh), the bias and the statistic's
        own value among them, in natural units."""
        q, k = self.split(self.q), self.split(self.k)
        sc = 1 / np.sqrt(self.dh)
        bias = np.zeros((self.H, self.S, self.S))
        i = np.arange(self.S)
        dist = i[:, None] - i
        if self.bias is not None:
            bias = self.bias[:, np.maximum(dist, 0)]
        s = np.where(dist < 0, -np.inf, q @ k.transpose(0, 1, 3, 2) * sc + bias)
        l = lse2.reshape(self.B, self.H, self.S, 1) * np.log(2.0)
        P = np.exp(s - np.where(l == -np.inf, np.inf, l))
        err = (self.dh + 4) * U32 * (np.abs(q) @ np.abs(k).transpose(0, 1, 3, 2)) * sc
        err += 8 * U32 * (np.abs(np.where(np.isfinite(bias), bias, 0.0)) + np.abs(np.where(np.isfinite(l), l, 0.0)))
        return P, np.where(P > 0, err, 0.0)


def _attn_cases():
    return [(c, t) for t in ("bf16", "fp32") for c in ATTN] + [(c, "bf16") for c in ATTN128 + ATTN_MANY]


@pytest.mark.parametrize("case,dtype", _attn_cases(), ids=lambda c: "-".join(map(str, c)) if isinstance(c, tuple) else c)
def test_attention(binding, case, dtype):
    import torch
    c = Attn(case, dtype, 3)
    print(f"attention {case} {dtype}", flush=True)
    (q, k, v), kw = c.device()
    u = half_step(dtype)
    o = torch.full((c.T, c.d), float("nan"), device="cuda", dtype=q.dtype)
    lse2 = torch.full((c.B * c.H, c.S), float("nan"), device="cuda")
    binding.attention(q, k, v, o, lse2, **kw)
    P, err = c.probs(c.lse2.reshape(c.B * c.H, c.S))
    # a probability's relative error: its score's, the statistic's (a mean of the scores') and S + 8 additions
    rel = 2 * err.max() + (c.S + 16) * U32
    pv = c.merge(P @ np.abs(c.split(c.v)))
    unbiased = 0.0 if c.nb else u   # without a bias the statistic sums rounded probabilities
    check(host(o), c.o, (u + unbiased + rel) * pv + u * np.abs(c.o) if dtype == "bf16" else rel * pv + u * np.abs(c.o), "o")
    finite = np.where(np.isfinite(c.lse2), np.abs(c.lse2), 0.0).reshape(c.B * c.H, c.S)
    stat = c.lse2.reshape(c.B * c.H, c.S)
    check(host(lse2), stat, (rel + (unbiased if dtype == "bf16" else 0.0)) / np.log(2.0) + 4 * U32 * finite, "lse2")

    # backward of the o and lse2 that the kernel left
    do = dev(c.do, dtype)
    dq, dk, dv = (torch.full((c.T, c.d + 16), float("nan"), device="cuda", dtype=q.dtype) for _ in range(3))
    start = np.float32(np.random.default_rng(4).standard_normal((max(c.nb, 1), c.H)))
    g_table = dev(start) if c.nb else None
    binding.attention_backward(q, k, v, o, lse2, do, dq[:, :c.d], dk[:, :c.d], dv[:, :c.d], g_table=g_table, **kw)
    P, err = c.probs(host(lse2))
    Q, K, V, dO, O = (c.split(a) for a in (c.q, c.k, c.v, c.do, host(o)))
    sc = 1 / np.sqrt(c.dh)
    D = (dO * O).sum(-1, keepdims=True)
    dS = P * (dO @ V.transpose(0, 1, 3, 2) - D)
    # dS: (dh + 4) roundings of sum |dO v| + sum |dO o|, and the relative error of P
    mass = np.abs(dO) @ np.abs(V).transpose(0, 1, 3, 2) + (np.abs(dO) * np.abs(O)).sum(-1, keepdims=True)
    e_s = P * mass * (c.dh + 8) * U32 + np.abs(dS) * (err + 8 * U32)
    r = u if dtype == "bf16" else 0.0   # dS and P rounded before their products
    acc = (c.S + 8) * U32               # additions of the products
    want = {"dq": dS @ K * sc, "dk": dS.transpose(0, 1, 3, 2) @ Q * sc, "dv": P.transpose(0, 1, 3, 2) @ dO}
    absd = np.abs(dS)
    tol = {"dq": (((r + acc) * absd + e_s) @ np.abs(K)) * sc,
           "dk": (((r + acc) * absd + e_s).transpose(0, 1, 3, 2) @ np.abs(Q)) * sc,
           "dv": ((r + acc + err + 8 * U32) * P).transpose(0, 1, 3, 2) @ np.abs(dO)}
    for name, got in (("dq", dq), ("dk", dk), ("dv", dv)):
        check(host(got[:, :c.d]), c.merge(want[name]), c.merge(tol[name] + 1.01 * u * np.abs(want[name])) + 1e-37, name)
        assert torch.isnan(got[:, c.d:]).all(), name
    if not c.nb:
        return
    g = positions.table_grad(dS.sum(0), c.bounds, c.md)
    # additions on the way: of a tile's diagonal, along the sequence, over waves, blocks and sequences
    t = positions.table_grad((e_s + 64 * U32 * absd).sum(0), c.bounds, c.md) + 2 * U32 * np.abs(start)
    check(host(g_table), g + start, t + U32 * np.abs(g), "g_table")
    again = dev(start)
    binding.attention_backward(q, k, v, o, lse2, do, dq[:, :c.d], dk[:, :c.d], dv[:, :c.d], g_table=again, **kw)
    assert torch.equal(again, g_table), "two runs differ"


def test_attention_without_tokens(binding):
    import torch
    x = torch.empty(0, 64, device="cuda")
    for batch in (0, 2):
        lse2 = torch.empty(batch, 0, device="cuda")
        binding.attention(x, x, x, x, lse2, batch, 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("entry", [1e8, 3e38])
def test_attention_with_an_entry_beyond_every_score(binding, dtype, entry):
    """One distance outweighs all others in every head: each query returns the value that far back, the first ones
    what they would without it; the gradient of that query's scores vanishes and everything stays finite."""
    import torch
    B, S, H, dh, far = 2, 140, 2, 64, 3
    c = Attn((B, S, H, dh, 8, 7, ""), dtype, 6)
    c.bounds = np.arange(8, dtype=np.int32)   # a bucket per distance
    c.table[far] = entry
    (q, k, v), kw = c.device()
    o, lse2 = torch.empty(c.T, c.d, device="cuda", dtype=q.dtype), torch.empty(B * H, S, device="cuda")
    binding.attention(q, k, v, o, lse2, **kw)
    got, val = c.split(host(o)), c.split(c.v)
    # the one probability left is 2^e, e the rounding of a running maximum near 1e8 (not 0): in bf16 it is rounded
    # to 2^e (1 + u) before its product, against 2^e in the normaliser, and the output is rounded: (1 + u)^2 - 1.
    # In fp32: 1 / l, its product and the output, and the error of 2^e cancels
    u = half_step(dtype)
    check(got[:, :, far:], val[:, :, :-far], ((2.01 * u if dtype == "bf16" else u) + 4 * U32) * np.abs(val[:, :, :-far]), "o")
    assert torch.isfinite(lse2).all()
    grads = [torch.empty(c.T, c.d, device="cuda", dtype=q.dtype) for _ in range(3)]
    g_table = torch.zeros(8, H, device="cuda")
    binding.attention_backward(q, k, v, o, lse2, dev(c.do, dtype), *grads, g_table=g_table, **kw)
    assert all(torch.isfinite(t).all() for t in grads + [g_table])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_offsets_beyond_32_bits(binding, dtype):
    """Rows of one sequence further apart than 2^31 elements: the bits of the same call on dense copies."""
    import torch
    B, S, dh, ld = 2, 20000, 64, 131072
    T, act = B * S, torch.bfloat16 if dtype == "bf16" else torch.float32
    torch.manual_seed(4)
    wide, out = (torch.empty(T, ld, device="cuda", dtype=act) for _ in range(2))
    dense = torch.randn(T, 3 * dh, device="cuda").to(act)
    # the third columns end a row, so the last row's end is the buffer's
    cols = [slice(0, dh), slice(4096, 4096 + dh), slice(ld - dh, ld)]
    for i, c in enumerate(cols):
        wide[:, c] = dense[:, i * dh:(i + 1) * dh]
    gain, do = torch.rand(dh, device="cuda") + 0.5, torch.randn(T, dh, device="cuda").to(act)
    freq = torch.from_numpy(binding.rope_freqs(1e4, dh)).cuda()
    table, bounds = torch.randn(32, 1, device="cuda"), torch.from_numpy(binding.rel_bounds(32, 128)).cuda()
    rot = dict(q_heads=1, k_heads=0, seq=S, q_gain=gain, freq=freq)
    rel = dict(batch=B, n_heads=1, table=table, bounds=bounds, max_distance=128)

    def chain(x, y, g):
        """x: three columns of inputs, y: of results (the rotation and its backward in the last)."""
        o, lse2 = torch.empty(T, dh, device="cuda", dtype=act), torch.empty(B, S, device="cuda")
        binding.attention(*x, o, lse2, **rel)
        binding.attention_backward(*x, o, lse2, do, *y, g_table=g[0], **rel)
        grads = [t.clone() for t in y]
        binding.qk_norm_rope(x[2], y[2], **rot)
        turned = y[2].clone()
        binding.qk_norm_rope_backward(x[2], y[2], y[2], g_q_gain=g[1], g_bias=g[2], **rot)
        return [o, lse2, *grads, turned, y[2].clone(), *g]

    def zeros():
        return [torch.zeros(32, 1, device="cuda"), torch.zeros(dh, device="cuda"), torch.zeros(dh, device="cuda")]
    near = chain(list(dense.split(dh, 1)), [torch.empty(T, dh, device="cuda", dtype=act) for _ in range(3)], zeros())
    far = chain([wide[:, c] for c in cols], [out[:, c] for c in cols], zeros())
    for i, (a, b) in enumerate(zip(near, far)):
        assert torch.isfinite(a).all() and torch.equal(a, b), i


def test_calls_at_once_on_two_streams(binding):
    """Two chains of different sizes enqueued side by side, workspaces from the allocator: the bits of each alone."""
    import torch
    torch.manual_seed(9)

    def make(B, S, H, dh, act):
        d, T = H * dh, B * S
        x, do = torch.randn(T, 3 * d, device="cuda").to(act), torch.randn(T, d, device="cuda").to(act)
        gain, table = torch.rand(dh, device="cuda") + 0.5, torch.randn(16, H, device="cuda")
        freq, bounds = torch.from_numpy(binding.rope_freqs(1e4, dh)).cuda(), torch.from_numpy(binding.rel_bounds(16, 50)).cuda()
        rot = dict(q_heads=H, k_heads=H, seq=S, q_gain=gain, k_gain=gain, freq=freq)
        rel = dict(batch=B, n_heads=H, table=table, bounds=bounds, max_distance=50)

        def chain():
            qk, o, lse2 = torch.empty(T, 2 * d, device="cuda", dtype=act), torch.empty_like(do), torch.empty(B * H, S, device="cuda")
            dqkv, g = torch.empty_like(x), torch.zeros(2 * dh + 16 * H, device="cuda")
            gq, gk, gt = g.split([dh, dh, 16 * H])
            binding.qk_norm_rope(x[:, :2 * d], qk, **rot)
            q, k = qk.split(d, 1)
            binding.attention(q, k, x[:, 2 * d:], o, lse2, **rel)
            binding.attention_backward(q, k, x[:, 2 * d:], o, lse2, do, *dqkv.split(d, 1), g_table=gt.view(16, H), **rel)
            binding.qk_norm_rope_backward(x[:, :2 * d], dqkv[:, :2 * d], dqkv[:, :2 * d], g_q_gain=gq, g_k_gain=gk, **rot)
            return o, lse2, dqkv, g
        return chain
    chains = [make(4, 300, 8, 64, torch.bfloat16), make(2, 190, 4, 32, torch.float32)]
    alone = [c() for c in chains]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in chains]
    got = [[], []]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(chains[i]())
    torch.cuda.synchronize()
    for i, runs in enumerate(got):
        for r in runs:
            for a, b in zip(alone[i], r):
                assert torch.equal(a, b), i


def test_first_call_of_a_process_can_be_captured(binding, root):
    """A fresh process whose first device work of this library is under capture."""
    import subprocess
    import sys
    code = """
import sys
sys.path.insert(0, {root!r})
import torch
from paper_2606_07881_amd import binding
x = torch.randn(64, 192, device="cuda")
y, o, l = torch.empty(64, 128, device="cuda"), torch.empty(64, 64, device="cuda"), torch.empty(4, 32, device="cuda")
g, t = torch.ones(32, device="cuda"), torch.zeros(8, 2, device="cuda")
b = torch.from_numpy(binding.rel_bounds(8, 20)).cuda()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
def chain():
    binding.qk_norm_rope(x[:, :128], y, 2, 2, seq=32, q_gain=g, k_gain=g)
    binding.attention(y[:, :64], y[:, 64:], x[:, 128:], o, l, 2, 2, t, b, 20)
with torch.cuda.graph(graph):
    chain()
for _ in range(3):
    x.normal_()
    graph.replay()
    a = o.clone()
    chain()
    torch.cuda.synchronize()
    assert torch.equal(a, o)
print("replays agree")
""".format(root=root)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "replays agree" in r.stdout, r.stdout + r.stderr
