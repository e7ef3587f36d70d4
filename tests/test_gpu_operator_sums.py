"""The parameter gradients of the norms and the rotation, to a tolerance that a single lost head of a single token would
exceed: the sums over tokens are spread over workgroups, threads and a second launch, each with remainders of its own."""
import numpy as np
import pytest

from oracle import positions
from test_gpu_operators import ROTARY, Rotary, check, host, rounded

U32 = 2.0 ** -24
# more tokens than one round of workgroups takes, with remainders; few and many heads, and heads over two workgroups
CASES = ROTARY + [(4099, 16, 16, 64, 64, "half", True, "seq"), (5003, 3, 2, 64, 32, "adjacent", True, "given"),
                  (3001, 12, 4, 96, 96, "half", True, "far"), (1501, 40, 24, 256, 256, "half", True, "seq"),
                  (6007, 1, 0, 128, 128, "half", True, "seq"), (2049, 5, 3, 80, 0, "half", True, "seq")]


def make(case, dtype):
    """A Rotary case whose tokens all weigh about the same: magnitudes of 0.5 to 1.5."""
    c = Rotary(case, dtype, 21)
    g = np.random.default_rng(22)
    c.x, c.dy = (rounded(g.uniform(0.5, 1.5, c.x.shape) * g.choice([-1, 1], c.x.shape) * s, dtype) for s in (1, 1e-2))
    return c


def terms(c):
    """What the sums add, [T, heads, dh] each, and the error of every term: (dn xh, its error, dx, its error).

    dn turns dy back: with m the sum of the absolute values of a pair, 24 roundings of m (its cosine and sine to 8, 12 at
    positions near 2^31, two products and a sum). xh: 16 relative ones (16 squares and 4 lane moves, halved by the root; the
    root and its product). Then e = dn gain and the mean of e xh (16 + 4 additions): below 96 of r (|e| + |xh| mean |e xh|)."""
    x, dy = c.heads(c.x), c.heads(c.dy)
    dx, _ = positions.norm_rope_bwd(dy, x, c.gain, c.at, c.freq, c.pairs, c.eps)
    m, R = np.abs(dy), 2 * len(c.freq)
    dn = positions.rotate(dy, c.at, c.freq, c.pairs, -1) if R else dy
    if R:
        a, b = (np.arange(R // 2), np.arange(R // 2) + R // 2) if c.pairs == "half" else (np.arange(0, R, 2), np.arange(1, R, 2))
        both = m[..., a] + m[..., b]
        m[..., a], m[..., b] = both, both
    if c.gain is None:
        return None, None, dx, 24 * U32 * m
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + c.eps)
    xh, e = np.abs(x * r), m * np.abs(c.gain)
    return dn * x * r, 48 * U32 * m * xh, dx, 96 * U32 * r * (e + xh * (e * xh).mean(-1, keepdims=True))


def sums(c):
    """(sum, tolerance, terms [.., members, columns]) of the query gains, the key gains and the column sums. Additions on the
    way of a term: the tokens of a thread (at least one workgroup a CU, which takes up to 512 lanes of a token: T / 256 and 4
    at most, times the workgroups of a token), 9 rounds over tokens and 10 over heads, 32 rows of partial sums to a thread and
    16 threads in the second launch, the buffer's value."""
    lanes = 1 << (c.dh // 16 - 1).bit_length()   # of a head
    n = c.T * (-(-(c.qh + c.kh) * lanes // 512)) / 256 + 72
    dg, t_g, dx, t_x = terms(c)
    out = []
    if dg is not None:
        for lo, hi in ((0, c.qh), (c.qh, c.qh + c.kh)):
            part, err = dg[:, lo:hi].reshape(-1, c.dh), t_g[:, lo:hi].reshape(-1, c.dh)
            out.append((part.sum(0), (err + n * U32 * np.abs(part)).sum(0), part))
    part, err = dx.reshape(c.T, -1), t_x.reshape(c.T, -1)
    return out + [(part.sum(0), (err + n * U32 * np.abs(part)).sum(0), part)]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_the_tolerances_see_a_lost_member(case):
    """On the host: without any one head of any one token a gain's sum, or without any one token the column sums, would be
    outside in some column."""
    for total, tol, members in sums(make(case, "fp32")):
        if members.size:
            seen = (np.abs(members) > 2 * tol).any(-1)
            assert seen.all(), f"{np.count_nonzero(~seen)} of {seen.size} members would not be missed"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_rotary_sums(case, dtype):
    import torch
    from paper_2606_07881_amd import binding
    c = make(case, dtype)
    kw = c.args()
    got = [torch.zeros(c.dh, device="cuda"), torch.zeros(c.dh, device="cuda"), torch.zeros(c.n, device="cuda")]
    x, dy = c.wide(c.x), c.wide(c.dy)
    gains = dict(g_q_gain=got[0], g_k_gain=got[1]) if c.gain is not None else {}
    binding.qk_norm_rope_backward(x[:, :c.n], dy[:, :c.n], dy[:, :c.n], g_bias=got[2], **gains, **kw)
    want = sums(c)
    for name, g, (total, tol, _) in zip(("g_q_gain", "g_k_gain", "g_bias")[-len(want):], got[-len(want):], want):
        check(host(g), total, tol, name)
