"""Pins of the oracle's position operators: differences, special cases, and torch's complex
numbers and automatic differentiation as an independent implementation."""
import numpy as np
import pytest
import torch

from oracle import model, positions, stage


def _rotary_case(pairs, norm, seed=0):
    g = np.random.default_rng(seed)
    T, H, dh, R = 4, 3, 8, 4
    gain = 1 + 0.3 * g.standard_normal((H, dh)) if norm else None
    return g.standard_normal((T, H, dh)), gain, g.integers(-9, 9, T), positions.freqs(100.0, R), g.standard_normal((T, H, dh))


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
@pytest.mark.parametrize("norm", [True, False])
def test_norm_rope_gradients_match_central_differences(pairs, norm):
    x, gain, pos, freq, dy = _rotary_case(pairs, norm)
    dx, dg = positions.norm_rope_bwd(dy, x, gain, pos, freq, pairs)
    h = 1e-6
    for arr, grad in ((x, dx), (gain, dg)):
        if arr is None:
            assert grad is None
            continue
        for ix in np.ndindex(arr.shape):
            old = arr[ix]
            arr[ix] = old + h
            a = (positions.norm_rope_fwd(x, gain, pos, freq, pairs) * dy).sum()
            arr[ix] = old - h
            b = (positions.norm_rope_fwd(x, gain, pos, freq, pairs) * dy).sum()
            arr[ix] = old
            assert abs((a - b) / (2 * h) - grad[ix]) < 1e-7


@pytest.mark.parametrize("pairs", ["half", "adjacent"])
def test_rotation_is_a_complex_product_and_relative(pairs):
    x, _, pos, freq, _ = _rotary_case(pairs, False)
    y = positions.rotate(x, pos, freq, pairs)
    R = 2 * len(freq)
    a, b = (x[..., :R // 2], x[..., R // 2:R]) if pairs == "half" else (x[..., 0:R:2], x[..., 1:R:2])
    z = (a + 1j * b) * np.exp(1j * pos[:, None, None] * freq)
    got = (y[..., :R // 2], y[..., R // 2:R]) if pairs == "half" else (y[..., 0:R:2], y[..., 1:R:2])
    np.testing.assert_allclose(got[0], z.real, atol=1e-14)
    np.testing.assert_allclose(got[1], z.imag, atol=1e-14)
    np.testing.assert_array_equal(y[..., R:], x[..., R:])
    # products of rotated heads depend on the distance of their positions alone
    moved = positions.rotate(x, pos + 7, freq, pairs)
    np.testing.assert_allclose((y[0] * y[1]).sum(-1), (moved[0] * moved[1]).sum(-1), atol=1e-13)
    np.testing.assert_allclose(positions.rotate(y, pos, freq, pairs, -1), x, atol=1e-14)


def test_bounds_and_buckets():
    assert positions.bounds(8, 16) == [0, 1, 2, 3, 4, 6, 8, 12]
    # whole powers, where a floating-point logarithm misses: e = 16, ratio 16, steps of a quarter octave
    assert positions.bounds(32, 256)[16:] == [16, 20, 23, 27, 32, 39, 46, 54, 64, 77, 91, 108, 128, 153, 182, 216]
    b = positions.buckets([0, 1, 2, 4], 3, 8)
    assert b.tolist() == [0, 1, 2, 2, 2, 2, 2, 2]   # max_distance 3 never reaches the last bound


def _attn_case(hidden, seed=1):
    g = np.random.default_rng(seed)
    mu, S, H, dh, nb, md = 2, 7, 2, 4, 4, 5
    bnd = positions.bounds(nb, md)
    table = g.standard_normal((nb, H))
    if hidden:
        table[0, 0] = -np.inf
    return mu, S, H, dh, bnd, md, table, g.standard_normal((mu * S, 3 * H * dh)), g.standard_normal((mu * S, H * dh))


@pytest.mark.parametrize("hidden", [False, True])
def test_biased_attention_matches_automatic_differentiation(hidden):
    mu, S, H, dh, bnd, md, table, qkv, do = _attn_case(hidden)
    bias = positions.bias_by_distance(table, bnd, md, S)
    o, lse = model.attention_fwd(qkv, mu, S, H, dh, bias=bias)
    dqkv, ds = model.attention_bwd(do, qkv, lse, mu, S, H, dh, bias=bias)
    g_table = positions.table_grad(ds, bnd, md)
    x = torch.tensor(qkv, requires_grad=True)
    tb = torch.tensor(table, requires_grad=True)
    q, k, v = x.reshape(mu, S, 3, H, dh).permute(2, 0, 3, 1, 4)
    i = torch.arange(S)
    idx = torch.tensor(positions.buckets(bnd, md, S))[(i[:, None] - i).clamp(min=0)]
    s = q @ k.transpose(-1, -2) / dh ** 0.5 + tb[idx].permute(2, 0, 1)
    s = s.masked_fill(i[:, None] < i, -torch.inf)
    empty = (s == -torch.inf).all(-1, keepdim=True)
    p = s.masked_fill(empty, 0.0).softmax(-1).masked_fill(empty, 0.0)
    ref = (p @ v).transpose(1, 2).reshape(mu * S, H * dh)
    ref.backward(torch.tensor(do))
    np.testing.assert_allclose(o, ref.detach().numpy(), atol=1e-13)
    np.testing.assert_allclose(dqkv, x.grad.numpy(), atol=1e-12)
    np.testing.assert_allclose(g_table, tb.grad.numpy(), atol=1e-12)
    assert (np.isneginf(lse[:, 0, 0])).all() == hidden   # the first query of head 0 sees only itself


def test_biased_attention_gradients_match_central_differences():
    mu, S, H, dh, bnd, md, table, qkv, do = _attn_case(False)

    def f():
        return (model.attention_fwd(qkv, mu, S, H, dh, bias=positions.bias_by_distance(table, bnd, md, S))[0] * do).sum()
    bias = positions.bias_by_distance(table, bnd, md, S)
    _, lse = model.attention_fwd(qkv, mu, S, H, dh, bias=bias)
    dqkv, ds = model.attention_bwd(do, qkv, lse, mu, S, H, dh, bias=bias)
    h = 1e-6
    for arr, grad in ((table, positions.table_grad(ds, bnd, md)), (qkv, dqkv)):
        for ix in list(np.ndindex(arr.shape))[::3]:
            old = arr[ix]
            arr[ix] = old + h
            a = f()
            arr[ix] = old - h
            b = f()
            arr[ix] = old
            assert abs((a - b) / (2 * h) - grad[ix]) < 1e-7, ix


POSITION_CFG = dict(n_layers=2, d_model=8, n_heads=2, head_dim=4, d_ff=32, seq=5, micro_batch=2, vocab=11, max_pos=7,
                    ln_eps=1e-5, qk_norm=1, rope_dims=4, rope_theta=50.0, rel_buckets=4, rel_max_distance=4)


@pytest.mark.parametrize("kind", ["middle", "first", "last"])
@pytest.mark.parametrize("over", [{}, dict(rope_pairs="adjacent"), dict(qk_norm=0), dict(rope_dims=0), dict(rel_buckets=0)],
                         ids=str)
def test_stage_gradients_match_central_differences(kind, over):
    """The whole stage function with its position options, every parameter."""
    cfg = dict(POSITION_CFG, kind=kind, **over)
    g = np.random.default_rng(5)
    theta = {n: (1 + 0.2 * g.standard_normal(s)) if n.endswith("_g") else 0.3 * g.standard_normal(s)
             for n, s in stage.param_shapes(cfg)}
    T = cfg["micro_batch"] * cfg["seq"]
    inp = g.integers(0, 11, (2, 5)) if kind == "first" else g.standard_normal((T, 8))
    tgt = g.integers(0, 11, (2, 5)) if kind == "last" else None
    dy = None if kind == "last" else g.standard_normal((T, 8))

    def f():
        out, _ = stage.stage_fwd(cfg, theta, inp, tgt)
        return out if kind == "last" else float((out * dy).sum())
    _, saved = stage.stage_fwd(cfg, theta, inp, tgt)
    _, grads = stage.stage_bwd(cfg, theta, saved, dy, 1, ids=inp if kind == "first" else None)
    assert sorted(grads) == sorted(theta)
    h = 1e-6
    for name, arr in theta.items():
        idx = list(np.ndindex(arr.shape))
        for ix in [idx[i] for i in g.permutation(len(idx))[:12]]:
            old = arr[ix]
            arr[ix] = old + h
            a = f()
            arr[ix] = old - h
            b = f()
            arr[ix] = old
            fd = (a - b) / (2 * h)
            assert abs(grads[name][ix] - fd) <= 1e-7 * max(1.0, abs(fd)) + 1e-8, (name, ix)


def test_entries_count_within_2_to_the_15():
    t = np.float32([[-3e38], [-32768.0], [-32767.0], [32767.0], [32769.0], [3e38]])
    got = positions.bias_by_distance(t, list(range(6)), 5, 6)[0]
    assert got.tolist() == [-np.inf, -np.inf, -32767.0, 32767.0, 32768.0, 32768.0]
