"""Stages with norms and rotation of the query and key heads and a relative position bias
inside their attention: replays against the oracle, as in test_gpu_stage.py (the same
protocol and tolerances), and the operators run one after the other as a block runs them."""
import numpy as np
import pytest

from parity import (Inputs, compare_replays, drift_check, forced_oracle, gpu_replay, oracle_replay, rel_err, small_cfg,
                    stash_oracle, to_host, to_torch, tol)
from paper_2606_07881_amd import inputs

pytestmark = pytest.mark.gpu

NORM, ROPE, REL = dict(qk_norm=1), dict(rope_dims=32, rope_theta=100.0), dict(rel_buckets=16, rel_max_distance=60)
ALL = dict(NORM, **ROPE, **REL)
# workload -> overrides. Gains and tables start away from their defaults (see _inputs).
CASES = {
    "norm_ckpt_tiny_fp32": ("ckpt_tiny_fp32", NORM),
    "rope_ragged_fp32": ("ragged_fp32", ROPE),
    "rel_ragged_fp32": ("ragged_fp32", REL),
    "all_ragged_fp32": ("ragged_fp32", dict(ALL, rope_pairs="adjacent")),
    "all_dh64_fp32": ("dh64_fp32", dict(ALL, rope_dims=64)),
    "norm_ragged_bf16": ("ragged_bf16", NORM),
    "rope_ragged_bf16": ("ragged_bf16", dict(ROPE, rope_dims=64)),
    "rel_ragged_bf16": ("ragged_bf16", REL),
    "all_ragged_bf16": ("ragged_bf16", ALL),
    # a table of 24 elements: the tensors behind it begin 16 bytes off a 32-byte boundary
    "rel8_ragged_bf16": ("ragged_bf16", dict(ALL, rel_buckets=8, rel_max_distance=100)),
    "all_dh128_bf16": ("dh128_bf16", dict(ALL, rope_dims=128, rope_pairs="adjacent")),
    "all_dh32_bf16": ("dh32_bf16", ALL),
    "all_ckpt_ragged_bf16": ("ckpt_ragged_bf16", ALL),
    "all_win_bf16": ("win_bf16", ALL),
    "all_first_bf16": ("first_bf16", ALL),
    "all_last_bf16": ("last_bf16", ALL),
    "all_fused_last_bf16": ("fused_last_bf16", ALL),
    "all_drop_ragged_bf16": ("drop_ragged_bf16", ALL),
    "all_drop_ragged_fp32": ("drop_ragged_fp32", ALL),
}


def _inputs(c, seed, M):
    """Inputs with gains 1 +- 0.3 and bias tables of unit size."""
    inp = Inputs(c, seed, M)
    g = np.random.default_rng(seed + 100)
    for n, a in inp.params.items():
        leaf = n.split(".")[-1]
        if leaf in ("q_g", "k_g"):
            inp.params[n] = np.float32(1 + 0.3 * g.standard_normal(a.shape))
        elif leaf == "rel":
            inp.params[n] = np.float32(g.standard_normal(a.shape))
    return inp


@pytest.fixture(scope="module")
def binding():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no HIP device")
    from paper_2606_07881_amd import binding as b
    return b


@pytest.mark.parametrize("name", list(CASES))
def test_replay_parity(binding, name):
    base, over = CASES[name]
    c = small_cfg(base, **over)
    c["name"] = name
    inp = _inputs(c, 1, c["M"])
    print(f"{name}: replay of {c['M']} micro-batches", flush=True)
    g = gpu_replay(c, inp)
    rep = compare_replays(c, g, forced_oracle(c, inp, g), theta0=inp.params)
    print(name, {k: f"{v:.2e}" for k, v in rep.items()}, flush=True)
    assert g["counters"]["version"] == c["M"] // c["K"]


def test_a_stale_backward_keeps_its_forward_s_bias(binding):
    """At a raised learning rate the tables move by 1e-2 an update. A backward differentiates the
    probabilities of its forward: the fp32 replay is within 1e-4 of that, and the gains and weights are
    the ones current now, at least 3 tolerances away from weight stashing."""
    c = small_cfg("ragged_fp32", lr=1e-2, **ALL)
    inp = _inputs(c, 3, c["M"])
    g = gpu_replay(c, inp)
    o = forced_oracle(c, inp, g)
    rep = compare_replays(c, g, o, theta0=inp.params)
    checked, closest = drift_check(c, g, o, stash_oracle(c, inp, g))
    print({k: f"{v:.2e}" for k, v in rep.items()}, checked, f"{closest:.1f}", flush=True)
    assert checked > 0


def test_options_left_off_are_the_plain_stage(binding):
    """All options zero: the bits of a stage whose configuration does not mention them."""
    c = small_cfg("ragged_bf16")
    inp = Inputs(c, 2, 4)
    a = gpu_replay(c, inp)
    b = gpu_replay(dict(c, qk_norm=0, rope_dims=0, rel_buckets=0, rel_max_distance=0), inp)
    for x, y in zip(a["out"] + a["grad_in"], b["out"] + b["grad_in"]):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_operators_in_line_are_the_block_s(binding, dtype):
    """One block with every option against the operators called one after the other on the same projection: the
    attention's input is normalised and rotated, biased attention reads it, and the backwards run in reverse in
    the projection's gradient buffer. Both sides against the oracle of the whole chain."""
    import torch
    from oracle import model
    B, S, H, dh = 2, 90, 3, 64
    d, T = H * dh, B * S
    cfg = dict(n_heads=H, head_dim=dh, d_model=d, seq=S, micro_batch=B, ln_eps=1e-5, **dict(ALL, rope_dims=dh))
    g = np.random.default_rng(8)
    act = torch.bfloat16 if dtype == "bf16" else torch.float32
    cast = (lambda a: inputs.bf16_round(np.float32(a))) if dtype == "bf16" else np.float32
    qkv, do = cast(g.standard_normal((T, 3 * d))), cast(g.standard_normal((T, d)))
    p = dict(q_g=np.float32(1 + 0.3 * g.standard_normal(dh)), k_g=np.float32(1 + 0.3 * g.standard_normal(dh)),
             rel=np.float32(g.standard_normal((16, H))))
    p64 = {k: v.astype(np.float64) for k, v in p.items()}
    att, bias = model.position_fwd(qkv.astype(np.float64), p64, cfg)
    o64, lse = model.attention_fwd(att, B, S, H, dh, bias=bias)
    datt, ds = model.attention_bwd(do.astype(np.float64), att, lse, B, S, H, dh, bias=bias)
    dqkv64, grads = model.position_bwd(datt, ds, qkv.astype(np.float64), p64, cfg)

    x = torch.from_numpy(qkv).cuda().to(act)
    dev = {k: torch.from_numpy(v).cuda() for k, v in p.items()}
    freq = torch.from_numpy(binding.rope_freqs(100.0, dh)).cuda()
    bounds = torch.from_numpy(binding.rel_bounds(16, 60)).cuda()
    rot = dict(q_heads=H, k_heads=H, seq=S, q_gain=dev["q_g"], k_gain=dev["k_g"], eps=1e-5, freq=freq)
    rel = dict(batch=B, n_heads=H, table=dev["rel"], bounds=bounds, max_distance=60)
    G = {k: torch.zeros_like(v) for k, v in dev.items()}
    gb = torch.zeros(3 * d, device="cuda")

    def chain():
        qk = torch.empty(T, 2 * d, device="cuda", dtype=act)
        o, lse2 = torch.empty(T, d, device="cuda", dtype=act), torch.empty(B * H, S, device="cuda")
        dqkv = torch.empty_like(x)
        binding.qk_norm_rope(x[:, :2 * d], qk, **rot)
        q, k = qk.split(d, 1)
        binding.attention(q, k, x[:, 2 * d:], o, lse2, **rel)
        dq, dk, dv = dqkv.split(d, 1)
        binding.attention_backward(q, k, x[:, 2 * d:], o, lse2, torch.from_numpy(do).cuda().to(act), dq, dk, dv,
                                   g_table=G["rel"], **rel)
        binding.qk_norm_rope_backward(x[:, :2 * d], dqkv[:, :2 * d], dqkv[:, :2 * d], g_q_gain=G["q_g"],
                                      g_k_gain=G["k_g"], g_bias=gb[:2 * d], **rot)
        return o, dqkv
    o, dqkv = chain()
    c = dict(dtype=dtype)
    assert rel_err(to_host(o), o64) <= tol(c, "act")
    assert rel_err(to_host(dqkv), dqkv64) <= tol(c, "grad")
    for k in G:
        assert rel_err(to_host(G[k]), grads[k]) <= tol(c, "grad"), k
    assert rel_err(to_host(gb[:2 * d]), dqkv64[:, :2 * d].sum(0)) <= tol(c, "grad")
    # another stream, and with its gradients added a second time
    first = {k: v.clone() for k, v in G.items()}
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        o2, dqkv2 = chain()
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(o, o2) and torch.equal(dqkv, dqkv2)
    for k in G:
        assert rel_err(to_host(G[k]), 2 * to_host(first[k])) <= 1e-6, k


def test_captured_chain_replays(binding):
    """Forward and backward of both operators in one graph, replayed with eager work between: every replay gives
    the eager bits, on inputs that change in place. Two graphs share nothing but the inputs."""
    import torch
    B, S, H, dh = 2, 130, 4, 64
    d, T = H * dh, B * S
    torch.manual_seed(0)
    x = torch.randn(T, 3 * d, device="cuda").bfloat16()
    do = torch.randn(T, d, device="cuda").bfloat16()
    gain = torch.rand(dh, device="cuda") + 0.5
    table = torch.randn(32, H, device="cuda")
    freq = torch.from_numpy(binding.rope_freqs(1e4, dh)).cuda()
    bounds = torch.from_numpy(binding.rel_bounds(32, 128)).cuda()
    rot = dict(q_heads=H, k_heads=H, seq=S, q_gain=gain, k_gain=gain, freq=freq)
    rel = dict(batch=B, n_heads=H, table=table, bounds=bounds, max_distance=128)

    def buffers():
        z = lambda *s, t=torch.bfloat16: torch.zeros(*s, device="cuda", dtype=t)  # noqa: E731
        return dict(qk=z(T, 2 * d), o=z(T, d), lse2=z(B * H, S, t=torch.float32), dqkv=z(T, 3 * d),
                    g=z(2 * dh + 2 * d + 32 * H, t=torch.float32))

    def chain(b):
        b["g"].zero_()
        gq, gk, gb, gt = b["g"].split([dh, dh, 2 * d, 32 * H])
        binding.qk_norm_rope(x[:, :2 * d], b["qk"], **rot)
        q, k = b["qk"].split(d, 1)
        binding.attention(q, k, x[:, 2 * d:], b["o"], b["lse2"], **rel)
        dq, dk, dv = b["dqkv"].split(d, 1)
        binding.attention_backward(q, k, x[:, 2 * d:], b["o"], b["lse2"], do, dq, dk, dv, g_table=gt.view(32, H), **rel)
        binding.qk_norm_rope_backward(x[:, :2 * d], b["dqkv"][:, :2 * d], b["dqkv"][:, :2 * d], g_q_gain=gq, g_k_gain=gk,
                                      g_bias=gb, **rot)
    eager, a, b = buffers(), buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(a)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for buf in (a, b):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            chain(buf)
        graphs.append(graph)
    for i in range(4):
        x.copy_(torch.randn(T, 3 * d, device="cuda"))
        chain(eager)
        for graph, buf in zip(graphs, (a, b)):
            graph.replay()
        torch.cuda.synchronize()
        for buf in (a, b):
            for n in eager:
                assert torch.equal(buf[n], eager[n]), (i, n)
