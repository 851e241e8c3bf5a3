"""The model path with its linears in 8-bit integers: blocks, stacks and whole chunks."""
import numpy as np
import pytest

import oracle as O
from harness import BlockRun, dev_bf16, host_bits, host_f32
from oracle import ardit_ref as R
from oracle import int_ref as I
from test_gpu_chunk import LQ, SH, Model, _sampler_bits
from workloads import WORKLOADS, BlockShape, bits_to_f32, normal_bf16
from workloads.gen import Workload, draw_block_case

pytestmark = pytest.mark.gpu

MATRICES = ("w_qkv", "w_o", "w_cq", "w_co", "w_1", "w_2")


@pytest.fixture(scope="module")
def A(gpu):
    from paper_2606_15319_amd import ardit
    return ardit


def _sync():
    import torch
    torch.cuda.synchronize()


def int_weights(A, w_dev, keep):
    """Codes and scales of a layer's six matrices (`keep` holds the buffers)."""
    import torch
    d = {}
    for name in MATRICES:
        w = w_dev[name]
        n, k = w.shape
        c = torch.empty((n, k), dtype=torch.int8, device="cuda")
        s = torch.empty(n, dtype=torch.float32, device="cuda")
        A.ardit_int_quantize(None, w, A.BF16, n, k, k, c, k, s)
        d[name], d["s" + name[1:]] = c, s
    keep.append(d)
    return A.block_weights_int(d)


def _reference(run, b):
    """Float64 block of stream b through quantised linears."""
    c, sh = run.case, run.shape
    w, eps, D = c.block_w, sh.eps, sh.dim
    q8 = {n: I.quantize(w[n])[:2] for n in MATRICES}

    def lin(x, name):
        return I.quantized_linear(x, *q8[name], np.asarray(w["b" + name[1:]], np.float64))

    m = O.time_modulation(c.t[b], c.time_w, D)
    M = R._modulation(m, w)
    kc, vc = O.context_kv(c.ctx[b], w, eps)
    x = c.x[b].astype(np.float64)
    z = lin(I.norm(x, eps, scale=M["scale1"], shift=M["shift1"]), "w_qkv")
    H, d = sh.n_heads, sh.head_dim
    where = O.chunk_positions(sh.frames, sh.lat_h, sh.lat_w, c.frame_pos0[b])
    q = O.rope3d(O.rms_norm(z[:, :D], eps, w["g_q"]).reshape(-1, H, d), where, sh.theta)
    k = O.rope3d(O.rms_norm(z[:, D:2 * D], eps, w["g_k"]).reshape(-1, H, d), where, sh.theta)
    v = z[:, 2 * D:].reshape(-1, H, d)
    keys, vals = k, v
    if c.cache_len[b]:
        keys = np.concatenate([c.cache_k[b].reshape(-1, H, d), k])
        vals = np.concatenate([c.cache_v[b].reshape(-1, H, d), v])
    o = O.attention(q, keys, vals).reshape(-1, D)
    x1 = x + M["gate1"] * lin(o, "w_o")
    qc = O.rms_norm(lin(I.norm(x1, eps, gain=w["g_n3"]), "w_cq"), eps, w["g_cq"])
    oc = O.attention(qc.reshape(-1, H, d), kc.reshape(-1, H, d), vc.reshape(-1, H, d)).reshape(-1, D)
    x2 = x1 + lin(oc, "w_co")
    u = O.gelu_tanh(lin(I.norm(x2, eps, scale=M["scale2"], shift=M["shift2"]), "w_1"))
    return x2 + M["gate2"] * lin(u, "w_2")


@pytest.mark.parametrize("name", ["tiny", "wide"])
def test_a_block(A, name):
    """The block against a float64 block of the same weight codes whose activations are quantised in
    float64, with gates near two, so that the branches are not small beside x.

    What the two sides do not share is the bf16 storage of the activations (2^-9 of a value on
    average); next to a border it moves a code by a step.  A step is max / 127, about 0.03 of a
    row's spread, so of a hundred codes about five move: 0.03 sqrt(0.05) = 0.7% of a linear's output
    for each of the six, below 2% in all of the branches' sum; the result's own rounding is 2^-9.
    Without codes the block is further away: a code's rounding alone is 0.03 / sqrt(12) = 0.9% of
    each linear's input, and as much again for its weights."""
    wl = WORKLOADS["tiny"] if name == "tiny" else Workload(
        wid=78, name="wide", cache_chunks=(2, 0, 1), frame_pos0=(4, 0, 9), ctx_len=24,
        shape=BlockShape(dim=256, n_heads=2, head_dim=128, ffn_dim=768, frames=2, lat_h=6, lat_w=12))
    case = draw_block_case(wl)
    case.block_w["mod_table"] = (case.block_w["mod_table"] + 2.0).astype(np.float32)
    run = BlockRun(wl, A, case=case)
    sh, c, L = run.shape, run.case, run.shape.chunk_tokens
    keep = []
    w8 = int_weights(A, run.w_dev, keep)
    run.run()               # (modulation and text keys and values)
    wts = A.block_weights({k: v for k, v in run.w_dev.items() if k not in MATRICES})
    run.out.fill_(float("nan"))
    A.ardit_stack_fwd_int(None, run.dims, run.batch, run.x, [run.pages.kv(A)], run.mod, [run.ctx_k], [run.ctx_v], [wts], [w8],
                          run.out, run.ws, run.ws_bytes)
    _sync()
    out = host_f32(run.out).astype(np.float64)
    for b in range(run.B):
        got = out[b * L:(b + 1) * L]
        ref = _reference(run, b)
        plain = run.reference(b)["out"]
        branch = np.linalg.norm(ref - c.x[b])
        assert branch > 0.3 * np.linalg.norm(c.x[b])
        far = np.linalg.norm(got - ref)
        assert far <= 0.02 * branch + 2.0 ** -9 * np.linalg.norm(ref), (far, branch)
        assert far < np.linalg.norm(got - plain)


@pytest.mark.parametrize("sparsity,quant", [(None, None), ([0.5, 0.0], None), (None, [1, 0])])
def test_a_stack_equals_its_layers(A, sparsity, quant):
    """Two layers in one call and one after the other: the same bits, also of the pages."""
    import torch
    wl = Workload(wid=79, name="two", cache_chunks=(2, 1), frame_pos0=(4, 9), ctx_len=24,
                  shape=BlockShape(dim=256, n_heads=2, head_dim=128, ffn_dim=768, frames=2, lat_h=8, lat_w=8))
    runs = [BlockRun(wl, A) for _ in range(2)]
    sh = runs[0].shape
    keep = []
    outs = []
    for way, run in enumerate(runs):
        batch = A.Batch([sh.chunk_tokens] * 2, run.case.cache_len, run.case.frame_pos0, [24, 24], sparsity, quant)
        n = A.ardit_workspace_size(run.dims, batch)
        ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        w, w8 = A.block_weights(run.w_dev), int_weights(A, run.w_dev, keep)
        other = {k: v.flip(0).contiguous() for k, v in run.w_dev.items()}
        keep.append(other)
        u, u8 = A.block_weights(other), int_weights(A, other, keep)
        run.run()                       # (modulation and text keys and values)
        k2, v2 = run.pages.k.clone(), run.pages.v.clone()
        kv2 = [run.pages.kv(A), A.kv_paged(k2, v2, run.pages.table, run.pages.n_pages, run.pages.max_frames)]
        if way == 0:
            A.ardit_stack_fwd_int(None, run.dims, batch, run.x, kv2, run.mod, [run.ctx_k] * 2, [run.ctx_v] * 2, [w, u],
                                  [w8, u8], run.out, ws, n)
        else:
            mid = torch.empty_like(run.out)
            A.ardit_stack_fwd_int(None, run.dims, batch, run.x, kv2[:1], run.mod, [run.ctx_k], [run.ctx_v], [w], [w8], mid,
                                  ws, n)
            A.ardit_stack_fwd_int(None, run.dims, batch, mid, kv2[1:], run.mod, [run.ctx_k], [run.ctx_v], [u], [u8],
                                  run.out, ws, n)
        _sync()
        outs.append([host_bits(t).copy() for t in (run.out, run.pages.k, run.pages.v, k2, v2)])
    for a, b in zip(*outs):
        assert np.array_equal(a, b)


def _pools(m, cached, seed):
    """Per-layer bf16 pools of streams in order, their first `cached` tokens drawn."""
    import torch
    T, H, d = SH.tokens_per_frame, SH.n_heads, SH.head_dim
    frames = [(c + LQ) // T for c in cached]
    table = np.zeros((len(cached), max(frames)), np.int32)
    at = 0
    for b, f in enumerate(frames):
        table[b, :f] = at + np.arange(f)
        at += f
    out = []
    for l in range(m.n_layers):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed + l)
        k = torch.randn((at, H, T, d), device="cuda", generator=g).bfloat16()
        v = torch.randn((at, H, d, T), device="cuda", generator=g).bfloat16()
        t = torch.from_numpy(table).to("cuda")
        out.append((k, v, t, m.A.kv_paged(k, v, t, at, max(frames))))
    return out


def _chunk_model(A, seed):
    m = Model(A, seed, 2, [20, 9])
    m.keep = []
    m.w8 = [int_weights(A, w, m.keep) for w in m.w_dev]
    return m


def test_a_chunk_equals_its_passes(A):
    import torch
    n_steps, ts, cached = [2, 1], [[1000.0, 500.0], [800.0]], [2 * LQ, LQ]
    m = _chunk_model(A, 93)
    pools = [_pools(m, cached, 50) for _ in range(2)]
    pos = [c // SH.tokens_per_frame for c in cached]
    batch = A.Batch([LQ] * 2, cached, pos, m.ctx_lens)
    ws, n = m.workspace(batch)
    x = normal_bf16(m.rng, (2 * LQ, SH.dim))
    noise = normal_bf16(m.rng, (1, 2 * LQ, SH.dim))
    x_dev, noise_dev = dev_bf16(x), dev_bf16(noise)
    x0 = torch.full((2 * LQ, SH.dim), float("nan"), dtype=torch.bfloat16, device="cuda")
    A.ardit_chunk_generate_int(None, m.dims, batch, n_steps, ts, x_dev, noise_dev, [p[3] for p in pools[0]], m.tw, m.ctx_k,
                               m.ctx_v, m.w, m.w8, x0, ws, n)
    _sync()

    def one_pass(xb, t, streams):
        sub = A.Batch([LQ] * streams, cached[:streams], pos[:streams], m.ctx_lens[:streams])
        mod = torch.empty((streams, 6, SH.dim), dtype=torch.float32, device="cuda")
        A.ardit_time_mod(None, m.dims, t, m.tw, mod, ws, n)
        xd = dev_bf16(bits_to_f32(xb[:streams * LQ]))
        v = torch.empty_like(xd)
        A.ardit_stack_fwd_int(None, m.dims, sub, xd, [p[3] for p in pools[1]], mod, m.ctx_k, m.ctx_v, m.w, m.w8, v, ws, n)
        _sync()
        return host_f32(v)

    cur = host_bits(x_dev).copy()
    xf = bits_to_f32(cur)
    v = one_pass(cur, [1000.0, 800.0], 2)
    cur[:LQ] = _sampler_bits(xf[:LQ], v[:LQ], 1.0, 0.5, noise[0, :LQ])
    cur[LQ:] = _sampler_bits(xf[LQ:], v[LQ:], 0.8, None, None)
    xf = bits_to_f32(cur)
    v = one_pass(cur, [500.0, 0.0], 2)              # the second stream commits
    cur[:LQ] = _sampler_bits(xf[:LQ], v[:LQ], 0.5, None, None)
    one_pass(cur, [0.0], 1)
    assert np.array_equal(host_bits(x0), cur)
    for a, b in zip(*pools):
        assert torch.equal(a[0].view(torch.int16), b[0].view(torch.int16))
        assert torch.equal(a[1].view(torch.int16), b[1].view(torch.int16))


def test_a_chunk_captured_and_replayed(A):
    import torch
    n_steps, ts, cached = [2, 1], [[1000.0, 500.0], [800.0]], [2 * LQ, LQ]
    m = _chunk_model(A, 94)
    pools = _pools(m, cached, 60)
    batch = A.Batch([LQ] * 2, cached, [c // SH.tokens_per_frame for c in cached], m.ctx_lens)
    ws, n = m.workspace(batch)
    x = dev_bf16(normal_bf16(m.rng, (2 * LQ, SH.dim)))
    noise = dev_bf16(normal_bf16(m.rng, (1, 2 * LQ, SH.dim)))
    x0 = torch.empty((2 * LQ, SH.dim), dtype=torch.bfloat16, device="cuda")

    def step():
        A.ardit_chunk_generate_int(None, m.dims, batch, n_steps, ts, x, noise, [p[3] for p in pools], m.tw, m.ctx_k, m.ctx_v,
                                   m.w, m.w8, x0, ws, n)

    def state():
        _sync()
        return [host_bits(x0).copy()] + [host_bits(t).copy() for p in pools for t in p[:2]]

    step()
    _sync()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        x.copy_(dev_bf16(normal_bf16(m.rng, (2 * LQ, SH.dim))))
        x0.fill_(float("nan"))
        g.replay()
        got = state()
        assert np.isfinite(host_f32(x0)).all()
        x0.fill_(float("nan"))
        step()
        for a, b in zip(got, state()):
            assert np.array_equal(a, b)
