"""Attention under a sliding window with sinks (first tokens that stay visible) against the fp64 oracle: heads of 128 and 64 on the MFMA kernels, others and fp32 on the
shape-agnostic ones; ragged chunks, padding, sinks that end inside a tile, across key blocks or reach into the window, rows that see nothing; layers,
adapters and the stack."""
import numpy as np
import pytest
import torch

from oracle import attn as o_attn
from oracle import layer as o_layer
from oracle import lora as o_lora
from paper_2506_03077_amd import binding as sb
from paper_2506_03077_amd import synth

from gpu_util import TOL, assert_close, code, dev, host, lib_layer_cfg, oracle_cfg

pytestmark = pytest.mark.gpu


def sinks_case(dtype, Hq, Hkv, dh, s, c, window, kv_first, sinks, seed=0):
    inp = synth.attn_inputs(Hq, Hkv, dh, s, c, dtype, seed)
    scale = 1.0 / np.sqrt(dh)
    o_ref, lse_ref = o_attn.chunk_forward(inp["q"], inp["k"], inp["v"], s, scale, window, kv_first, sinks)
    dq_ref, dk_ref, dv_ref = o_attn.chunk_backward(inp["q"], inp["k"], inp["v"], inp["d_o"], s, scale, window, kv_first, sinks)
    q, k, v, d_o = (dev(inp[n], dtype) for n in ("q", "k", "v", "d_o"))
    ac = sb.attn_cfg(code(dtype), Hq, Hkv, dh, s, c, scale, window, kv_first, sinks)
    o, lse = sb.streambp_attn_chunk_forward(ac, q, k, v)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    start = [torch.randn(k.shape, generator=gen, device="cuda") for _ in range(2)]      # dk and dv are added to
    dq, dk, dv = sb.streambp_attn_chunk_backward(ac, q, k, v, o, lse, d_o, dk=start[0].clone(), dv=start[1].clone())
    torch.cuda.synchronize()
    tol = TOL[dtype]
    empty = ~np.isfinite(lse_ref)
    lse_g = host(lse)
    assert np.array_equal(~np.isfinite(lse_g), empty) and np.all(lse_g[empty] == -np.inf)
    if empty.any():
        rows = torch.from_numpy(empty.T.copy()).cuda()
        assert torch.all(o[rows] == 0) and torch.all(dq[rows] == 0)
    assert_close(host(o), o_ref, tol, "o")
    # scores of up to |q| |k| / sqrt(dh) ~ 20: their fp32 sums of up to 128 products and the sum of the row, well within 1e-5 of values of order 1 to 10
    assert np.abs(np.where(empty, 0.0, lse_g - np.where(empty, 0.0, lse_ref))).max() < 1e-5
    assert_close(host(dq), dq_ref, tol, "dq")
    assert_close(host(dk - start[0])[:s + c], dk_ref, tol, "dk")
    assert_close(host(dv - start[1])[:s + c], dv_ref, tol, "dv")
    hidden = torch.from_numpy(~o_attn.visible(s + np.arange(c), np.arange(s + c), window, kv_first, sinks).any(axis=0)).cuda()
    assert torch.equal(dk[:s + c][hidden], start[0][:s + c][hidden]) and torch.equal(dv[:s + c][hidden], start[1][:s + c][hidden])
    return ac, q, k, v, d_o, o, lse, dq, (dk, dv), start


# start, queries, window, kv_first, sinks
MASKS = [
    (0, 200, 10, 0, 4),            # window shorter than a key tile, sinks inside its first one
    (300, 177, 100, 0, 1),         # one sink, ragged chunk
    (1000, 256, 300, 0, 130),      # sinks across two key blocks of dK/dV
    (1000, 300, 64, 120, 20),      # ... that begin behind padding, in the middle of a block
    (0, 300, 17, 130, 3),          # rows that see nothing, then rows that see sinks alone beside themselves
    (513, 255, 1, 0, 7),           # a window of the query itself
    (100, 64, 5000, 0, 50),        # window longer than the sequence: nothing stays behind
    (700, 1, 64, 0, 4),            # one query
    (0, 1, 1, 0, 1),               # one token
    (2000, 200, 64, 3, 300),       # more sinks than window
    (0, 500, 50, 0, 10000),        # every key a sink: plain causal
    (400, 70, 128, 460, 4),        # padding that ends inside the chunk
    (100, 50, 20, 400, 4),         # padding beyond all of it: every row empty
    (128, 130, 65, 64, 64),        # borders of tiles and blocks
    (5000, 333, 127, 1, 63),
]


@pytest.mark.parametrize("s,c,window,kv_first,sinks", MASKS)
def test_heads_of_128(s, c, window, kv_first, sinks):
    before = sb.streambp_generic_launches()
    sinks_case("bf16", 8, 2, 128, s, c, window, kv_first, sinks)
    assert sb.streambp_generic_launches() == before


@pytest.mark.parametrize("s,c,window,kv_first,sinks", MASKS)
def test_heads_of_64(s, c, window, kv_first, sinks):
    sinks_case("bf16", 6, 3, 64, s, c, window, kv_first, sinks)


@pytest.mark.parametrize("s,c,window,kv_first,sinks", MASKS)
@pytest.mark.parametrize("dtype,hq,hkv,dh", [("f32", 4, 2, 16), ("f32", 2, 2, 40), ("bf16", 3, 1, 96), ("f32", 2, 1, 200)])
def test_shape_agnostic_kernels(dtype, hq, hkv, dh, s, c, window, kv_first, sinks):
    sinks_case(dtype, hq, hkv, dh, s, c, window, kv_first, sinks)


# one K/V head and many, one query head and groups; launches of whole and of half tiles of queries, of one and of many rounds
@pytest.mark.parametrize("hq,hkv,dh,s,c,window,sinks", [(7, 1, 128, 900, 600, 200, 4), (4, 4, 128, 0, 1100, 128, 9), (28, 4, 128, 3000, 2048, 256, 4), (32, 8, 64, 0, 2500, 300, 16),
                                                        (28, 4, 128, 100, 4000, 100, 33), (16, 16, 64, 6000, 50, 1000, 2)])
def test_head_layouts_and_launch_sizes(hq, hkv, dh, s, c, window, sinks):
    sinks_case("bf16", hq, hkv, dh, s, c, window, 0, sinks)


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 32)])
def test_no_sinks_and_no_window_are_the_calls_without_them(dtype, dh):
    inp = synth.attn_inputs(4, 2, dh, 300, 200, dtype, 1)
    q, k, v, d_o = (dev(inp[n], dtype) for n in ("q", "k", "v", "d_o"))

    def run(**kw):
        ac = sb.attn_cfg(code(dtype), 4, 2, dh, 300, 200, 0.1, **kw)
        o, lse = sb.streambp_attn_chunk_forward(ac, q, k, v)
        return (o, lse) + sb.streambp_attn_chunk_backward(ac, q, k, v, o, lse, d_o)
    for a, b in ((dict(window=64), dict(window=64, sinks=0)), (dict(), dict(sinks=9)), (dict(kv_first=400, window=30), dict(kv_first=400, window=30, sinks=0))):
        assert all(torch.equal(x, y) for x, y in zip(run(**a), run(**b)))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 16), ("bf16", 80)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_was_evicted_between_sinks_and_window_may_hold_anything(dtype, dh, bad):
    s, c, window, kv_first, sinks = 1500, 100, 200, 37, 30
    ac, q, k, v, d_o, o, lse, dq, grads, start = sinks_case(dtype, 4, 2, dh, s, c, window, kv_first, sinks, seed=3)
    hidden = torch.from_numpy(~o_attn.visible(s + np.arange(c), np.arange(s + c), window, kv_first, sinks).any(axis=0)).cuda()
    k2, v2 = k.clone(), v.clone()
    k2[hidden], v2[hidden] = bad, bad
    o2, lse2 = sb.streambp_attn_chunk_forward(ac, q, k2, v2)
    dq2, dk2, dv2 = sb.streambp_attn_chunk_backward(ac, q, k2, v2, o2, lse2, d_o, dk=start[0].clone(), dv=start[1].clone())
    torch.cuda.synchronize()
    if dtype == "bf16" and dh in (64, 128):
        assert torch.equal(o2, o) and torch.equal(lse2, lse) and torch.equal(dq2, dq)
        assert torch.equal(dk2, grads[0]) and torch.equal(dv2, grads[1])
        return
    # the shape-agnostic kernels sum a block that holds such rows pair by pair, in another order: the gates of the comparison with fp64, and hidden rows as they were
    for x, y, n in ((o2, o, "o"), (dq2, dq, "dq"), (dk2 - start[0], grads[0] - start[0], "dk"), (dv2 - start[1], grads[1] - start[1], "dv")):
        assert_close(host(x), host(y), TOL[dtype], n)
    assert torch.equal(lse2, lse) and torch.equal(dk2[hidden], start[0][hidden]) and torch.equal(dv2[hidden], start[1][hidden])


@pytest.mark.parametrize("hq,hkv,dh,s,c,window,kv_first,sinks", [(8, 2, 128, 1000, 700, 100, 0, 5), (8, 2, 64, 300, 333, 64, 20, 200), (28, 4, 128, 0, 1024, 128, 0, 4)])
def test_the_workspace_changes_no_bit(hq, hkv, dh, s, c, window, kv_first, sinks):
    """Parts in the workspace, walked in turn without the room for them, and the entry point without a workspace."""
    inp = synth.attn_inputs(hq, hkv, dh, s, c, "bf16", 2)
    q, k, v, d_o = (dev(inp[n], "bf16") for n in ("q", "k", "v", "d_o"))
    ac = sb.attn_cfg(sb.SBP_BF16, hq, hkv, dh, s, c, dh ** -0.5, window, kv_first, sinks)
    need, least = sb.streambp_attn_workspace_bytes(ac), -(-2 * c * hq * 4 // 256) * 256
    assert need > least
    o, lse = sb.streambp_attn_chunk_forward(ac, q, k, v)
    start = [torch.randn(k.shape, device="cuda") for _ in range(2)]
    got = []
    for room in (need, need - 1, least):
        ws = torch.full((room,), 0xFF, dtype=torch.uint8, device="cuda")
        got.append(sb.streambp_attn_chunk_backward(ac, q, k, v, o, lse, d_o, dk=start[0].clone(), dv=start[1].clone(), workspace=ws))
    got.append(sb.streambp_attn_chunk_backward_noalloc(ac, q, k, v, o, lse, d_o, torch.empty_like(q), start[0].clone(), start[1].clone()))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


def test_chunks_of_a_sequence_add_up():
    """Gradients of one call over a sequence and of its chunks, the last first, as the layer walks them."""
    hq, hkv, dh, T, window, sinks = 4, 2, 128, 900, 150, 6
    inp = synth.attn_inputs(hq, hkv, dh, 0, T, "bf16", 4)
    q, k, v, d_o = (dev(inp[n], "bf16") for n in ("q", "k", "v", "d_o"))
    _, dk_ref, dv_ref = o_attn.chunk_backward(inp["q"], inp["k"], inp["v"], inp["d_o"], 0, dh ** -0.5, window, 0, sinks)
    dk, dv = torch.zeros(k.shape, device="cuda"), torch.zeros(k.shape, device="cuda")
    for a, b in ((640, 900), (256, 640), (0, 256)):
        ac = sb.attn_cfg(sb.SBP_BF16, hq, hkv, dh, a, b - a, dh ** -0.5, window, 0, sinks)
        qc, dc = q[a:b].contiguous(), d_o[a:b].contiguous()
        o, lse = sb.streambp_attn_chunk_forward(ac, qc, k[:b].contiguous(), v[:b].contiguous())
        sb.streambp_attn_chunk_backward(ac, qc, k[:b].contiguous(), v[:b].contiguous(), o, lse, dc, dk=dk, dv=dv)
    assert_close(host(dk), dk_ref, 2e-2, "dk")
    assert_close(host(dv), dv_ref, 2e-2, "dv")


def test_tensors_without_16_byte_alignment():
    hq, hkv, dh, s, c = 4, 2, 128, 300, 100
    inp = synth.attn_inputs(hq, hkv, dh, s, c, "bf16", 6)
    want = None
    for off in (0, 1):
        t = {}
        for n in ("q", "k", "v", "d_o"):
            x = dev(inp[n], "bf16")
            t[n] = torch.empty(x.numel() + off, dtype=x.dtype, device="cuda")[off:].view(x.shape).copy_(x)
        ac = sb.attn_cfg(sb.SBP_BF16, hq, hkv, dh, s, c, dh ** -0.5, 50, 0, 5)
        o, lse = sb.streambp_attn_chunk_forward(ac, t["q"], t["k"], t["v"])
        got = (o, lse) + sb.streambp_attn_chunk_backward(ac, t["q"], t["k"], t["v"], o, lse, t["d_o"])
        if want is None:
            want = [host(x) for x in got]
        else:
            for x, y in zip(got, want):
                assert_close(host(x), y, 2e-2, "unaligned")


def test_captured_and_replayed():
    hq, hkv, dh, s, c = 8, 2, 128, 1000, 500
    inp = synth.attn_inputs(hq, hkv, dh, s, c, "bf16", 7)
    q, k, v, d_o = (dev(inp[n], "bf16") for n in ("q", "k", "v", "d_o"))
    ac = sb.attn_cfg(sb.SBP_BF16, hq, hkv, dh, s, c, dh ** -0.5, 128, 0, 4)
    o, lse, dq = torch.empty_like(q), torch.empty((hq, c), device="cuda"), torch.empty_like(q)
    dk, dv = torch.zeros(k.shape, device="cuda"), torch.zeros(k.shape, device="cuda")
    ws = torch.empty(sb.streambp_attn_workspace_bytes(ac), dtype=torch.uint8, device="cuda")

    def step():
        dk.zero_()
        dv.zero_()
        sb.streambp_attn_chunk_forward(ac, q, k, v, o, lse)
        sb.streambp_attn_chunk_backward(ac, q, k, v, o, lse, d_o, dq, dk, dv, ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    for seed in range(3):
        fresh = synth.attn_inputs(hq, hkv, dh, s, c, "bf16", 20 + seed)
        for x, n in ((q, "q"), (k, "k"), (v, "v"), (d_o, "d_o")):
            x.copy_(dev(fresh[n], "bf16"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (o, lse, dq, dk, dv)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (o, lse, dq, dk, dv)))


def test_log_sum_exps_that_differ_by_much():
    """Sinks whose scores are far above and far below the window's."""
    hq, hkv, dh, s, c, window, sinks = 4, 2, 128, 600, 200, 100, 4
    for size in (6.0, 0.0):
        inp = synth.attn_inputs(hq, hkv, dh, s, c, "bf16", 8)
        inp["k"][:sinks] = synth.to_storage(inp["k"][:sinks] * size, "bf16")
        o_ref, lse_ref = o_attn.chunk_forward(inp["q"], inp["k"], inp["v"], s, dh ** -0.5, window, 0, sinks)
        refs = o_attn.chunk_backward(inp["q"], inp["k"], inp["v"], inp["d_o"], s, dh ** -0.5, window, 0, sinks)
        q, k, v, d_o = (dev(inp[n], "bf16") for n in ("q", "k", "v", "d_o"))
        ac = sb.attn_cfg(sb.SBP_BF16, hq, hkv, dh, s, c, dh ** -0.5, window, 0, sinks)
        o, lse = sb.streambp_attn_chunk_forward(ac, q, k, v)
        got = sb.streambp_attn_chunk_backward(ac, q, k, v, o, lse, d_o)
        assert_close(host(o), o_ref, 2e-2, "o")
        assert np.abs(host(lse) - lse_ref).max() < 2e-5
        for x, y, n in zip(got, refs, ("dq", "dk", "dv")):
            assert_close(host(x), y, 2e-2, n)


MID = dict(dtype="bf16", hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=128, mlp_width=512)
MID64 = dict(dtype="bf16", hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=64, mlp_width=512)
TINY = synth.CONFIGS["tiny"]


def layer_case(cfg, T, chunk, window, sinks, first):
    cfg = dict(cfg, window=window)
    B = len(first) if first else 1
    inp = synth.layer_inputs(cfg, seed=7, seq_len=T, batch=B)
    oc = dict(oracle_cfg(cfg), sinks=sinks)
    lc = lib_layer_cfg(cfg, T, chunk, B, seq_first=first)
    lc.sinks = sinks
    return cfg, B, inp, oc, lc


@pytest.mark.parametrize("cfg,T,chunk,window,sinks,first", [
    (MID, 640, 256, 100, 4, None), (MID, 333, 100, 20, 9, [50, 0]), (MID, 500, 128, 200, 140, [130, 7]), (MID64, 400, 128, 30, 5, [0, 60]),
    (TINY, 96, 40, 16, 3, [10, 0, 41]), (TINY, 256, 64, 20, 2, [100]), (MID, 260, 64, 30, 3, [260, 100]),
])
def test_layer(cfg, T, chunk, window, sinks, first):
    """Backward and forward of a layer, sequences of a batch with padding of their own - one of them nothing but padding -, several passes."""
    cfg, B, inp, oc, lc = layer_case(cfg, T, chunk, window, sinks, first)
    _, dx_ref, g_ref = o_layer.layer_forward_backward(inp["x"], inp["w"], oc, inp["dy"], first)
    dt = cfg["dtype"]
    w = {k: dev(v, dt) for k, v in inp["w"].items()}
    dx, dw = sb.streambp_layer_backward(lc, w, dev(inp["x"], dt), dev(inp["dy"], dt))
    torch.cuda.synchronize()
    assert_close(host(dx), dx_ref, TOL[dt], "dx")
    for n in sb.WEIGHT_NAMES:
        assert_close(host(dw[n]), g_ref[n], TOL[dt], f"d{n}")
    y_ref = np.stack([o_layer.layer_forward(inp["x"][b], inp["w"], dict(oc, first_valid=(first[b] if first else 0)))[0] for b in range(B)])
    assert_close(host(sb.streambp_layer_forward(lc, w, dev(inp["x"], dt))), y_ref, TOL[dt] if dt == "f32" else 1e-2, "y")


def test_layer_of_many_passes_at_7b_widths():
    """More rows than a pass takes: sinks that lie in another pass's keys, and in the first pass's own."""
    cfg, B, inp, oc, lc = layer_case(synth.CONFIGS["7b"], 4608, 2048, 512, 8, [300])
    _, dx_ref, g_ref = o_layer.layer_forward_backward(inp["x"], inp["w"], oc, inp["dy"], [300])
    w = {k: dev(v, "bf16") for k, v in inp["w"].items()}
    dx, dw = sb.streambp_layer_backward(lc, w, dev(inp["x"], "bf16"), dev(inp["dy"], "bf16"))
    torch.cuda.synchronize()
    assert_close(host(dx), dx_ref, 2e-2, "dx")
    for n in sb.WEIGHT_NAMES:
        assert_close(host(dw[n]), g_ref[n], 2e-2, f"d{n}")


def test_adapters():
    from test_gpu_lora import make_adapters
    cfg, B, inp, oc, lc = layer_case(MID, 300, 128, 40, 5, None)
    ad = make_adapters(cfg, inp["w"], 8, ("wq", "wv"), 0, 0.05)
    _, dx_ref, dA_ref, dB_ref = o_lora.layer_forward_backward(inp["x"], inp["w"], ad, 2.0, oc, inp["dy"], None)
    w = {k: dev(v, "bf16") for k, v in inp["w"].items()}
    dx, da, db = sb.streambp_layer_lora_backward(lc, w, {n: (dev(A, "bf16"), dev(B, "bf16")) for n, (A, B) in ad.items()}, 8, 2.0, dev(inp["x"], "bf16"), dev(inp["dy"], "bf16"))
    torch.cuda.synchronize()
    assert_close(host(dx), dx_ref, 2e-2, "dx")
    for n in ad:
        assert_close(host(da[n]), dA_ref[n], 2e-2, f"dA[{n}]")
        assert_close(host(db[n]), dB_ref[n], 2e-2, f"dB[{n}]")
