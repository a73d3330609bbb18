"""Calls with sinks that the sizes allow and programs make: windows and sinks up to the types' ends, single tokens one after the other as serving makes them, two streams at
once, outputs with something beside them."""
import numpy as np
import pytest
import torch

from oracle import attn as o_attn
from paper_2506_03077_amd import binding as sb
from paper_2506_03077_amd import synth

from gpu_util import TOL, assert_close, code, dev, host, tdtype

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


def run(ac, q, k, v, d_o, **kw):
    o, lse = sb.streambp_attn_chunk_forward(ac, q, k, v)
    return (o, lse) + tuple(sb.streambp_attn_chunk_backward(ac, q, k, v, o, lse, d_o, **kw))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 32)])
@pytest.mark.parametrize("window,sinks,same", [(MOST, MOST, dict(window=500, sinks=500)), (MOST, 4, dict(window=500, sinks=4)), (500, 4, dict(window=501, sinks=4)), (499, MOST, dict(window=499, sinks=500)),
                                               (60, MOST, dict(window=60, sinks=500))])
def test_windows_and_sinks_up_to_the_end_of_the_type(dtype, dh, window, sinks, same):
    """500 keys: a window of 500 loses none of them, one of 499 the first, to the last query."""
    inp = synth.attn_inputs(4, 2, dh, 300, 200, dtype, 1)
    q, k, v, d_o = (dev(inp[n], dtype) for n in ("q", "k", "v", "d_o"))
    got = run(sb.attn_cfg(code(dtype), 4, 2, dh, 300, 200, 0.1, window=window, sinks=sinks), q, k, v, d_o)
    want = run(sb.attn_cfg(code(dtype), 4, 2, dh, 300, 200, 0.1, **same), q, k, v, d_o)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dq, dk, dv = o_attn.chunk_backward(inp["q"], inp["k"], inp["v"], inp["d_o"], 300, 0.1, window, 0, sinks)
    for a, b, n in zip(got[2:], (dq, dk, dv), ("dq", "dk", "dv")):
        assert_close(host(a), b, TOL[dtype], n)


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("bf16", 4, 4, 64), ("f32", 4, 2, 16)])
def test_tokens_one_after_the_other(dtype, hq, hkv, dh):
    """A prompt, then single tokens behind a prefix that grows past the window; the rows between sinks and window hold NaN by then, as a ring that was overwritten might."""
    T, prompt, window, sinks = 420, 150, 130, 3
    inp = synth.attn_inputs(hq, hkv, dh, 0, T, dtype, 3)
    scale = dh ** -0.5
    want, want_lse = o_attn.chunk_forward(inp["q"], inp["k"], inp["v"], 0, scale, window, 0, sinks)
    q, k, v = (dev(inp[n], dtype) for n in ("q", "k", "v"))
    o, lse = torch.empty_like(q), torch.empty((T, hq), device="cuda")
    a, b = 0, prompt
    while a < T:
        ac = sb.attn_cfg(code(dtype), hq, hkv, dh, a, b - a, scale, window, 0, sinks)
        part, stats = sb.streambp_attn_chunk_forward(ac, q[a:b], k[:b], v[:b])
        o[a:b], lse[a:b] = part, stats.t()
        if b - window > sinks:
            k[sinks:b - window + 1] = float("nan")
            v[sinks:b - window + 1] = float("nan")
        a, b = b, b + 1
    assert_close(host(o), want, TOL[dtype], "o")
    assert np.abs(host(lse) - want_lse.T).max() < 1e-5


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 2, 128), ("bf16", 8, 2, 64), ("f32", 4, 2, 24)])
def test_nothing_beside_the_outputs_is_written(dtype, hq, hkv, dh):
    s, c, window, sinks = 700, 77, 90, 150
    inp = synth.attn_inputs(hq, hkv, dh, s, c, dtype, 5)
    q, k, v, d_o = (dev(inp[n], dtype) for n in ("q", "k", "v", "d_o"))
    held = []

    def guarded(shape, dt):
        size = int(np.prod(shape)) * torch.empty((), dtype=dt).element_size()
        raw = torch.full((size + 8192,), 0x5A, dtype=torch.uint8, device="cuda")
        held.append((raw, size))
        view = raw[4096:4096 + size].view(dt).view(shape)
        return view.zero_()
    ac = sb.attn_cfg(code(dtype), hq, hkv, dh, s, c, dh ** -0.5, window, 0, sinks)
    o, lse = guarded(q.shape, tdtype(dtype)), guarded((hq, c), torch.float32)
    dq, dk, dv = guarded(q.shape, tdtype(dtype)), guarded((s + c, hkv, dh), torch.float32), guarded((s + c, hkv, dh), torch.float32)
    for room in (sb.streambp_attn_workspace_bytes(ac), -(-2 * c * hq * 4 // 256) * 256):
        sb.streambp_attn_chunk_forward(ac, q, k, v, o, lse)
        sb.streambp_attn_chunk_backward(ac, q, k, v, o, lse, d_o, dq, dk, dv, guarded((room,), torch.uint8))
    torch.cuda.synchronize()
    for raw, size in held:
        assert bool((raw[:4096] == 0x5A).all()) and bool((raw[4096 + size:] == 0x5A).all())
    want = o_attn.chunk_backward(inp["q"], inp["k"], inp["v"], inp["d_o"], s, dh ** -0.5, window, 0, sinks)
    for a, b, n in zip((dq, dk / 2, dv / 2), want, ("dq", "dk", "dv")):
        assert_close(host(a), b, TOL[dtype], n)


def test_two_streams_at_once():
    """Calls with workspaces and outputs of their own, under way together."""
    cases = []
    for seed, (hq, hkv, dh, s, c, window, sinks) in enumerate([(28, 4, 128, 2000, 1000, 256, 4), (16, 4, 64, 1000, 900, 200, 16)]):
        inp = synth.attn_inputs(hq, hkv, dh, s, c, "bf16", 30 + seed)
        t = [dev(inp[n], "bf16") for n in ("q", "k", "v", "d_o")]
        ac = sb.attn_cfg(sb.SBP_BF16, hq, hkv, dh, s, c, dh ** -0.5, window, 0, sinks)
        cases.append((ac, t, run(ac, *t)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        got = []
        for stream, (ac, t, _) in zip(streams, cases):
            with torch.cuda.stream(stream):
                got.append(run(ac, *t))
        torch.cuda.synchronize()
        for x, (_, _, want) in zip(got, cases):
            assert all(torch.equal(a, b) for a, b in zip(x, want))


@pytest.mark.parametrize("dtype,dh", [("bf16", 128), ("bf16", 64), ("f32", 16)])
@pytest.mark.parametrize("s,c,kv_first", [(0, 2, 2), (0, 1, 5), (200, 77, 277), (200, 77, 1000), (200, 77, MOST), (100, 300, 400)])
def test_padding_all_the_way(dtype, dh, s, c, kv_first):
    """No query sees anything: the outputs say so, and dk and dv keep their bits, whatever K and V hold."""
    inp = synth.attn_inputs(4, 2, dh, s, c, dtype, 9)
    q, d_o = dev(inp["q"], dtype), dev(inp["d_o"], dtype)
    k = torch.full((s + c, 2, dh), float("nan") if dtype == "bf16" else 1.0, dtype=tdtype(dtype), device="cuda")
    ac = sb.attn_cfg(code(dtype), 4, 2, dh, s, c, 0.1, window=64, kv_first=kv_first, sinks=3)
    o, lse = sb.streambp_attn_chunk_forward(ac, q, k, k)
    start = [torch.randn((s + c, 2, dh), device="cuda") for _ in range(2)]
    dq, dk, dv = sb.streambp_attn_chunk_backward(ac, q, k, k, o, lse, d_o, dk=start[0].clone(), dv=start[1].clone())
    assert not bool(o.any()) and bool((lse == -float("inf")).all()) and not bool(dq.any())
    assert torch.equal(dk, start[0]) and torch.equal(dv, start[1])


@pytest.mark.parametrize("dtype,hq,hkv,dh", [("bf16", 8, 4, 128), ("bf16", 8, 8, 64), ("f32", 4, 4, 64)])
def test_a_cache_of_more_than_4_GiB(dtype, hq, hkv, dh):
    """Sinks at its beginning, a window at its end, nothing between them is looked at (bf16: NaN)."""
    if torch.cuda.mem_get_info()[0] < 64e9:
        pytest.skip("27 GB")
    s, c, window, sinks = 4_400_000, 333, 200, 5
    n, lo = s + c, s - window - 50
    gap = lo - sinks                                  # rows that the oracle is spared: its row u + sinks is row lo + u
    inp = synth.attn_inputs(hq, hkv, dh, s - gap, c, dtype, 11)
    k, v = (torch.full((n, hkv, dh), float("nan") if dtype == "bf16" else 1.0, dtype=tdtype(dtype), device="cuda") for _ in range(2))
    assert k.numel() * k.element_size() > 2 ** 32
    for x, name in ((k, "k"), (v, "v")):
        x[:sinks], x[lo:] = dev(inp[name][:sinks], dtype), dev(inp[name][sinks:], dtype)
    q, d_o = dev(inp["q"], dtype), dev(inp["d_o"], dtype)
    ac = sb.attn_cfg(code(dtype), hq, hkv, dh, s, c, dh ** -0.5, window, 0, sinks)
    o, lse, dq, dk, dv = run(ac, q, k, v, d_o)
    torch.cuda.synchronize()
    assert not any(bool(x[sinks:lo].any()) for x in (dk, dv))
    o_ref, lse_ref = o_attn.chunk_forward(inp["q"], inp["k"], inp["v"], s - gap, dh ** -0.5, window, 0, sinks)
    refs = o_attn.chunk_backward(inp["q"], inp["k"], inp["v"], inp["d_o"], s - gap, dh ** -0.5, window, 0, sinks)
    assert_close(host(o), o_ref, TOL[dtype], "o")
    assert np.abs(host(lse) - lse_ref).max() < 1e-5
    assert_close(host(dq), refs[0], TOL[dtype], "dq")
    for x, ref, name in ((dk, refs[1], "dk"), (dv, refs[2], "dv")):
        assert_close(np.concatenate([host(x[:sinks]), host(x[lo:])]), ref, TOL[dtype], name)
