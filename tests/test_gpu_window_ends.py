"""Sliding windows up to the end of the type: longer than the sequence, they are a window of all its keys."""
import pytest
import torch

from oracle import attn as o_attn
from oracle import layer as o_layer
from paper_2506_03077_amd import binding as sb
from paper_2506_03077_amd import synth

from gpu_util import TOL, assert_close, code, dev, host, lib_layer_cfg, oracle_cfg

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,hq,hkv,dh,s,c", [("bf16", 4, 2, 128, 300, 200), ("bf16", 4, 2, 64, 0, 333), ("f32", 4, 2, 32, 300, 200), ("bf16", 4, 1, 80, 100, 70)])
def test_attention(dtype, hq, hkv, dh, s, c):
    inp = synth.attn_inputs(hq, hkv, dh, s, c, dtype, 1)
    q, k, v, d_o = (dev(inp[n], dtype) for n in ("q", "k", "v", "d_o"))
    got = []
    for window in (s + c, s + c + 1, 2 ** 31 - 1):
        ac = sb.attn_cfg(code(dtype), hq, hkv, dh, s, c, 0.1, window)
        o, lse = sb.streambp_attn_chunk_forward(ac, q, k, v)
        got.append((o, lse) + tuple(sb.streambp_attn_chunk_backward(ac, q, k, v, o, lse, d_o)))
        assert sb.streambp_attn_workspace_bytes(ac) == sb.streambp_attn_workspace_bytes(sb.attn_cfg(code(dtype), hq, hkv, dh, s, c, 0.1, s + c))
    for x in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(x, got[0]))
    want = o_attn.chunk_backward(inp["q"], inp["k"], inp["v"], inp["d_o"], s, 0.1)
    for a, b, n in zip(got[-1][2:], want, ("dq", "dk", "dv")):
        assert_close(host(a), b, TOL[dtype], n)


@pytest.mark.parametrize("name", ["tiny", "mid"])
def test_layer(name):
    cfg = dict(synth.CONFIGS["tiny"]) if name == "tiny" else dict(dtype="bf16", hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=128, mlp_width=512)
    cfg["window"] = 2 ** 31 - 1
    inp = synth.layer_inputs(cfg, seed=7, seq_len=300, batch=1)
    _, dx_ref, g_ref = o_layer.layer_forward_backward(inp["x"], inp["w"], oracle_cfg(cfg), inp["dy"])
    dt = cfg["dtype"]
    dx, dw = sb.streambp_layer_backward(lib_layer_cfg(cfg, 300, 128), {k: dev(v, dt) for k, v in inp["w"].items()}, dev(inp["x"], dt), dev(inp["dy"], dt))
    assert_close(host(dx), dx_ref, TOL[dt], "dx")
    for n in sb.WEIGHT_NAMES:
        assert_close(host(dw[n]), g_ref[n], TOL[dt], f"d{n}")
