"""Pins of the oracle's sinks (the first positions that stay visible behind a sliding window), and what the library's attention, layer and stack calls
refuse of them (CPU only)."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import attn, layer
from paper_2506_03077_amd import binding as sb

from test_oracle_layer import make as make_layer
from test_oracle_masks import make

RULES = [(3, 0, 2), (4, 7, 1), (1, 0, 1), (2, 9, 3), (100, 0, 5), (3, 2, 50), (1, 3, 4)]


@pytest.mark.parametrize("window,kv_first,sinks", RULES)
def test_forward_matches_scalar_loops(window, kv_first, sinks):
    c, s, scale = 5, 6, 0.5
    q, k, v, _ = make(c, s)
    o, lse = attn.chunk_forward(q, k, v, s, scale, window, kv_first, sinks)
    for t in range(c):
        pos = s + t
        keys = [u for u in range(pos + 1) if u >= kv_first and (u > pos - window or u < kv_first + sinks)]
        for h in range(4):
            if not keys:
                assert np.all(o[t, h] == 0) and lse[h, t] == -np.inf
                continue
            sc = [scale * sum(q[t, h, j] * k[u, h // 2, j] for j in range(4)) for u in keys]
            den = sum(math.exp(x) for x in sc)
            assert abs(lse[h, t] - math.log(den)) < 1e-12
            for j in range(4):
                assert abs(o[t, h, j] - sum(math.exp(x) / den * v[u, h // 2, j] for x, u in zip(sc, keys))) < 1e-12


@pytest.mark.parametrize("window,kv_first,sinks", RULES)
def test_backward_finite_differences(window, kv_first, sinks):
    c, s, scale, step = 5, 6, 0.5, 1e-6
    q, k, v, d_o = make(c, s, seed=1)
    grads = attn.chunk_backward(q, k, v, d_o, s, scale, window, kv_first, sinks)
    f = lambda q, k, v: float(np.sum(attn.chunk_forward(q, k, v, s, scale, window, kv_first, sinks)[0] * d_o))
    rng = np.random.default_rng(2)
    for i, g in enumerate(grads):
        for _ in range(30):
            at = tuple(rng.integers(0, n) for n in g.shape)
            up, down = [x.copy() for x in (q, k, v)], [x.copy() for x in (q, k, v)]
            up[i][at] += step
            down[i][at] -= step
            assert abs((f(*up) - f(*down)) / (2 * step) - g[at]) < 1e-7


def test_limits():
    q, k, v, d_o = make()
    plain = attn.chunk_forward(q, k, v, 6, 0.5)
    assert all(np.array_equal(a, b) for a, b in zip(plain, attn.chunk_forward(q, k, v, 6, 0.5, 2, 0, 100)))      # every key a sink
    assert all(np.array_equal(a, b) for a, b in zip(plain, attn.chunk_forward(q, k, v, 6, 0.5, 0, 0, 3)))        # no window: nothing to stay behind
    window = attn.chunk_forward(q, k, v, 6, 0.5, 3, 2)
    assert all(np.array_equal(a, b) for a, b in zip(window, attn.chunk_forward(q, k, v, 6, 0.5, 3, 2, 0)))


def test_layer_with_sinks_is_the_chunk_attention_of_its_rows():
    """The layer's mask against attention's, by the layer's own o."""
    cfg, W, x, dy = make_layer()
    T, Hq, Hkv = x.shape[0], cfg["n_q_heads"], cfg["n_kv_heads"]
    dh = cfg["head_dim"]
    cfg = dict(cfg, window=3, sinks=2, first_valid=1)
    a, _ = layer.rmsnorm_forward(x, W["g1"], cfg.get("rms_eps", 1e-6))
    cos, sin = layer.rope_tables(T, dh, cfg.get("rope_theta", 1e4), cfg.get("pos_offset", 0))
    q = layer.rope_apply((a @ W["wq"].T).reshape(T, Hq, dh), cos, sin)
    k = layer.rope_apply((a @ W["wk"].T).reshape(T, Hkv, dh), cos, sin)
    v = (a @ W["wv"].T).reshape(T, Hkv, dh)
    o, _ = attn.chunk_forward(q, k, v, 0, 1 / np.sqrt(dh), 3, 1, 2)
    other = dict(W, wdown=np.zeros_like(W["wdown"]), wo=np.eye(W["wo"].shape[0], Hq * dh))      # y = x + o, as far as the widths go
    y, _ = layer.layer_forward(x, other, cfg)
    n = min(W["wo"].shape)
    assert np.abs((y - x)[:, :n] - o.reshape(T, -1)[:, :n]).max() < 1e-12


def test_negative_sinks_are_refused():
    ac = sb.attn_cfg(sb.SBP_BF16, 8, 2, 128, 100, 10, 0.1, window=5, sinks=-1)
    assert sb.streambp_attn_workspace_bytes(ac) == 0 and "sinks" in sb.streambp_last_error()
    lc = sb.layer_cfg(sb.SBP_F32, 1, 16, 8, 32, 2, 2, 16, 64, window=4, sinks=-3)
    assert sb.streambp_layer_workspace_bytes(lc) == 0 and "sinks" in sb.streambp_last_error()
    sc = sb.stack_cfg(lc, 2, 100, 8)
    assert sb.streambp_stack_workspace_bytes(sc) == 0


def test_the_layer_struct_keeps_its_size():
    """`sinks` lies in what was padding before seq_first."""
    assert sb.LayerCfg.seq_first.offset == 64 and sb.LayerCfg.sinks.offset == 60 and sb.LayerCfg.window.offset == 56
    assert C.sizeof(sb.LayerCfg) == 72


def test_sinks_cost_a_layer_no_workspace():
    lc = lambda sinks: sb.layer_cfg(sb.SBP_BF16, 1, 8192, 1024, 1024, 16, 4, 64, 2816, window=512, sinks=sinks)
    assert sb.streambp_layer_workspace_bytes(lc(16)) == sb.streambp_layer_workspace_bytes(lc(0)) > 0


def test_attention_workspace_covers_the_parts_of_the_sinks():
    """28 / 4 heads, 4096 queries from 4096 on, window 1024: slices [2][sink][head][128] fp32 of the sinks, as many as give every CU a workgroup."""
    need = lambda **kw: sb.streambp_attn_workspace_bytes(sb.attn_cfg(sb.SBP_BF16, 28, 4, 128, 4096, 4096, 0.1, window=1024, **kw))
    stats = 2 * 4096 * 28 * 4
    assert need() >= stats and need(sinks=4) >= stats + 2 * 2 * 4 * 4 * 128 * 4
    assert sb.streambp_attn_workspace_bytes(sb.attn_cfg(sb.SBP_BF16, 28, 4, 128, 0, 500, 0.1, window=1024, sinks=2 ** 31 - 1)) > 0
