"""A training run of the stack under a sliding window with sinks: forward, backward, the norm of all gradients, AdamW with the factor that limits it, and the
next step with the weights and states that it left - all on a stream of its own.  Each part of a step is held against the fp64 oracle at what it was
given: the gradients at the weights of that step, the norm at the gradients, the new weights and states at both; so a bound covers one step's roundings."""
import numpy as np
import pytest
import torch

from oracle import head as o_head
from oracle import layer as o_layer
from oracle import optim
from paper_2506_03077_amd import binding as sb
from paper_2506_03077_amd import synth

from gpu_util import TOL, assert_close, code, dev, host, oracle_cfg, tdtype
from test_gpu_adamw import HYPER, before, check

pytestmark = pytest.mark.gpu

WINDOW, SINKS, SEED = 48, 3, 7


def oracle_gradients(ids, emb, layers, g_final, w_head, targets, cfg, loss_scale):
    x = host(emb)[ids]
    ocfg = dict(oracle_cfg(cfg), window=WINDOW, sinks=SINKS)
    caches = []
    for w in layers:
        x, cache = o_layer.layer_forward(x, {n: host(v) for n, v in w.items()}, ocfg)
        caches.append(cache)
    h, r = o_layer.rmsnorm_forward(x, host(g_final), 1e-6)
    hd = o_head.sft(h[None], host(w_head), targets[None], loss_scale)
    dy, dg_final = o_layer.rmsnorm_backward(hd["dh"][0], x, host(g_final), r)
    grads = []
    for cache in reversed(caches):
        dy, g = o_layer.layer_backward(cache, dy)
        grads = [g[n] for n in sb.WEIGHT_NAMES] + grads
    demb = np.zeros(emb.shape)
    np.add.at(demb, ids, dy)
    return hd["loss"], grads + [dg_final, hd["dw"], demb]


@pytest.mark.parametrize("name,grad_dtype,state,master", [("tiny", "f32", "f32", False), ("tiny", "f32", "8bit", False), ("mid", "f32", "f32", True), ("mid", "bf16", "8bit", False)])
def test_steps(name, grad_dtype, state, master):
    cfg = dict(synth.CONFIGS["tiny"]) if name == "tiny" else dict(dtype="bf16", hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=128, mlp_width=512)
    cfg["vocab"] = 150
    dt, L, T, d, eight = cfg["dtype"], 2, 300, cfg["hidden"], state == "8bit"
    ids = np.arange(T, dtype=np.int32) * 7 % 150                 # every row of the embedding has a gradient
    targets = np.random.default_rng(2).integers(0, 150, T).astype(np.int32)
    layers = [{n: dev(v, dt) for n, v in synth.layer_weights(cfg, seed=10 + l).items()} for l in range(L)]
    w_head = dev(synth.head_inputs(cfg, seed=3, seq_len=1, vocab=150)["w"], dt)
    rng = np.random.default_rng(5)
    g_final, emb = dev(1 + rng.normal(0, 0.02, d), dt), dev(rng.normal(0, 1, (150, d)), dt)
    lc = sb.layer_cfg(code(dt), 1, T, 96, d, cfg["n_q_heads"], cfg["n_kv_heads"], cfg["head_dim"], cfg["mlp_width"], grad_dtype=code(grad_dtype), window=WINDOW, sinks=SINKS)
    sc = sb.stack_cfg(lc, L, 150, 100, sb.SBP_OBJ_SFT, 1.0 / T)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        ckpt = [torch.empty((1, T, d), dtype=tdtype(dt), device="cuda") for _ in range(L + 1)]
        dev_ids, dev_targets = torch.from_numpy(ids).cuda(), torch.from_numpy(targets).cuda()
        grads = dict(dlayers=[sb.new_layer_grads(w, code(grad_dtype)) for w in layers], dg_final=torch.zeros(d, device="cuda"),
                     dw_head=torch.zeros((150, d), dtype=tdtype(grad_dtype), device="cuda"), demb=torch.zeros((150, d), device="cuda"))
        pairs = [(w[n], g[n]) for w, g in zip(layers, grads["dlayers"]) for n in sb.WEIGHT_NAMES] + [(g_final, grads["dg_final"]), (w_head, grads["dw_head"]), (emb, grads["demb"])]
        decays = [0.0 if p.dim() == 1 else 0.1 for p, _ in pairs]
        code_of_state = sb.SBP_STATE_8BIT if eight else sb.SBP_STATE_F32
        table = sb.adamw_tensors([dict(sb.new_adamw_states(p, code_of_state, master), grad=g, weight_decay=w) for (p, g), w in zip(pairs, decays)])
        flat = [{n: x.reshape(-1) for n, x in t.items() if n != "weight_decay"} for t in table.tensors]
        losses = []
        for t in (1, 2, 3):
            want_loss, want = oracle_gradients(ids, emb, layers, g_final, w_head, targets, cfg, 1.0 / T)
            sb.streambp_stack_forward(sc, layers, ckpt, emb, dev_ids)
            out = sb.streambp_stack_backward(sc, layers, g_final, w_head, ckpt, dev_targets, ids=dev_ids, **grads)
            stream.synchronize()
            assert abs(float(out["loss"].item()) - want_loss) <= (TOL[dt] if dt == "f32" else 1e-2) * abs(want_loss)
            for i, ((_, g), w) in enumerate(zip(pairs, want)):
                assert_close(host(g), w, TOL[dt], f"step {t}, gradient {i}")
            norm, factor = sb.streambp_grad_norm(table, 0.05)
            stream.synchronize()
            exact, limit = optim.norm([host(g) for _, g in pairs], 0.05)
            assert abs(norm.item() - exact) <= 5 * 2.0 ** -24 * exact            # (five roundings, as in the norm's own tests; the factor three more)
            assert abs(factor.item() - limit) <= 8 * 2.0 ** -24 * limit
            old = [before(x, eight) for x in flat]
            sb.streambp_adamw_step(sb.adamw_cfg(**HYPER, step=t, state=code_of_state, seed=SEED, zero_grads=True), table, grad_scale=factor)
            stream.synchronize()
            for i, (x, s) in enumerate(zip(flat, old)):
                check(x, s, i, t, eight, decays[i], scale=factor.item(), seed=SEED)
                assert not bool(x["grad"].any()), "a gradient was not cleared"
            losses.append(want_loss)
    assert len(set(losses)) == 3                                                  # each step used the weights that the one before left
