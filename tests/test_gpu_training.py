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


def now_of(lr, step):
    raw = np.zeros(16, np.uint8)
    raw[:8] = np.frombuffer(np.float64(lr).tobytes(), np.uint8)
    raw[8:12] = np.frombuffer(np.int32(step).tobytes(), np.uint8)
    return torch.from_numpy(raw).cuda()


def test_a_captured_training_step():
    """The whole step in one graph, replayed with other tokens, rates and step numbers: the bits of the same step taken eagerly, weights and 8-bit states among them."""
    cfg = dict(dtype="bf16", hidden=256, n_q_heads=4, n_kv_heads=2, head_dim=128, mlp_width=512, vocab=150)
    L, T, d = 2, 300, 256
    lc = sb.layer_cfg(sb.SBP_BF16, 1, T, 96, d, 4, 2, 128, 512, window=WINDOW, sinks=SINKS)
    sc = sb.stack_cfg(lc, L, 150, 100, sb.SBP_OBJ_SFT, 1.0 / T)
    ids, targets = (torch.zeros((1, T), dtype=torch.int32, device="cuda") for _ in range(2))
    now, norm, factor = now_of(1e-3, 1), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(sb.streambp_stack_workspace_bytes(sc), dtype=torch.uint8, device="cuda")
    acfg = sb.adamw_cfg(**HYPER, step=1, state=sb.SBP_STATE_8BIT, seed=SEED, zero_grads=True)

    def model():
        layers = [{n: dev(v, "bf16") for n, v in synth.layer_weights(cfg, seed=10 + l).items()} for l in range(L)]
        rng = np.random.default_rng(5)
        rest = [dev(1 + rng.normal(0, 0.02, d), "bf16"), dev(rng.normal(0, 0.05, (150, d)), "bf16"), dev(rng.normal(0, 1, (150, d)), "bf16")]
        grads = dict(dlayers=[sb.new_layer_grads(w) for w in layers], dg_final=torch.zeros(d, device="cuda"), dw_head=torch.zeros((150, d), device="cuda"),
                     demb=torch.zeros((150, d), device="cuda"), dx0=torch.empty((1, T, d), dtype=torch.bfloat16, device="cuda"), loss=torch.zeros(1, device="cuda"),
                     n_active=torch.zeros(1, dtype=torch.int64, device="cuda"))
        pairs = [(w[n], g[n]) for w, g in zip(layers, grads["dlayers"]) for n in sb.WEIGHT_NAMES] + list(zip(rest, (grads["dg_final"], grads["dw_head"], grads["demb"])))
        table = sb.adamw_tensors([dict(sb.new_adamw_states(p, sb.SBP_STATE_8BIT), grad=g, weight_decay=0.1) for p, g in pairs])
        ckpt = [torch.empty((1, T, d), dtype=torch.bfloat16, device="cuda") for _ in range(L + 1)]
        norm_ws = torch.empty(sb.streambp_grad_norm_workspace_bytes(len(table)), dtype=torch.uint8, device="cuda")

        def step():
            sb.streambp_stack_forward(sc, layers, ckpt, rest[2], ids, workspace=ws)
            sb.streambp_stack_backward(sc, layers, rest[0], rest[1], ckpt, targets, ids=ids, workspace=ws, **grads)
            sb.streambp_grad_norm(table, 0.05, norm, factor, norm_ws)
            sb.streambp_adamw_step(acfg, table, grad_scale=factor, now=now)
        return step, table, grads

    step, table, grads = model()
    eager, other, eager_grads = model()
    kept = [{n: x.clone() for n, x in t.items() if n != "weight_decay"} for t in table.tensors]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for t, k in zip(table.tensors, kept):
        for n in k:
            t[n].copy_(k[n])
    for i in range(1, 5):
        gen = torch.Generator("cuda").manual_seed(i)
        ids.copy_(torch.randint(0, 150, (1, T), generator=gen, device="cuda", dtype=torch.int32))
        targets.copy_(torch.randint(0, 150, (1, T), generator=gen, device="cuda", dtype=torch.int32))
        now.copy_(now_of(HYPER["lr"] / i, i))
        for g in (grads, eager_grads):
            g["loss"].zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = (norm.clone(), factor.clone(), grads["loss"].clone(), grads["dx0"].clone())
        eager()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (norm, factor, eager_grads["loss"], eager_grads["dx0"])))
        for t, o in zip(table.tensors, other.tensors):
            for n in kept[0]:
                assert torch.equal(t[n].reshape(-1).view(torch.uint8), o[n].reshape(-1).view(torch.uint8)), (i, n)
