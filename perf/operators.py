"""Operators of a training step around the layer-wise backward: attention under a sliding window with sinks, the norm of all
gradients, and AdamW over many tensors.

A case is a dict of plain values.  `op` names the operator, the rest its sizes:

  attn   forward and backward of one chunk of queries against the cached prefix, keys visible in the window or among the sinks
         (the first tokens of the sequence); `start`: position of the first query, `pad`: rows of padding in front
  adamw  one AdamW step over the tensors of a model part, with 32-bit or 8-bit states
  norm   norm of the gradients of a model part and the factor that clips them

Plain forms: elementary torch operations in 32 bits, rounded once at the end.  Values: activations N(0, 1), upstream gradients
N(0, 1e-3), weights N(0, 0.02), gradients of a different size in every row, as the rows of a weight matrix have them.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
BLOCK = 256      # elements that share a scale of the 8-bit states
BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.95, 1e-8, 3e-4, 0.1

# Widths of one decoder layer: hidden, query heads, key/value heads, head size, MLP width.
WIDTHS = {
    "7b": (3584, 28, 4, 128, 18944),
    "small": (1024, 16, 4, 64, 2816),
    "tiny": (64, 4, 4, 16, 172),
}


def _attn(name, dtype, hq, hkv, dh, start, q, window, sinks, pad=0):
    return dict(op="attn", name=name, dtype=dtype, hq=hq, hkv=hkv, dh=dh, start=start, q=q, window=window, sinks=sinks, pad=pad)


def _step(name, op, widths, layers, vocab, dtype, grad, **more):
    return dict(op=op, name=name, widths=widths, layers=layers, vocab=vocab, rows=0, dtype=dtype, grad=grad, **more)


def listed():
    return [
        # the smallest call: one chunk of the tiny fp32 configuration, where launches and latency count
        _attn("sinks_tiny_f32", "f32", 4, 4, 16, 192, 64, 32, 2),
        # the last chunk of a 32k sequence at 7B widths: what a chunked backward calls sixteen times per layer
        _attn("sinks_chunk_of_32k", "bf16", 28, 4, 128, 30720, 2048, 4096, 4),
        # a whole 32k sequence in one call
        _attn("sinks_sequence_32k", "bf16", 28, 4, 128, 0, 32768, 4096, 4),
        # a ragged chunk behind front padding, more sinks than one key block of a wave
        _attn("sinks_ragged_padded", "bf16", 32, 8, 128, 3001, 777, 1024, 40, 100),
        # a small model's 64-wide heads, a short window
        _attn("sinks_heads_of_64", "bf16", 16, 4, 64, 0, 4095, 512, 16),
        # the tiny fp32 model: a dozen small tensors, latency
        _step("adamw_tiny_f32", "adamw", "tiny", 1, 512, "f32", "f32", master=False, bits=32),
        # one layer at 7B widths: bf16 weights with an fp32 copy, fp32 gradients, 32-bit states
        _step("adamw_7b_layer_master", "adamw", "7b", 1, 0, "bf16", "f32", master=True, bits=32),
        # the LM head at 7B widths in the least memory: bf16 weights and gradients, 8-bit states
        _step("adamw_7b_head_8bit", "adamw", "7b", 0, 152064, "bf16", "bf16", master=False, bits=8),
        # a small model with a vocabulary that is no round number: a hundred tensors, large and small, 8-bit states
        _step("adamw_small_model_8bit", "adamw", "small", 12, 50257, "bf16", "f32", master=False, bits=8),
        # norms: latency, and one layer at 7B widths
        _step("norm_tiny_f32", "norm", "tiny", 1, 512, "f32", "f32"),
        _step("norm_7b_layer", "norm", "7b", 1, 0, "bf16", "f32"),
        # ... and bf16 gradients of a small model
        _step("norm_small_model_bf16", "norm", "small", 12, 50257, "bf16", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "adamw", "adamw", "norm"])
    if op == "attn":
        kind = rng.choice(["f32", "bf16_128", "bf16_128", "bf16_64"])
        if kind == "f32":
            hkv = rng.choice([1, 2, 4])
            c = dict(dtype="f32", hq=hkv * rng.choice([1, 2, 4]), hkv=hkv, dh=rng.choice([16, 32, 40, 64]), start=_log(rng, 1, 2000) - 1,
                     q=_log(rng, 1, 1000), window=_log(rng, 1, 500))
        else:
            hkv = rng.choice([2, 4, 8])
            c = dict(dtype="bf16", hq=hkv * rng.choice([1, 2, 4, 7]), hkv=hkv, dh=128 if kind == "bf16_128" else 64, start=_log(rng, 1, 30000) - 1,
                     q=_log(rng, 1, 8192), window=_log(rng, 16, 4096))
            c["hq"] = min(c["hq"], 28 // hkv * hkv)
        return dict(op=op, **c, sinks=_log(rng, 1, 200), pad=rng.choice([0, 0, rng.randrange(1, 300)]))
    # rows: one more matrix of odd sizes, beside the layers
    c = dict(op=op, widths=rng.choice(["small", "small", "tiny"]), layers=rng.randrange(0, 5), vocab=rng.choice([0, _log(rng, 100, 60000)]),
             rows=_log(rng, 1, 20000), dtype=rng.choice(["f32", "bf16"]), grad="f32")
    if c["dtype"] == "bf16":
        c["grad"] = rng.choice(["f32", "bf16"])
    if op == "adamw":
        c["master"] = c["dtype"] == "bf16" and rng.random() < 0.5
        c["bits"] = rng.choice([8, 32])
    return c


def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _shapes(c):
    """The tensors of a model part: layers of seven matrices and two norm gains, final norm, embedding and head, and a matrix of `rows` rows."""
    d, hq, hkv, dh, f = WIDTHS[c["widths"]]
    layer = [(hq * dh, d), (hkv * dh, d), (hkv * dh, d), (d, hq * dh), (f, d), (f, d), (d, f), (d,), (d,)]
    s = layer * c["layers"]
    if c["vocab"]:
        s += [(c["vocab"], d)] if not c["layers"] else [(c["vocab"], d), (d,), (c["vocab"], d)]
    if c["rows"]:
        s.append((c["rows"], 2 * (c["rows"] % 300) + 1))
    return s


def _numel(s):
    n = 1
    for x in s:
        n *= x
    return n


def prepare(case, seed):
    g = torch.Generator(DEV)
    g.manual_seed(int(seed))

    def randn(shape, size=1.0, dtype=torch.float32):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * size).to(dtype)

    c = dict(case)
    t = _type(c["dtype"])
    if c["op"] == "attn":
        n = c["start"] + c["q"]
        s = dict(q=randn((c["q"], c["hq"], c["dh"]), 1.0, t), k=randn((n, c["hkv"], c["dh"]), 1.0, t), v=randn((n, c["hkv"], c["dh"]), 1.0, t),
                 d_o=randn((c["q"], c["hq"], c["dh"]), 1e-3, t))
        return dict(s, case=c)
    shapes, grads, params, states = _shapes(c), [], [], []
    # weights and states: a flat buffer of each kind, every tensor at a multiple of 256 elements
    starts = [0]
    for shape in shapes:
        starts.append(starts[-1] + -(-_numel(shape) // BLOCK) * BLOCK)
    flat = {}
    if c["op"] == "adamw":
        kinds = dict(p=t, m=torch.float32, v=torch.float32)
        if c["master"]:
            kinds["master"] = torch.float32
        if c["bits"] == 8:
            kinds.update(m=torch.float8_e4m3fn, v=torch.float8_e4m3fn, m_scale=torch.float8_e8m0fnu, v_scale=torch.float8_e8m0fnu)
        flat = {k: torch.zeros(starts[-1] // (BLOCK if "scale" in k else 1), dtype=torch.uint8 if "float8" in str(d) else d, device=DEV).view(d) for k, d in kinds.items()}

    def place(kind, i, value):
        if kind not in flat:
            return None
        n, per = value.numel(), BLOCK if "scale" in kind else 1
        to = flat[kind][starts[i] // per:starts[i] // per + n].reshape(value.shape)
        to.copy_(value)
        return to

    for i, shape in enumerate(shapes):
        rows = torch.exp(randn((shape[0],) + (1,) * (len(shape) - 1), 1.0)) * 1e-3      # the size of a row's gradients
        matrix = len(shape) > 1
        grads.append((randn(shape) * rows).to(_type(c["grad"]) if matrix else torch.float32))      # gains: fp32, as the library leaves them
        if c["op"] == "norm":
            continue
        p = randn(shape, 0.02) if matrix else 1 + randn(shape, 0.02)
        params.append((place("p", i, p), place("master", i, p)))
        m, r = randn(shape) * rows * 0.2, torch.abs(randn(shape, 0.3) + 1) * rows
        (m, ms), (v, vs) = (_quantize(m, None), _quantize(r, None)) if c["bits"] == 8 else ((m, None), (r * r, None))
        states.append((place("m", i, m), None if ms is None else place("m_scale", i, ms), place("v", i, v), None if vs is None else place("v_scale", i, vs)))
    s = dict(case=c, grads=grads, params=params, states=states, flat=flat, starts=starts)
    if c["op"] == "norm":
        s["max_norm"] = 1.0
    else:
        s.update(step=1000, seed=int(seed) & 0xffff, scale=torch.full((1,), 0.75, device=DEV))
    if own:      # the table of tensors, which a program makes once
        from paper_2506_03077_amd import binding as sb
        if c["op"] == "norm":
            s["table"] = sb.adamw_tensors([dict(grad=x) for x in grads])
        else:
            s["table"] = sb.adamw_tensors([dict(param=p, master=w, grad=x, m=m, m_scale=ms, v=v, v_scale=vs, weight_decay=DECAY if p.dim() > 1 else 0.0)
                                           for (p, w), x, (m, ms, v, vs) in zip(params, grads, states)])
            s["cfg"] = sb.adamw_cfg(lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS, step=s["step"], seed=s["seed"],
                                    state=sb.SBP_STATE_8BIT if c["bits"] == 8 else sb.SBP_STATE_F32)
    return s


# ------------------------------------------------------------------------------------------------------------ AdamW --
def _mix(x):
    """A 32-bit word, well mixed (in 64-bit integers)."""
    x = (x ^ (x >> 16)) * 0x9E3779B1 & 0xffffffff
    x = (x ^ (x >> 15)) * 0xB504F333 & 0xffffffff
    return x ^ (x >> 16)


def _random(seed, step, tensor, n):
    """32 random bits for each element of a tensor."""
    key = _mix(_mix(_mix(seed) + step & 0xffffffff) + tensor & 0xffffffff)
    return _mix(torch.arange(n, device=DEV) ^ key)      # (fewer than 2^32 elements)


def _quantize(x, u, at_least_one=False):
    """x as e4m3 values times a power of two (e8m0) for each block of 256: the largest magnitude lies in [128, 256) of it.
    u in [0, 1): what is added before the part of a step is cut off; None: 1/2.  at_least_one: nothing but zero becomes zero."""
    n = x.numel()
    flat = torch.nn.functional.pad(x.reshape(-1).double(), (0, -n % BLOCK)).reshape(-1, BLOCK)
    # (64 bits: a value next to the border of two steps is to fall on its own side)
    top = flat.float().abs().amax(dim=1)
    e = torch.where(top > 0, torch.frexp(top).exponent.clamp(min=-118), -118) - 8
    a = torch.ldexp(flat.abs(), -e[:, None])
    step = torch.exp2(torch.frexp(a).exponent.clamp(min=-5).double() - 4)      # of three bits behind the leading one, from 2^-6 on
    u = 0.5 if u is None else torch.nn.functional.pad(u, (0, -n % BLOCK)).reshape(-1, BLOCK)
    k = torch.floor(a / step + u)
    if at_least_one:
        k = torch.where((a > 0) & (k < 1), 1.0, k)
    q = torch.copysign(k * step, flat).reshape(-1)[:n].reshape(x.shape)
    return q.float().to(torch.float8_e4m3fn), (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _value(q, scale, dtype):
    n = q.numel()
    e = scale.view(torch.uint8).to(dtype)
    x = q.reshape(-1).to(torch.float32).to(dtype)
    return (x * torch.exp2(e - 127).repeat_interleave(BLOCK)[:n]).reshape(q.shape)


def _adamw_plain(s, tensor):
    c, t = s["case"], s["step"]
    (p, master), grad, (m, ms, v, vs) = s["params"][tensor], s["grads"][tensor], s["states"][tensor]
    eight = c["bits"] == 8
    bits = _random(s["seed"], t, tensor, p.numel()) if eight or (p.dtype == torch.bfloat16 and master is None) else None
    g = grad.float() * s["scale"]
    m1 = (_value(m, ms, torch.float32) if eight else m) * BETA1 + g * (1 - BETA1)
    v1 = (_value(v, vs, torch.float32).square() if eight else v) * BETA2 + g * g * (1 - BETA2)
    root = torch.sqrt(v1)
    w = (p if master is None else master).float() * (1 - LR * (DECAY if p.dim() > 1 else 0.0))
    w = w - LR / (1 - BETA1 ** t) * m1 / (root / math.sqrt(1 - BETA2 ** t) + EPS)
    if master is not None:
        master.copy_(w)
    if p.dtype == torch.bfloat16 and master is None:      # rounded up with the probability of what is cut off
        word = w.view(torch.int32) + (bits & 0xffff).reshape(w.shape).to(torch.int32)
        p.copy_((word & -65536).view(torch.float32))
    else:
        p.copy_(w)
    if eight:
        for to, scale, x, u, one in ((m, ms, m1, bits >> 12, False), (v, vs, root, bits & 0xfffff, True)):
            q, e = _quantize(x, u.double() / 2 ** 20, one)
            to.copy_(q)
            scale.copy_(e)
    else:
        m.copy_(m1)
        v.copy_(v1)


def _exact_eight(x, u, at_least_one):
    """x in 64 bits as the step stores it: the neighbours among the e4m3 values by a search, the upper one where u covers what is left."""
    codes = torch.arange(127, device=DEV)
    grid = torch.where(codes < 8, codes * 2.0 ** -9, (1 + (codes % 8) / 8.0) * torch.exp2((codes // 8 - 7).double()))
    n, blocks = x.numel(), -(-x.numel() // BLOCK)
    padded = torch.zeros(blocks * BLOCK, dtype=torch.float64, device=DEV)
    padded[:n] = x.reshape(-1)
    top = padded.reshape(blocks, BLOCK).abs().amax(1)
    e = torch.where(top > 0, torch.floor(torch.log2(top)) - 7, -126.0).clamp(min=-126)
    a = padded.abs() / torch.exp2(e).repeat_interleave(BLOCK)
    low = torch.searchsorted(grid, a, right=True) - 1
    part = (a - grid[low]) / (grid[low + 1] - grid[low])
    low[:n] += part[:n] + u >= 1
    if at_least_one:
        low = torch.where((a > 0) & (low == 0), 1, low)
    return torch.copysign(grid[low], padded)[:n], torch.exp2(e)


def _adamw_exact(s):
    """The step in 64 bits, laid out like the state's buffers."""
    c, t = s["case"], s["step"]
    eight = c["bits"] == 8
    out = {k: torch.zeros(x.numel(), dtype=torch.float64, device=DEV) for k, x in s["flat"].items()}
    if eight:
        out["m_scale"].fill_(2.0 ** -127)      # (a byte of zero, between the tensors)
        out["v_scale"].fill_(2.0 ** -127)
    decode = lambda q, e: q.float().double() * torch.exp2(e.view(torch.uint8).double() - 127).repeat_interleave(BLOCK)[:q.numel()].reshape(q.shape)
    for i, ((p, master), grad, (m, ms, v, vs)) in enumerate(zip(s["params"], s["grads"], s["states"])):
        m0, v0 = (decode(m, ms), decode(v, vs) ** 2) if eight else (m.double(), v.double())
        g = grad.double() * s["scale"].double()
        m1, v1 = BETA1 * m0 + (1 - BETA1) * g, BETA2 * v0 + (1 - BETA2) * g ** 2
        mh, vh = m1 / (1 - BETA1 ** t), v1 / (1 - BETA2 ** t)
        w = (p if master is None else master).double()
        w = w - LR * ((DECAY if p.dim() > 1 else 0.0) * w + mh / (vh ** 0.5 + EPS))
        found = dict(p=w, master=w, m=m1, v=v1)
        if eight:
            bits = _random(s["seed"], t, i, p.numel())
            found["m"], found["m_scale"] = _exact_eight(m1, (bits >> 12) / 2.0 ** 20, False)
            found["v"], found["v_scale"] = _exact_eight(v1 ** 0.5, (bits & 0xfffff) / 2.0 ** 20, True)
        for k in out:
            at = s["starts"][i] // (BLOCK if "scale" in k else 1)
            out[k][at:at + found[k].numel()] = found[k].reshape(-1)
    return out


# -------------------------------------------------------------------------------------------------------- attention --
def _attn_plain(s):
    """All blocks of queries at once, each against the sinks and the keys that its window reaches, in 32 bits."""
    c = s["case"]
    hq, hkv, dh, start, nq, window, pad = (c[x] for x in ("hq", "hkv", "dh", "start", "q", "window", "pad"))
    group, scale, n = hq // hkv, 1 / math.sqrt(dh), start + nq
    sinks = max(0, min(c["sinks"], n - pad))
    size = min(512, nq)                                   # queries of a block
    blocks = -(-nq // size)
    reach = min(window - 1 + size, n + size)
    pos = start + torch.arange(blocks * size, device=DEV).reshape(blocks, size, 1)
    key = torch.cat([pad + torch.arange(sinks, device=DEV).expand(blocks, sinks),
                     start + size * (torch.arange(blocks, device=DEV)[:, None] + 1) - reach + torch.arange(reach, device=DEV)], 1)[:, None, :]
    near = (key > pos - window) & (key >= pad) & (key <= pos)
    far = (key < pad + sinks) & (key <= pos - window)
    seen = torch.where(torch.arange(sinks + reach, device=DEV) < sinks, far, near) & (pos < n)
    at = key.reshape(-1).clamp(0, n - 1)

    def rows(x):      # [blocks, kv heads, queries of its heads, dh]
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, blocks * size - nq)).reshape(blocks, size, hkv, group, dh)
        return x.permute(0, 2, 3, 1, 4).reshape(blocks, hkv, group * size, dh)

    def back(x):
        return x.reshape(blocks, hkv, group, size, dh).permute(0, 3, 1, 2, 4).reshape(blocks * size, hq, dh)[:nq]

    def keys(x):      # [blocks, kv heads, keys, dh]
        return x.float()[at].reshape(blocks, -1, hkv, dh).permute(0, 2, 1, 3).contiguous()

    q, d_o, k, v = rows(s["q"]), rows(s["d_o"]), keys(s["k"]), keys(s["v"])
    mask = seen.repeat(1, group, 1)[:, None]
    x = (q @ k.transpose(2, 3) * scale).masked_fill_(~mask, -math.inf)
    top = x.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp_(x.sub_(top))
    total = p.sum(3, keepdim=True)
    lse = (torch.log(total) + top).reshape(blocks, hkv, group, size).permute(1, 2, 0, 3).reshape(hq, blocks * size)[:, :nq]
    p.mul_(torch.where(total > 0, 1 / total, 0.0))
    o = p @ v
    dp = d_o @ v.transpose(2, 3)
    ds = dp.sub_((d_o * o).sum(3, keepdim=True)).mul_(p).mul_(scale)
    dq, dk, dv = ds @ k, ds.transpose(2, 3) @ q, p.transpose(2, 3) @ d_o

    def sums(x):      # of a key over the blocks that read it
        return torch.zeros(n, hkv, dh, device=DEV).index_add_(0, at, x.permute(0, 2, 1, 3).reshape(-1, hkv, dh))

    t = s["q"].dtype
    return [back(o).to(t), lse.contiguous(), back(dq).to(t), sums(dk).to(t), sums(dv).to(t)]


def _attn_exact(s):
    c = s["case"]
    n, group, scale = c["start"] + c["q"], c["hq"] // c["hkv"], c["dh"] ** -0.5
    q, k, v, d_o = (s[x].double().transpose(0, 1).contiguous() for x in ("q", "k", "v", "d_o"))
    o, dq, dk, dv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    lse = torch.full(q.shape[:2], -math.inf, device=DEV, dtype=torch.float64)
    for a in range(0, c["q"], 1024):
        b = min(a + 1024, c["q"])
        p = torch.arange(c["start"] + a, c["start"] + b, device=DEV)[:, None]
        first = min(max(c["pad"], c["start"] + a - c["window"] + 1), n)
        u = torch.arange(first, c["start"] + b, device=DEV)
        u = torch.cat([torch.arange(c["pad"], max(c["pad"], min(c["pad"] + c["sinks"], first)), device=DEV), u])
        vis = (u >= c["pad"]) & (u <= p) & ((u > p - c["window"]) | (u < c["pad"] + c["sinks"]))
        if not bool(vis.any()):
            continue
        for h in range(c["hq"]):
            g = h // group
            kk, vv = k[g, u], v[g, u]
            z = torch.where(vis, q[h, a:b] @ kk.T * scale, -math.inf)
            lse[h, a:b] = torch.logsumexp(z, 1)
            w = torch.where(vis, torch.exp(z - lse[h, a:b, None]), 0.0)
            o[h, a:b] = w @ vv
            dw = d_o[h, a:b] @ vv.T
            dz = w * (dw - (w * dw).sum(1, keepdim=True))
            dq[h, a:b] = scale * dz @ kk
            dk[g].index_add_(0, u, scale * dz.T @ q[h, a:b])
            dv[g].index_add_(0, u, w.T @ d_o[h, a:b])
    turn = lambda x: x.transpose(0, 1).contiguous()
    return [turn(o), lse, turn(dq), turn(dk), turn(dv)]


# -------------------------------------------------------------------------------------------------------------- all --
def run(state):
    c = state["case"]
    if c["op"] == "attn":
        if not own:
            return _attn_plain(state)
        from paper_2506_03077_amd import binding as sb
        q, k, v = state["q"], state["k"], state["v"]
        cfg = sb.attn_cfg(sb.SBP_BF16 if c["dtype"] == "bf16" else sb.SBP_F32, c["hq"], c["hkv"], c["dh"], c["start"], c["q"], 1 / math.sqrt(c["dh"]),
                          window=c["window"], kv_first=c["pad"], sinks=c["sinks"])
        o, lse = sb.streambp_attn_chunk_forward(cfg, q, k, v)
        dq, dk, dv = sb.streambp_attn_chunk_backward(cfg, q, k, v, o, lse, state["d_o"])
        return [o, lse, dq, dk.to(k.dtype), dv.to(v.dtype)]
    if c["op"] == "norm":
        if not own:
            norm = torch.sqrt(torch.stack([x.float().square().sum(dtype=torch.float64) for x in state["grads"]]).sum()).float()
            return [norm.reshape(1), torch.clamp(state["max_norm"] / norm, max=1.0).reshape(1)]
        from paper_2506_03077_amd import binding as sb
        return list(sb.streambp_grad_norm(state["table"], state["max_norm"]))
    if not own:
        for i in range(len(state["params"])):
            _adamw_plain(state, i)
        return state["flat"]
    from paper_2506_03077_amd import binding as sb
    sb.streambp_adamw_step(state["cfg"], state["table"], grad_scale=state["scale"])
    return state["flat"]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attn":
        return _attn_exact(s)
    if case["op"] == "norm":
        total = torch.zeros((), dtype=torch.float64, device=DEV)
        for x in s["grads"]:
            total += (x.double() ** 2).sum()
        norm = total ** 0.5
        return [norm.reshape(1), torch.minimum(s["max_norm"] / norm, torch.ones_like(norm)).reshape(1)]
    return _adamw_exact(s)


def _pairs(c):
    """Visible (query, key) pairs of a head."""
    n = 0
    for t in range(c["q"]):
        p = c["start"] + t
        lo = max(c["pad"], p - c["window"] + 1)
        n += max(0, p - lo + 1) + max(0, min(c["pad"] + c["sinks"], lo) - c["pad"]) * (p >= c["pad"])
    return n


def work(case):
    c = case
    if c["op"] == "attn":
        es = 2 if c["dtype"] == "bf16" else 4
        first = max(c["pad"], c["start"] - c["window"] + 1)
        keys = max(0, c["start"] + c["q"] - first) + max(0, min(c["pad"] + c["sinks"], first) - c["pad"])
        # q and d_o in, o, dq and the log-sum-exps out; k and v in, dk and dv out
        return dict(bytes=4 * c["q"] * c["hq"] * c["dh"] * es + 4 * c["q"] * c["hq"] + 4 * keys * c["hkv"] * c["dh"] * es, flops=14 * c["dh"] * c["hq"] * _pairs(c))
    shapes = _shapes(c)
    es = 2 if c["dtype"] == "bf16" else 4
    n = sum(_numel(s) for s in shapes)
    grads = sum(_numel(s) * (2 if c["grad"] == "bf16" and len(s) > 1 else 4) for s in shapes)
    if c["op"] == "norm":
        return dict(bytes=grads, flops=2 * n)
    state = 4 * n if c["bits"] == 8 else 16 * n
    return dict(bytes=2 * es * n + (8 * n if c["master"] else 0) + grads + state, flops=15 * n)
