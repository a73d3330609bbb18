"""AdamW over many tensors against the fp64 oracle: every pair of types, 32-bit and 8-bit states, sizes around the thread's eight, the block's
256, the pass's 2048 and the workgroup's 8192 elements, tensors that start anywhere, gradients that are not finite, captured steps.

Bounds, eps = 2^-24 (half a step of fp32, relative): constants are rounded once, products and sums once each.
  m: two products of three roundings (constant, scaled gradient, product) and a sum: 4 eps (|b1 m| + |(1 - b1) g|), tested with 6
  v: gradient scaled, squared, times a rounded constant, and a sum: at most 6 eps of v (8-bit states: times a constant of three roundings' product, squared, and a sum: 7), tested with 8
  p: m's error and at most 12 roundings of the update (v's 8 count half through the root; root, two products, sum, quotient, constant, product), the decayed weight's three and
     the difference: bias1 / den * 6 eps Sm + 12 eps |update| + 4 eps |p|, tested with 16 and 6
"""
import numpy as np
import pytest
import torch

from oracle import optim
from paper_2506_03077_amd import binding as sb

pytestmark = pytest.mark.gpu

EPS32 = 2.0 ** -24
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.97, eps=1e-8)
SIZES = [1, 7, 8, 255, 256, 257, 2047, 2048, 2049, 8191, 8192, 8193, 20001]


def make(n, dtype, grad_dtype, master, eight, seed, offset=0, spread=2.0):
    """A tensor's dict (device) in the middle of guarded buffers, `offset` elements behind a 256-byte border."""
    rng = np.random.default_rng(seed)
    out, guards = {}, {}

    def place(name, values, dt):
        size = torch.empty((), dtype=dt).element_size()
        raw = torch.full(((n + 512) * size,), 0x5A, dtype=torch.uint8, device="cuda")
        view = raw[(256 + offset) * size:(256 + offset + len(values)) * size].view(dt)
        view.copy_(values if isinstance(values, torch.Tensor) else torch.from_numpy(values).to("cuda"))
        out[name], guards[name] = view, (raw, (256 + offset) * size, len(values) * size)

    rows = np.exp(spread * rng.standard_normal(-(-n // 100))).repeat(100)[:n] * 1e-3
    p = rng.standard_normal(n)
    place("param", p.astype(np.float32), dtype)
    if master:
        place("master", p.astype(np.float32), torch.float32)
    place("grad", (rng.standard_normal(n) * rows).astype(np.float32), grad_dtype)
    m, r = rng.standard_normal(n) * rows * 0.3, np.abs(1 + 0.3 * rng.standard_normal(n)) * rows
    if n > 3:
        m[n // 3] = r[n // 3] = 0.0                    # an element that has seen nothing
    if not eight:
        place("m", m.astype(np.float32), torch.float32)
        place("v", (r * r).astype(np.float32), torch.float32)
    else:
        for name, x in (("m", m), ("v", r)):
            e, _ = optim.exponents(x)
            code, _ = optim.quantize(x, e, 0.5)
            code = np.where((x != 0) & (code == 0), 1, code) if name == "v" else code
            code = code | np.where(x < 0, 128, 0)
            place(name, torch.from_numpy(code.astype(np.uint8)).to("cuda").view(torch.float8_e4m3fn), torch.float8_e4m3fn)
            place(name + "_scale", torch.from_numpy((e + 127).astype(np.uint8)).to("cuda"), torch.uint8)
    return out, guards


def check_guards(guards):
    for name, (raw, first, size) in guards.items():
        assert bool((raw[:first] == 0x5A).all()) and bool((raw[first + size:] == 0x5A).all()), f"{name}: bytes beside the tensor were written"


def host(x):
    if x.dtype == torch.float8_e8m0fnu:      # (the byte)
        x = x.view(torch.uint8)
    return x.detach().to(torch.float64).cpu().numpy() if x.dtype != torch.uint8 else x.cpu().numpy()


def codes(x):
    return x.view(torch.uint8).cpu().numpy().astype(np.int64)


def decoded(x, scale):
    c = codes(x)
    return np.where(c >= 128, -1.0, 1.0) * np.where((c & 127) == 127, np.nan, optim.GRID[np.minimum(c & 127, 126)]) * 2.0 ** optim.per_element(host(scale).astype(np.float64) - 127, len(c))


def before(t, eight):
    s = {k: host(x) for k, x in t.items()}
    if eight:
        s["m"], s["v"] = decoded(t["m"], t["m_scale"]), decoded(t["v"], t["v_scale"]) ** 2
    s["w"] = s["master"] if "master" in s else s["param"]
    return s


def check(t, s, index, step, eight, decay, scale=1.0, seed=0):
    """A tensor after the step against what it was before."""
    n = len(s["w"])
    p, m, v = optim.step(s["w"], s["m"], s["v"], s["grad"], step, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], decay, scale)
    b1, b2 = HYPER["beta1"], HYPER["beta2"]
    sm = b1 * np.abs(s["m"]) + (1 - b1) * np.abs(s["grad"] * scale)
    den = np.sqrt(v) / np.sqrt(1 - b2 ** step) + HYPER["eps"]
    rate = HYPER["lr"] / (1 - b1 ** step)
    tiny = 1e-37                                      # (fp32's own end)
    m_off, v_off = 6 * EPS32 * sm + tiny, 8 * EPS32 * v + tiny
    p_off = rate / den * m_off + 16 * EPS32 * rate * np.abs(m) / den + 6 * EPS32 * np.abs(s["w"])
    word = optim.random_bits(seed, step, index, n)
    if t["param"].dtype == torch.float32:
        assert (np.abs(host(t["param"]) - p) <= p_off).all()
    elif "master" in t:
        assert (np.abs(host(t["master"]) - p) <= p_off).all()
        assert torch.equal(t["param"], t["master"].bfloat16())
    else:
        got = host(t["param"])
        unit = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(p), 1e-30))) - 7)       # a step of bf16
        low = np.floor(np.abs(p) / unit) * unit
        part = (np.abs(p) - low) / unit
        up = part + (word & np.uint64(0xffff)) / 65536.0
        want = np.copysign(np.where(up >= 1, low + unit, low), p)
        off = p_off / unit + 2.0 ** -16                                           # of a step; what fp32 has below bf16's last bit is cut to 16 bits
        sure = np.minimum(np.abs(up - 1), np.minimum(part, 1 - part)) > off
        assert sure.mean() > 0.95 or n < 100
        assert (got[sure] == want[sure]).all()
        assert (np.abs(got - p) <= unit * (1 + off)).all()
    if not eight:
        assert (np.abs(host(t["m"]) - m) <= m_off).all() and (np.abs(host(t["v"]) - v) <= v_off).all()
        return
    for name, x, off, u, one in (("m", m, m_off, (word >> np.uint64(12)) / 2.0 ** 20, False),
                                 ("v", np.sqrt(v), 6 * EPS32 * np.sqrt(v) + tiny, (word & np.uint64(0xfffff)) / 2.0 ** 20, True)):
        e, room = optim.exponents(x)
        byte = host(t[name + "_scale"]).astype(np.int64)
        clear = room > 64 * EPS32
        assert clear.mean() > 0.9 and (byte[clear] == e[clear] + 127).all()
        e = byte - 127
        want, margin = optim.quantize(x, e, u, one)
        got = codes(t[name])
        assert (((got >= 128) == (x < 0)) | (x == 0) | (np.abs(x) < off)).all()
        got = got & 127
        step_of = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 1e-300) / 2.0 ** optim.per_element(e.astype(float), n))) - 3), 2.0 ** -9) * \
            2.0 ** optim.per_element(e.astype(float), n)
        sure = margin > off / step_of + 2.0 ** -19                                # (a step's 20 bits are cut, in the fixed-point range rounded)
        assert sure.mean() > 0.99 or n < 1000
        assert (got[sure] == want[sure]).all(), (name, np.flatnonzero(sure & (got != want))[:5])
        assert (np.abs(got - want) <= 1).all()
        if one:
            assert (got[x > 0] > 0).all()


TYPES = [(torch.float32, torch.float32, False), (torch.float32, torch.bfloat16, False), (torch.bfloat16, torch.float32, False),
         (torch.bfloat16, torch.bfloat16, False), (torch.bfloat16, torch.float32, True), (torch.bfloat16, torch.bfloat16, True)]


def run(tensors, eight, step=3, seed=11, decays=None, scale=None, zero=False, now=None):
    decays = decays or [0.1] * len(tensors)
    table = sb.adamw_tensors([dict(t, weight_decay=d) for t, d in zip(tensors, decays)])
    cfg = sb.adamw_cfg(**HYPER, step=step, seed=seed, state=int(eight), zero_grads=zero)
    sb.streambp_adamw_step(cfg, table, grad_scale=scale, now=now)
    torch.cuda.synchronize()
    return table


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,grad_dtype,master", TYPES)
def test_sizes(dtype, grad_dtype, master, eight):
    made = [make(n, dtype, grad_dtype, master, eight, 100 + n) for n in SIZES]
    old = [before(t, eight) for t, _ in made]
    decays = [0.1 * (i % 3) for i in range(len(made))]
    run([t for t, _ in made], eight, decays=decays)
    for i, ((t, guards), s) in enumerate(zip(made, old)):
        check(t, s, i, 3, eight, decays[i], seed=11)
        check_guards(guards)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,grad_dtype,master", TYPES)
def test_tensors_that_start_anywhere(dtype, grad_dtype, master, eight):
    made = [make(n, dtype, grad_dtype, master, eight, n, offset=1 + i % 7) for i, n in enumerate((5, 300, 4097, 9000))]
    old = [before(t, eight) for t, _ in made]
    run([t for t, _ in made], eight)
    for i, ((t, guards), s) in enumerate(zip(made, old)):
        check(t, s, i, 3, eight, 0.1, seed=11)
        check_guards(guards)


@pytest.mark.parametrize("eight", [False, True])
def test_the_start_of_a_tensor_changes_no_bit(eight):
    """Eight at a time or element by element: the same arithmetic."""
    made = [make(6000, torch.bfloat16, torch.float32, False, eight, 5, offset=o)[0] for o in (0, 3)]
    for t in made:
        run([t], eight)
    for name in made[0]:
        assert torch.equal(made[0][name].view(torch.uint8), made[1][name].view(torch.uint8)), name


@pytest.mark.parametrize("eight", [False, True])
def test_more_tensors_than_a_launch_takes(eight):
    """100 tensors of different types, some of them empty, over several launches: each gets its own bits and decay."""
    made = [make(1 + 37 * i % 900, *TYPES[i % 6], eight, i) for i in range(100)]
    empty = dict(param=torch.empty(0, device="cuda"), grad=torch.empty(0, device="cuda"), m=torch.empty(0, device="cuda"), v=torch.empty(0, device="cuda"))
    if eight:
        byte = torch.empty(0, dtype=torch.uint8, device="cuda")
        empty.update(m=byte, v=byte, m_scale=byte, v_scale=byte)
    tensors = [t for t, _ in made]
    tensors[40:40] = [empty] * 3
    tensors.append(empty)
    old = [None if t is empty else before(t, eight) for t in tensors]
    run(tensors, eight, decays=[0.01 * (i % 5) for i in range(len(tensors))])
    for i, (t, s) in enumerate(zip(tensors, old)):
        if s is not None:
            check(t, s, i, 3, eight, 0.01 * (i % 5), seed=11)
    for _, guards in made:
        check_guards(guards)


@pytest.mark.parametrize("eight", [False, True])
def test_states_start_from_zeros(eight):
    p = torch.randn(3000, device="cuda").bfloat16()
    t = sb.new_adamw_states(p, state=int(eight))
    t["grad"] = torch.randn(3000, device="cuda") * 1e-3
    s = before(t, eight)
    run([t], eight, step=1)
    check(t, s, 0, 1, eight, 0.1, seed=11)


@pytest.mark.parametrize("eight", [False, True])
def test_the_same_call_gives_the_same_bits_and_another_seed_or_step_others(eight):
    out = []
    for seed, step in ((1, 3), (1, 3), (2, 3)):
        t, _ = make(5000, torch.bfloat16, torch.float32, False, eight, 9)
        run([t], eight, seed=seed, step=step)
        out.append(t["param"].clone())
    assert torch.equal(out[0], out[1]) and not torch.equal(out[0], out[2])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("zero", [False, True])
def test_grad_scale_and_zeroed_gradients(eight, zero):
    for dtype, grad_dtype, master in TYPES:
        t, guards = make(2500, dtype, grad_dtype, master, eight, 21)
        s = before(t, eight)
        run([t], eight, scale=torch.full((1,), 0.25, device="cuda"), zero=zero)
        check(t, s, 0, 3, eight, 0.1, scale=0.25, seed=11)
        assert np.array_equal(host(t["grad"]), np.zeros(2500) if zero else s["grad"])
        check_guards(guards)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("zero", [False, True])
def test_a_scale_that_is_not_finite_moves_nothing(bad, zero):
    for eight in (False, True):
        t, guards = make(9000, torch.bfloat16, torch.bfloat16, True, eight, 22)
        old = {k: x.clone() for k, x in t.items()}
        run([t], eight, scale=torch.full((1,), bad, device="cuda"), zero=zero)
        for k, x in t.items():
            want = torch.zeros_like(x) if zero and k == "grad" else old[k]
            assert torch.equal(x.view(torch.uint8), want.view(torch.uint8)), k
        check_guards(guards)


@pytest.mark.parametrize("eight", [False, True])
def test_gradients_that_are_not_finite_stay_with_their_elements(eight):
    t, _ = make(1024, torch.float32, torch.float32, False, eight, 23)
    t["grad"][5], t["grad"][300], t["grad"][1023] = float("nan"), float("inf"), -float("inf")
    s = before(t, eight)
    run([t], eight)
    rest = np.ones(1024, bool)
    rest[[5, 300, 1023]] = False
    with np.errstate(invalid="ignore"):
        p, _, _ = optim.step(s["w"], s["m"], s["v"], s["grad"], 3, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], 0.1)
    got = host(t["param"])
    assert np.isnan(got[[5, 300, 1023]]).all() and np.allclose(got[rest], p[rest], rtol=1e-5)
    if eight:
        m = decoded(t["m"], t["m_scale"])
        assert np.isnan(m[~rest]).all() and np.isfinite(m[rest]).all()
        e, _ = optim.exponents(np.where(rest, HYPER["beta1"] * s["m"] + (1 - HYPER["beta1"]) * s["grad"], 0.0))
        assert np.array_equal(host(t["m_scale"]).astype(int), e + 127)


def test_betas_and_eps_of_zero():
    t, _ = make(1000, torch.float32, torch.float32, False, False, 24)
    t["grad"][t["grad"] == 0] = 1e-3
    s = before(t, False)
    table = sb.adamw_tensors([t])
    sb.streambp_adamw_step(sb.adamw_cfg(lr=1e-2, beta1=0.0, beta2=0.0, eps=0.0, step=5), table)
    # the sign of the gradient: squared and rooted again, 4 roundings, and the weight's
    want = s["w"] - 1e-2 * np.sign(s["grad"])
    assert np.abs(host(t["param"]) - want).max() <= 1e-2 * 8 * EPS32 + 4 * EPS32 * np.abs(s["w"]).max()
    assert (np.abs(host(t["v"]) - s["grad"] ** 2) <= 4 * EPS32 * s["grad"] ** 2).all()


def now_of(lr, step):
    return torch.from_numpy(np.frombuffer(np.float64(lr).tobytes() + np.int32(step).tobytes() + b"\0" * 4, np.uint8).copy()).to("cuda")


@pytest.mark.parametrize("eight", [False, True])
def test_step_and_rate_on_the_device(eight):
    """now: the same as the configuration's, up to the device's own 1 - b^t; its step is part of the random bits."""
    t, guards = make(5000, torch.bfloat16, torch.float32, True, eight, 31)
    s = before(t, eight)
    table = sb.adamw_tensors([dict(t, weight_decay=0.1)])
    hyper = dict(HYPER, lr=123.0)
    sb.streambp_adamw_step(sb.adamw_cfg(**hyper, step=999, seed=11, state=int(eight)), table, now=now_of(HYPER["lr"], 3))
    torch.cuda.synchronize()
    check(t, s, 0, 3, eight, 0.1, seed=11)
    check_guards(guards)


@pytest.mark.parametrize("eight", [False, True])
def test_a_captured_step_replays_with_the_step_of_the_moment(eight):
    t, _ = make(5000, torch.bfloat16, torch.float32, False, eight, 41)
    other = {k: x.clone() for k, x in t.items()}
    cfg = sb.adamw_cfg(**HYPER, step=1, seed=5, state=int(eight))
    table, eager = sb.adamw_tensors([t]), sb.adamw_tensors([other])
    now, norm, scale = now_of(HYPER["lr"], 1), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(sb.streambp_grad_norm_workspace_bytes(1), dtype=torch.uint8, device="cuda")

    def both(tab, now):
        sb.streambp_grad_norm(tab, 0.01, norm, scale, ws)
        sb.streambp_adamw_step(cfg, tab, grad_scale=scale, now=now)

    keep = {k: x.clone() for k, x in t.items()}
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both(table, now)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both(table, now)
    torch.cuda.synchronize()
    for k in t:
        t[k].copy_(keep[k])
    for i in range(1, 5):
        g = torch.randn(5000, device="cuda") * 1e-3
        t["grad"].copy_(g)
        other["grad"].copy_(g)
        now.copy_(now_of(HYPER["lr"] / i, i))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        captured = scale.clone()
        both(eager, now_of(HYPER["lr"] / i, i))
        torch.cuda.synchronize()
        assert torch.equal(captured, scale)
        for k in t:
            assert torch.equal(t[k].view(torch.uint8), other[k].view(torch.uint8)), (i, k)


def test_small_updates_of_bf16_weights_arrive_on_average():
    """Updates of a fiftieth of a bf16 step: rounded to nearest none would arrive; after 50 steps of them the mean has moved by one step.  65536 weights, each
    the sum of 50 coin flips of probability 1/50: a mean's standard deviation is sqrt(50 * 0.02 * 0.98) / 256 = 0.004 of a step."""
    p = torch.ones(65536, device="cuda").bfloat16()
    t = dict(sb.new_adamw_states(p), grad=torch.full((65536,), -1.0, device="cuda"))
    table = sb.adamw_tensors([t])
    for i in range(1, 51):      # m / sqrt(v) = -1: the update is lr, upwards; a step of bf16 above 1 is 2^-7
        sb.streambp_adamw_step(sb.adamw_cfg(lr=2.0 ** -7 / 50, beta1=0.9, beta2=0.9, eps=0.0, step=i, seed=77), table)
    moved = (p.double().mean().item() - 1.0) * 128
    assert abs(moved - 1.0) < 0.02


def test_second_moments_of_8_bits_decay_on_average():
    """Gradients of zero: v halves in 68 steps of beta2 = 0.99 although sqrt(v) shrinks by 0.5 % a step, less than half of e4m3's 6 to 12 %."""
    n = 65536
    p = torch.zeros(n, device="cuda")
    t = sb.new_adamw_states(p, state=sb.SBP_STATE_8BIT)
    t["grad"] = torch.ones(n, device="cuda")
    table = sb.adamw_tensors([t])
    step = lambda i: sb.streambp_adamw_step(sb.adamw_cfg(lr=0.0, beta1=0.9, beta2=0.99, step=i, state=sb.SBP_STATE_8BIT, seed=5), table)
    step(1)
    start = np.mean(decoded(t["v"], t["v_scale"]))
    t["grad"].zero_()
    for i in range(2, 70):
        step(i)
    # E sqrt(v): each step rounds without bias; 65536 elements, so the mean is exact to well under 1 %
    assert abs(np.mean(decoded(t["v"], t["v_scale"])) / start / 0.99 ** 34 - 1) < 0.02


def test_a_side_stream():
    made = [make(9000, torch.bfloat16, torch.float32, True, True, 51)[0] for _ in range(2)]
    run([made[0]], True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    sb.streambp_adamw_step(sb.adamw_cfg(**HYPER, step=3, seed=11, state=1), sb.adamw_tensors([dict(made[1], weight_decay=0.1)]), stream=side)
    side.synchronize()
    for k in made[0]:
        assert torch.equal(made[0][k].view(torch.uint8), made[1][k].view(torch.uint8)), k
