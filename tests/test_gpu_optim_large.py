"""The optimizer step and the norm of calls of more than 2^27 elements, whose loads and stores pass the caches by: the same bits as in a small call, and the norm of all of them."""
import pytest
import torch

from oracle import optim
from paper_2506_03077_amd import binding as sb

from test_gpu_adamw import HYPER, TYPES, before, check, make

pytestmark = pytest.mark.gpu

LARGE = 2 ** 27 + 12345


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,grad_dtype,master", TYPES)
def test_a_large_call_gives_the_bits_of_a_small_one(dtype, grad_dtype, master, eight):
    """A tensor next to a large one, and alone."""
    n = LARGE if eight else 5000
    other = dict(param=torch.zeros(n, dtype=torch.bfloat16, device="cuda"), grad=torch.full((n,), 0.5, dtype=torch.bfloat16, device="cuda"))
    other.update({k: v for k, v in sb.new_adamw_states(other["param"], int(eight)).items() if k != "param"})
    got = []
    for rest in ([], [other]):
        t, _ = make(70001, dtype, grad_dtype, master, eight, 5)
        old = before(t, eight)
        table = sb.adamw_tensors([dict(t, weight_decay=0.1)] + rest)
        sb.streambp_adamw_step(sb.adamw_cfg(**HYPER, step=3, seed=11, state=int(eight), zero_grads=True), table)
        torch.cuda.synchronize()
        assert not bool(t["grad"].any())
        t["grad"] = torch.empty(0, device="cuda")
        got.append(t)
    check(got[1], old, 0, 3, eight, 0.1, seed=11)
    assert all(torch.equal(got[0][k].view(torch.uint8), got[1][k].view(torch.uint8)) for k in got[0])
    # every element of the large one: m = 0.1 g, v = 0.03 g^2, so 0.01 (0.1 / (1 - 0.9^3)) / sqrt(0.03 / (1 - 0.97^3)) = 0.0063 of a step, to one of its two neighbours in
    # bf16 (2^-15 apart there), and its gradient is cleared
    want = optim.step(0.0, 0.0, 0.0, 0.5, 3, **HYPER, weight_decay=0.0)[0]
    low, high = float(other["param"].min()), float(other["param"].max())
    assert want - 2.0 ** -15 < low and high < want + 2.0 ** -15 and not bool(other["grad"].any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm(dtype):
    gen = torch.Generator("cuda").manual_seed(3)
    grads = [torch.randn(n, generator=gen, device="cuda").to(dtype) for n in (LARGE, 77)]
    want = float(torch.sqrt(sum((x.double() ** 2).sum() for g in grads for x in g.split(2 ** 24))))
    norm, factor = sb.streambp_grad_norm(sb.adamw_tensors([dict(grad=g) for g in grads]), want / 2)
    # squares and sums of eight in fp32, half of their relative error through the root, and the result's rounding; the factor three roundings more
    assert abs(norm.item() - want) <= 5 * 2.0 ** -24 * want and abs(factor.item() - 0.5) <= 8 * 2.0 ** -24


@pytest.mark.parametrize("eight", [True, False])
def test_elements_past_32_bits(eight, monkeypatch):
    """A bf16 tensor of more than 2^32 elements: its last ones are found, and have random words of their own (the high half of the index is part of the key)."""
    first, n = 2 ** 32 + 512, 2 ** 32 + 512 + 5000
    if torch.cuda.mem_get_info()[0] < 64e9:
        pytest.skip("26 GB, 52 with 32-bit states")
    small, _ = make(5000, torch.bfloat16, torch.bfloat16, False, eight, 7)
    old = before(small, eight)
    t = dict(param=torch.zeros(n, dtype=torch.bfloat16, device="cuda"), grad=torch.zeros(n, dtype=torch.bfloat16, device="cuda"))
    t.update({k: v for k, v in sb.new_adamw_states(t["param"], int(eight)).items() if k != "param"})
    for k in t:
        at = first // 256 if k.endswith("scale") else first
        t[k][at:at + len(small[k])].view(torch.uint8).copy_(small[k].view(torch.uint8))
    norm, _ = sb.streambp_grad_norm(sb.adamw_tensors([dict(grad=t["grad"])]))
    want = float(small["grad"].double().norm())
    assert abs(norm.item() - want) <= 5 * 2.0 ** -24 * want
    sb.streambp_adamw_step(sb.adamw_cfg(**HYPER, step=3, seed=11, state=int(eight)), sb.adamw_tensors([dict(t, weight_decay=0.1)]))
    torch.cuda.synchronize()
    words = optim.random_bits
    monkeypatch.setattr(optim, "random_bits", lambda seed, step, tensor, k: words(seed, step, tensor, k, first=first))
    last = {k: (x[first // 256:] if k.endswith("scale") else x[first:]).clone() for k, x in t.items()}
    check(last, old, 0, 3, eight, 0.1, seed=11)
    assert not any(bool(x.any()) for x in t["param"][:first].split(2 ** 28))
