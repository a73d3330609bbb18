"""8-bit states where v, or all of a block, lies below fp32's normal range: roots are taken of it all the same, none vanishes, and neighbours in other blocks of the wave keep their bits."""
import numpy as np
import pytest
import torch

from oracle import optim
from paper_2506_03077_amd import binding as sb

from test_gpu_adamw import HYPER, codes, decoded, host, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1e-16, 1e-19, 1e-20, 1e-21])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
def test_second_moments_below_the_normal_range(size, grad_dtype):
    """v = 0.03 g^2, for 1e-20 3e-42: a denormal number of 11 bits, half a unit of which moves its root by 2^-12 of it; a root is stored at most one e4m3 step off, 2^-3 of it, or in
    the fixed-point range, below 2^-6 of the block's scale, 2^-9 of that."""
    n = 5000
    rng = np.random.default_rng(1)
    g = torch.from_numpy((rng.uniform(0.5, 1.0, n) * np.where(rng.random(n) < 0.5, -1, 1) * size).astype(np.float32)).cuda().to(grad_dtype)
    g[::7] = 0
    p = torch.zeros(n, device="cuda")
    t = dict(sb.new_adamw_states(p, sb.SBP_STATE_8BIT), grad=g)
    sb.streambp_adamw_step(sb.adamw_cfg(**HYPER, step=1, state=sb.SBP_STATE_8BIT, seed=3), sb.adamw_tensors([t]))
    torch.cuda.synchronize()
    exact = np.sqrt(1 - HYPER["beta2"]) * np.abs(host(g))
    got = decoded(t["v"], t["v_scale"])
    scale = 2.0 ** optim.per_element(host(t["v_scale"]).astype(np.float64) - 127, n)
    assert (codes(t["v"])[exact > 0] > 0).all() and (codes(t["v"])[exact == 0] == 0).all()
    # v's own rounding: half of 2^-149, relative to v, half through the root; and for the smallest, 1e-21, where v is 5 to 21 units of 2^-149, up to 6 % of the root
    own = exact * np.where(exact > 0, 0.5 * 2.0 ** -149 / np.maximum(exact, 1e-30) ** 2, 0)
    assert (np.abs(got - exact) <= own + 2.0 ** -20 * exact + np.maximum(exact * (1 + 2.0 ** -4) * 2.0 ** -3, scale * 2.0 ** -9)).all()


def test_ordinary_blocks_beside_them_keep_their_bits():
    """Two blocks share a wave: what the small one needs changes nothing for the other."""
    got = []
    for size in (1.0, 1e-17):
        t, _ = make(512, torch.bfloat16, torch.float32, False, True, 5)
        t["grad"][256:] *= size
        if size != 1.0:
            t["v"].view(torch.uint8)[256:] = 0
        sb.streambp_adamw_step(sb.adamw_cfg(**HYPER, step=3, state=sb.SBP_STATE_8BIT, seed=3), sb.adamw_tensors([t]))
        got.append(t)
    for name in ("param", "m", "v"):
        assert torch.equal(got[0][name][:256].view(torch.uint8), got[1][name][:256].view(torch.uint8)), name
