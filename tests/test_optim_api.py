"""The optimizer step's entry points on the CPU: what they refuse, before anything is launched, and the random bits and 8-bit format of the oracle."""
import ctypes as C

import numpy as np
import pytest

from oracle import optim
from paper_2506_03077_amd import binding as sb

P = 4096      # a pointer that is never read: every check comes before the first launch


def cfg(**more):
    d = dict(lr=1e-3, step=1)
    d.update(more)
    return sb.adamw_cfg(**d)


def tensor(**more):
    d = dict(n=10, dtype=sb.SBP_BF16, grad_dtype=sb.SBP_F32, weight_decay=0.1, param=P, master=None, grad=P, m=P, v=P, m_scale=None, v_scale=None)
    d.update(more)
    return d


def call(c, tensors, grad_scale=None, now=None):
    table = (sb.AdamwTensor * max(1, len(tensors)))(*[sb.AdamwTensor(**t) for t in tensors])
    return sb.lib().streambp_adamw_step(None if c is None else C.byref(c), len(tensors), table, grad_scale, now, None)


NULL, SHAPE, UNSUPPORTED, WORKSPACE = -1, -2, -3, -4


@pytest.mark.parametrize("rc,c,t", [
    (NULL, None, {}), (UNSUPPORTED, cfg(state=2), {}), (SHAPE, cfg(step=0), {}), (SHAPE, cfg(lr=-1.0), {}), (SHAPE, cfg(lr=float("nan")), {}),
    (SHAPE, cfg(lr=float("inf")), {}), (SHAPE, cfg(beta1=1.0), {}), (SHAPE, cfg(beta2=-0.1), {}), (SHAPE, cfg(beta2=float("nan")), {}),
    (SHAPE, cfg(eps=-1e-8), {}), (SHAPE, cfg(eps=float("inf")), {}), (SHAPE, cfg(zero_grads=2), {}),
    (SHAPE, cfg(), dict(n=-1)), (SHAPE, cfg(), dict(n=2 ** 34 + 1)), (SHAPE, cfg(), dict(weight_decay=-0.1)), (SHAPE, cfg(), dict(weight_decay=float("nan"))),
    (UNSUPPORTED, cfg(), dict(dtype=2)), (UNSUPPORTED, cfg(), dict(grad_dtype=7)), (UNSUPPORTED, cfg(), dict(dtype=sb.SBP_F32, master=P)),
    (NULL, cfg(), dict(param=None)), (NULL, cfg(), dict(grad=None)), (NULL, cfg(), dict(m=None)), (NULL, cfg(), dict(v=None)),
    (NULL, cfg(state=1), {}), (NULL, cfg(state=1), dict(m_scale=P)), (UNSUPPORTED, cfg(), dict(m_scale=P, v_scale=P)),
    (UNSUPPORTED, cfg(), dict(param=P + 1)), (UNSUPPORTED, cfg(), dict(master=P + 2)), (UNSUPPORTED, cfg(), dict(grad=P + 2)), (UNSUPPORTED, cfg(), dict(m=P + 1)),
    (UNSUPPORTED, cfg(), dict(v=P + 2)),
])
def test_adamw_refuses(rc, c, t):
    assert call(c, [tensor(), tensor(**t)] if c is not None else [tensor()]) == rc
    assert sb.streambp_last_error()


def test_adamw_refuses_odd_scalars_and_counts():
    assert call(cfg(), [tensor()], grad_scale=P + 1) == UNSUPPORTED
    assert call(cfg(), [tensor()], now=P + 4) == UNSUPPORTED
    assert sb.lib().streambp_adamw_step(C.byref(cfg()), -1, None, None, None, None) == SHAPE
    assert sb.lib().streambp_adamw_step(C.byref(cfg()), 1, None, None, None, None) == NULL


def test_nothing_to_do_is_no_error():
    assert call(cfg(), []) == 0
    empty = dict(n=0, dtype=9, grad_dtype=9, param=None, grad=None, m=None, v=None)      # pointers and types of no elements are not looked at
    assert call(cfg(), [tensor(**empty)]) == 0
    assert call(cfg(step=0, lr=-1.0), [tensor(**empty)], now=P) == 0                     # with `now` these two are not looked at


def test_grad_norm_refuses():
    table = (sb.AdamwTensor * 1)(sb.AdamwTensor(n=5, grad_dtype=0, grad=P))
    f = sb.lib().streambp_grad_norm
    need = sb.streambp_grad_norm_workspace_bytes(1)
    assert need > 0 and need % 256 == 0 and sb.streambp_grad_norm_workspace_bytes(-1) == 0
    assert f(1, table, 1.0, P, P, P, need - 1, None) == WORKSPACE
    assert f(1, table, 1.0, P, P, P + 16, need, None) == WORKSPACE
    assert f(1, table, -1.0, P, P, P, need, None) == SHAPE
    assert f(1, table, float("nan"), P, P, P, need, None) == SHAPE
    assert f(1, table, 1.0, None, P, P, need, None) == NULL
    assert f(1, table, 1.0, P, P, None, need, None) == NULL
    assert f(1, table, 1.0, P + 2, P, P, need, None) == UNSUPPORTED
    assert f(1, None, 1.0, P, P, P, need, None) == NULL
    assert f(-1, table, 1.0, P, P, P, need, None) == SHAPE
    table[0].grad = None
    assert f(1, table, 1.0, P, P, P, need, None) == NULL
    table[0].grad, table[0].grad_dtype = P, 5
    assert f(1, table, 1.0, P, P, P, need, None) == UNSUPPORTED


def test_random_bits_round_like_independent_ones():
    """What rounding needs of the words: the three fields that are used are uniform, and errors of neighbours, of other steps, tensors and seeds do not add up.  Two
    multiplications leave correlations of up to one per cent between the bits of some neighbours, which is nothing to that: the
    variance of the sum of k neighbours' errors is 1 + 2 sum of the correlations times that of independent ones, tested to a quarter.  n = 2^20 words: of 2^20 / 256
    sums the variance is known to sqrt(2 / 4096) = 2.2 %, a mean to 0.29 / 1024 (5 of them: 0.0015), a correlation to 1 / 1024."""
    n = 1 << 20
    fields = [(12, 0xfffff), (0, 0xfffff), (0, 0xffff)]
    calls = ((0, 1, 0), (0, 2, 0), (0, 1, 1), (1, 1, 0))
    errors = [[((optim.random_bits(*c, n) >> np.uint64(shift)) & np.uint64(mask)) / (mask + 1.0) - 0.5 for c in calls] for shift, mask in fields]
    for of_field in errors:
        for x in of_field:
            assert abs(x.mean()) < 0.0015
            counts = np.bincount(((x + 0.5) * 256).astype(int), minlength=256)
            assert np.abs(counts / (n / 256) - 1).max() < 0.1                      # 4096 each: a standard deviation is 1/64
            for k in (2, 8, 64, 256):
                assert abs(x.reshape(-1, k).sum(1).var() * 12 / k - 1) < 0.25
        for other in of_field[1:]:
            assert abs(np.corrcoef(of_field[0], other)[0, 1]) < 0.02


def test_stochastic_rounding_of_the_oracle_is_right_on_average():
    """The mean of 4096 roundings of a value: off by at most 5 standard deviations, each at most half a step."""
    u = (optim.random_bits(3, 7, 0, 4096) & np.uint64(0xfffff)) / 2.0 ** 20
    for x in (130.0, 100.3, 1.07, 0.013, 0.0021, 0.0005):
        code, _ = optim.quantize(np.full(4096, x), np.zeros(16, int), u)
        low = np.searchsorted(optim.GRID, x, side="right") - 1
        gap = optim.GRID[low + 1] - optim.GRID[low]
        assert abs(optim.GRID[code].mean() - x) <= 5 * gap / 2 / 64
        assert set(code) <= {low, low + 1}


def test_the_grid_is_e4m3():
    import torch
    grid = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(grid, optim.GRID)
