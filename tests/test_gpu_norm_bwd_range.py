"""The norm's backward pass where a row's mean or what is beside it reaches the end of fp32.

Tolerances are those of test_gpu_norm.py; what is written below the normal numbers is off by 2^-134 at most (bf16) whatever its size, and
an intermediate number of fp32 by 2^-150, which rstd, the weight and the other factors show at most 2^30 times in these inputs.
"""
import pytest
import torch

from test_gpu_norm import DEV, check, grad64, inputs, run_backward, run_forward

pytestmark = pytest.mark.gpu

LARGEST = torch.finfo(torch.bfloat16).max
WIDTHS = [3, 100, 500, 1000, 1004, 2050, 4104, 5000, 8200, 16385, 20000, 40001]


def check_backward(gy, x, w, mean, rstd, rms):
    grads = run_backward(gy, x, w, mean, rstd, rms)
    for name, (value, tol) in grad64(gy, x, w, mean, rstd, rms).items():
        check(grads[name], (value, tol + 2.0 ** -119), name)


@pytest.mark.parametrize("D", WIDTHS)
def test_large_means_beside_a_small_eps(D):
    """Equal values: nothing is left of the row, and its mean times 1 / sqrt(eps) is beyond fp32.  Threads that lie behind the row's end
    have a part in no sum."""
    T = 5
    _, w, b, gy = inputs(T, D)
    x = torch.tensor([2.0 ** 121, -2.0 ** 126, LARGEST, 1.0, 2.0 ** 100], device=DEV).to(torch.bfloat16)[:, None].repeat(1, D)
    for eps in (2.0 ** -17, 2.0 ** -60):
        rstd = torch.full((T,), eps ** -0.5, device=DEV)
        check_backward(gy, x, w, x[:, 0].float().contiguous(), rstd, False)


@pytest.mark.parametrize("D", WIDTHS)
def test_differences_beyond_fp32(D):
    """The largest number but for one of the other sign, with the statistics that the forward pass leaves."""
    x, w, b, gy = inputs(4, D)
    x.fill_(LARGEST)
    x[1:3] *= -1
    x[:2, D // 2] *= -1
    x[3, 0] = 2.0 ** 119
    got = run_forward(x, w, b, 2.0 ** -20, False)
    rstd = got["rstd"].clone()
    rstd[2] = 2.0 ** 10
    check_backward(gy, x, w, got["mean"], rstd, False)


@pytest.mark.parametrize("e", [-100, -60, 0, 60, 110, 118, 119, 120, 126])
@pytest.mark.parametrize("D", [100, 1004, 20000])
def test_means_of_every_size(D, e):
    x, w, b, gy = inputs(6, D)
    x.copy_(((1 + 0.1 * x.double().clamp(-4, 4)) * 2.0 ** e).clamp(-LARGEST, LARGEST))
    got = run_forward(x, w, b, 0.0, False)
    # (the gradients of a row as large as its rstd is small, so that neither leaves the numbers there are)
    gy.mul_(2.0 ** (e // 2))
    check_backward(gy, x, w, got["mean"], got["rstd"], False)
