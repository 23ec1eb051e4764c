"""The norm over the whole range of bf16: rows whose squares, sums or differences lie beyond what fp32 holds, and no eps to hide them.

Tolerances are those of test_gpu_norm.py, and below the normal numbers: a number written or an intermediate one is off by 2^-150 at
most in fp32 and 2^-134 in bf16 whatever its size.  A row whose variance and eps are 2^-100 and more together is summed as it is, its
mean off by that 2^-150, which y shows rstd <= 2^50 times; of another one the row's power of two is taken out first, which is exact.
"""
import pytest
import torch

import paper_2605_05940_amd as npd
from test_gpu_norm import DEV, check, grad64, norm64, run_backward, run_forward

pytestmark = pytest.mark.gpu

TINY, TINY_BF16 = 2.0 ** -149, 2.0 ** -133
LARGEST = torch.finfo(torch.bfloat16).max
WIDTHS = [3, 100, 1000, 2048, 2050, 4096, 8192, 8200, 16384, 20001, 32768, 65536]
EXPONENTS = [-132, -126, -110, -80, -75, -64, -60, -51, -49, -30, 0, 40, 58, 63, 64, 90, 110, 120, 126, 127]


def rows(D, seed=0, exponents=EXPONENTS):
    """A row of every size: numbers around 2^e of both signs, in another half of them all of one."""
    g = torch.Generator(device=DEV).manual_seed(seed + D)
    v = torch.randn((2 * len(exponents), D), device=DEV, generator=g, dtype=torch.float64)
    v[::2] = 1 + 0.1 * v[::2]
    scale = torch.tensor([2.0 ** e for e in exponents], device=DEV, dtype=torch.float64).repeat_interleave(2)
    return (v * scale[:, None]).clamp(-LARGEST, LARGEST).to(torch.bfloat16)


def parameters(D, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + D)
    return [(1 + 0.3 * torch.randn(D, device=DEV, generator=g)).to(torch.bfloat16), torch.randn(D, device=DEV, generator=g).to(torch.bfloat16)]


def check_forward(x, w, b, eps, rms):
    got, want = run_forward(x, w, b, eps, rms), norm64(x, w, b, eps, rms)
    (y, y_tol), (rstd, rstd_tol) = want["y"], want["rstd"]
    none = rstd.isinf()  # rows of equal values, and no eps: the definition has 0 / 0 for them
    assert bool(got["y"][none].isnan().all()) and bool(got["rstd"][none].isinf().all())
    if bool(none.any()):
        assert eps == 0 and bool((x[none] == x[none][:, :1]).all())
        if bool(none.all()):
            return got
        return check_forward(x[~none], w, b, eps, rms)
    check(got["y"], (y, y_tol + w.double().abs() * TINY * rstd.clamp(max=2.0 ** 51)[:, None] + TINY_BF16), "y")
    if not rms:
        check(got["mean"], (want["mean"][0], want["mean"][1] + TINY), "mean")
    largest = torch.finfo(torch.float32).max
    inside = rstd + rstd_tol <= largest  # (a number beyond fp32 is inf; about the border it may be either)
    check(got["rstd"][inside], (rstd[inside], rstd_tol[inside] + TINY), "rstd")
    assert bool(got["rstd"][rstd - rstd_tol > 2 * largest].isinf().all())
    return got


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -126, 2.0 ** -40, 2.0 ** 100])
@pytest.mark.parametrize("D", WIDTHS)
def test_rows_of_every_size(D, eps, rms):
    check_forward(rows(D), *parameters(D), eps, rms)


@pytest.mark.parametrize("D", WIDTHS)
def test_equal_values_whose_sum_is_beyond_fp32(D):
    values = torch.tensor([LARGEST, -LARGEST, 2.0 ** 112, 2.0 ** -133, -3 * 2.0 ** -126], device=DEV).to(torch.bfloat16)
    w, b = parameters(D)
    got = run_forward(values[:, None].repeat(1, D), w, b, 2.0 ** -20, False)
    assert torch.equal(got["mean"], values.float())
    assert torch.equal(got["y"], b.expand(5, D))
    assert bool((got["rstd"] == 2.0 ** 10).all())


@pytest.mark.parametrize("D", WIDTHS)
def test_differences_beyond_fp32(D):
    """The largest number but for one of the other sign: twice the largest number lies between them."""
    x = torch.full((2, D), LARGEST, dtype=torch.bfloat16, device=DEV)
    x[:, D // 2] = -LARGEST
    x[1] *= -1
    w, b = parameters(D)
    check_forward(x, w, b, 1e-6, False)


@pytest.mark.parametrize("D", [100, 2048, 4096, 20000])
def test_one_value_that_stands_out(D):
    """Squares of the others vanish beside its own, at either end of the range."""
    x = torch.zeros((4, D), dtype=torch.bfloat16, device=DEV)
    x[:, 1::3] = torch.tensor([1e-38, 1e-30, 1e20, 2.0 ** -133], device=DEV)[:, None].to(torch.bfloat16)
    x[:, D - 1] = torch.tensor([1e-20, LARGEST, -LARGEST, 1e-38], device=DEV).to(torch.bfloat16)
    for rms in (False, True):
        check_forward(x, *parameters(D), 0.0, rms)


def test_rows_beside_others_are_as_they_are_alone():
    x = rows(1000)
    w, b = parameters(1000)
    got = run_forward(x, w, b, 0.0, False)
    for r in range(0, len(x), 7):
        alone = run_forward(x[r:r + 1], w, b, 0.0, False)
        assert torch.equal(alone["y"][0], got["y"][r]) and torch.equal(alone["rstd"][0], got["rstd"][r])


@pytest.mark.parametrize("T,D", [(600000, 8), (17000000, 8), (70000, 2500)])
def test_rows_that_threads_have_one_after_the_other(T, D):
    g = torch.Generator(device=DEV).manual_seed(T)
    x = torch.empty((T, D), dtype=torch.bfloat16, device=DEV)
    x.random_(-8, 9, generator=g)
    at = torch.cat([torch.tensor([0, 1, T - 1], device=DEV), torch.randint(0, T, (500,), device=DEV, generator=g)])
    x[at[::2]] = (x[at[::2]].float() * 2.0 ** -100).to(torch.bfloat16)
    x[at[1::2]] = (x[at[1::2]].float() * 2.0 ** 100).to(torch.bfloat16)
    w, b = parameters(D)
    y, mean, rstd = torch.empty_like(x), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    npd.npd_layer_norm(x, w, bias=b, eps=0.0, y_out=y, mean_out=mean, rstd_out=rstd)
    some = torch.unique(torch.cat([at, at + 1, torch.arange(0, T, T // 1000, device=DEV)]).clamp(max=T - 1))
    check_forward(x[some], w, b, 0.0, False)
    got = run_forward(x[some], w, b, 0.0, False)
    assert torch.equal(y[some].view(torch.int16), got["y"].contiguous().view(torch.int16))
    assert torch.equal(mean[some], got["mean"]) and torch.equal(rstd[some], got["rstd"])


def test_rows_with_nan_or_infinities_as_ever():
    x = rows(500)
    clean = run_forward(x, None, None, 0.0, False)
    for value in (float("nan"), float("inf"), float("-inf")):
        y = x.clone()
        y[::4, 3] = value
        got = run_forward(y, None, None, 0.0, False)
        others = torch.arange(len(x), device=DEV) % 4 != 0
        assert torch.equal(got["y"][others], clean["y"][others]) and bool(got["y"][::4].isnan().all())
        got = run_forward(y, None, None, 0.0, True)
        assert bool(got["y"][::4, 3].isnan().all())


def test_captured_and_replayed():
    D = 3000
    sets = [rows(D, seed=s) for s in range(2)]
    w, b = parameters(D)
    x, y, rstd = sets[0].clone(), torch.empty_like(sets[0]), torch.empty(len(sets[0]), device=DEV)

    def call():
        npd.npd_layer_norm(x, w, bias=b, eps=0.0, y_out=y, rstd_out=rstd)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for s in (1, 0, 1):
        x.copy_(sets[s])
        graph.replay()
        want = run_forward(sets[s], w, b, 0.0, False)
        torch.cuda.synchronize()
        assert torch.equal(y, want["y"]) and torch.equal(rstd, want["rstd"])
