"""Layer norm and its backward pass against 64 bits.

Tolerances, from the arithmetic alone: B = 2^-8 is the largest relative error of a rounding to bf16, u = 2^-24 of one to fp32.

  mean    a thread adds up to 64 values, a wave and a workgroup 6 + 16 more: fewer than K = 100 dependent roundings on sums of at
          most sum |x|, then the division by D:  dm = (K + 2) u sum |x| / D
  var     every difference is off by dm and a rounding, squares and their sum by K more:
          dv = 2 (dm + u |mean|) sum |d| / D + (K + 6) u var + dm^2
  rstd    relative: dr = dv / (2 (var + eps)) + 4 u  (sum with eps, root, reciprocal)
  y       |w| (dm rstd + |n| (dr + 3 u)) + u |b| + B |y|
  grad_x  n is off by 3 u |n| (difference, product), a = g w by u |a|; their means by (K + 6) u of the means of magnitudes (ma, man);
          rstd (6 u (|a| + |n| man + ma) + (K + 6) u (|n| man + ma)) + B |dx|
  grad_weight, grad_bias   a thread adds at most T / (rows side by side) of them, then up to 32 pieces and 16 + 4 sums: fewer than
          min(T, T / 512 + 8) + 64 roundings on sum |g n|, each term off by 4 u:  B |dw| on top
"""
import pytest
import torch

import paper_2605_05940_amd as npd

pytestmark = pytest.mark.gpu

B, U, K = 2.0 ** -8, 2.0 ** -24, 100
DEV = "cuda:0"


def matrix(T, D, g, pad=0, offset=0):
    """A bf16 matrix with a row stride of D + pad that begins `offset` values into its memory, filled with 7 around it."""
    whole = torch.full((T * (D + pad) + offset + 8,), 7.0, dtype=torch.bfloat16, device=DEV)
    view = whole[offset:offset + T * (D + pad)].view(T, D + pad)[:, :D]
    view.copy_(torch.randn((T, D), device=DEV, generator=g))
    return view, whole


def inputs(T, D, seed=0, pad=0, offset=0, weight=True, bias=True):
    g = torch.Generator(device=DEV).manual_seed(1000 * seed + 31 * T + D)
    x, _ = matrix(T, D, g, pad, offset)
    x.mul_(torch.exp(torch.randn((T, 1), device=DEV, generator=g))).add_(0.5)
    w = (1 + 0.3 * torch.randn(D, device=DEV, generator=g)).to(torch.bfloat16) if weight else None
    b = torch.randn(D, device=DEV, generator=g).to(torch.bfloat16) if bias else None
    gy, _ = matrix(T, D, g, pad, offset)
    return x, w, b, gy


def norm64(x, w, b, eps, rms):
    x = x.double()
    T, D = x.shape
    one, none = torch.ones(D, device=DEV).double(), torch.zeros(D, device=DEV).double()
    w, b = one if w is None else w.double(), none if b is None else b.double()
    mean = torch.zeros(T, device=DEV).double() if rms else x.mean(1)
    d = x - mean[:, None]
    var = (d * d).mean(1)
    rstd = 1 / torch.sqrt(var + eps)
    y = d * rstd[:, None] * w + b
    dm = torch.zeros_like(mean) if rms else (K + 2) * U * x.abs().mean(1)
    dv = 2 * (dm + U * mean.abs()) * d.abs().mean(1) + (K + 6) * U * var + dm * dm
    dr = dv / (2 * (var + eps)) + 4 * U
    n = (d * rstd[:, None]).abs()
    tol = w.abs() * ((dm * rstd)[:, None] + n * (dr + 3 * U)[:, None]) + U * b.abs() + B * y.abs()
    return {"mean": (mean, dm + U * mean.abs()), "rstd": (rstd, dr * rstd), "y": (y, tol)}


def grad64(gy, x, w, mean, rstd, rms):
    g, x, rstd = gy.double(), x.double(), rstd.double()[:, None]
    T, D = x.shape
    w = torch.ones(D, device=DEV).double() if w is None else w.double()
    n = (x - (0 if rms else mean.double()[:, None])) * rstd
    a = g * w
    along, flat = (a * n).mean(1, keepdim=True), 0 if rms else a.mean(1, keepdim=True)
    dx = rstd * (a - flat - n * along)
    ma, man = (a.abs().mean(1, keepdim=True) * (0 if rms else 1)), (a * n).abs().mean(1, keepdim=True)
    tol = rstd * (6 * U * (a.abs() + n.abs() * man + ma) + (K + 6) * U * (n.abs() * man + ma)) + B * dx.abs()
    terms = min(T, T / 512 + 8) + 68
    out = {"grad_x": (dx, tol)}
    for name, v in (("grad_weight", g * n), ("grad_bias", g)):
        out[name] = (v.sum(0), terms * U * v.abs().sum(0) + B * v.sum(0).abs())
    return out


def check(got, want, name):
    value, tol = want
    off = (got.double() - value).abs()
    assert bool((off <= tol + 1e-300).all()), (name, float((off / (tol + 1e-300)).max()))


def run_forward(x, w, b, eps, rms, pad=0):
    T, D = x.shape
    whole = torch.full((T, D + pad), 3.0, dtype=torch.bfloat16, device=DEV)
    mean, rstd = None if rms else torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    npd.npd_layer_norm(x, w, bias=b, eps=eps, rms=rms, y_out=whole[:, :D], mean_out=mean, rstd_out=rstd)
    assert bool((whole[:, D:] == 3.0).all())
    return {"y": whole[:, :D], "mean": mean, "rstd": rstd}


def run_backward(gy, x, w, mean, rstd, rms, pad=0, **more):
    T, D = x.shape
    whole = torch.full((T, D + pad), 3.0, dtype=torch.bfloat16, device=DEV)
    out = dict(grad_x=whole[:, :D], grad_weight=torch.empty(D, dtype=torch.bfloat16, device=DEV),
               grad_bias=torch.empty(D, dtype=torch.bfloat16, device=DEV))
    npd.npd_layer_norm_bwd(gy, x, w, mean=mean, rstd=rstd, rms=rms, **out, **more)
    assert bool((whole[:, D:] == 3.0).all())
    return out


SIZES = [(1, 1), (3, 7), (5, 8), (130, 64), (9, 100), (6, 512), (7, 513), (40, 1000), (33, 1024), (5, 1025), (300, 2048), (5, 2050),
         (17, 4096), (3, 4097), (4, 8191), (3, 8192), (3, 8195), (5, 16384), (6, 16385), (2, 32768), (3, 40001), (2, 65536), (2500, 72),
         (700, 3001)]


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("T,D", SIZES)
def test_against_64_bits(T, D, rms):
    pad, offset = (0, 0) if (T + D) % 2 else (5, 3)  # (aligned rows and rows that begin anywhere)
    x, w, b, gy = inputs(T, D, pad=pad, offset=offset)
    eps = 1e-5
    got = run_forward(x, w, b, eps, rms, pad)
    for name, want in norm64(x, w, b, eps, rms).items():
        if got[name] is not None:
            check(got[name], want, name)
    grads = run_backward(gy, x, w, got["mean"], got["rstd"], rms, pad)
    for name, want in grad64(gy, x, w, got["mean"], got["rstd"], rms).items():
        check(grads[name], want, name)


@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_without_parameters(weight, bias):
    x, w, b, gy = inputs(20, 300, weight=weight, bias=bias)
    got = run_forward(x, w, b, 1e-6, False)
    check(got["y"], norm64(x, w, b, 1e-6, False)["y"], "y")
    grads = run_backward(gy, x, w, got["mean"], got["rstd"], False)
    for name, want in grad64(gy, x, w, got["mean"], got["rstd"], False).items():
        check(grads[name], want, name)


@pytest.mark.parametrize("D", [200, 1024, 4096, 20000])
@pytest.mark.parametrize("which", ["grad_x", "grad_weight", "grad_bias"])
def test_one_gradient_alone_is_the_same(D, which):
    x, w, b, gy = inputs(50, D)
    got = run_forward(x, w, b, 1e-5, False)
    every = run_backward(gy, x, w, got["mean"], got["rstd"], False)
    alone = torch.empty_like(every[which])
    npd.npd_layer_norm_bwd(gy, x, w, mean=got["mean"], rstd=got["rstd"], **{which: alone})
    assert torch.equal(alone, every[which])


@pytest.mark.parametrize("D", [96, 2048, 17000])
def test_accumulate(D):
    x, w, b, gy = inputs(600, D)
    got = run_forward(x, w, b, 1e-5, True)
    want = grad64(gy, x, w, None, got["rstd"], True)
    g = torch.Generator(device=DEV).manual_seed(5)
    start = {n: torch.randn(D, device=DEV, generator=g).to(torch.bfloat16) for n in ("grad_weight", "grad_bias")}
    out = {n: v.clone() for n, v in start.items()}
    npd.npd_layer_norm_bwd(gy, x, w, rstd=got["rstd"], rms=True, accumulate=True, **out)
    for n, v in out.items():
        value, tol = want[n]
        total = value + start[n].double()
        check(v, (total, tol - B * value.abs() + U * total.abs() + B * total.abs()), n)


def test_gradients_against_differences():
    """The backward pass against central differences of the 64-bit forward pass: (f(x + h d) - f(x - h d)) / 2 h is off by a third
    derivative times h^2, far below the tolerance of the gradient's own rounding."""
    T, D, eps = 4, 40, 1e-3
    for rms in (False, True):
        x, w, b, gy = inputs(T, D)
        got = run_forward(x, w, b, eps, rms)
        grads = run_backward(gy, x, w, got["mean"], got["rstd"], rms)
        g = torch.Generator(device=DEV).manual_seed(2)
        h = 1e-5
        for name, at in (("grad_x", x), ("grad_weight", w), ("grad_bias", b)):
            d = torch.randn(at.shape, device=DEV, generator=g).double()

            def loss(step):
                args = {"grad_x": x, "grad_weight": w, "grad_bias": b}
                args = {n: v.double() + (step * d if n == name else 0) for n, v in args.items()}
                return (norm64(args["grad_x"], args["grad_weight"], args["grad_bias"], eps, rms)["y"][0] * gy.double()).sum()

            slope = float((loss(h) - loss(-h)) / (2 * h))
            # each entry of a gradient is off by B of itself and by what statistics in fp32 change (2^-16 of its terms)
            mine = grads[name].double() * d
            size = float((gy.double().abs().sum() * 8) * d.abs().max())
            assert abs(float(mine.sum()) - slope) <= B * float(mine.abs().sum()) + 2.0 ** -16 * size + 1e-8 * size


def test_rows_of_equal_values_and_of_zeros():
    x = torch.full((3, 100), 2.5, dtype=torch.bfloat16, device=DEV)
    x[1] = 0
    x[2] = -1000
    w, b = torch.ones(100, dtype=torch.bfloat16, device=DEV), torch.full((100,), 0.5, dtype=torch.bfloat16, device=DEV)
    got = run_forward(x, w, b, 1e-5, False)
    for name, want in norm64(x, w, b, 1e-5, False).items():
        check(got[name], want, name)


@pytest.mark.parametrize("D", [1, 3, 49, 100, 999, 1000, 2047, 2048, 5001, 8191, 20001, 32767, 65535, 65536])
def test_rows_of_equal_values_have_their_mean_exactly(D):
    """Their sums are whole multiples (16 bits) of 8 bits, exact in fp32: the mean is the value, and nothing is left of the row but the
    bias, however large the value is beside eps."""
    values = torch.tensor([2.5, -1000.0, 1.0078125, 30208.0, -3e30, 1e-30, 255.0, -0.3340], device=DEV).to(torch.bfloat16)
    x = values[:, None].repeat(1, D)
    w, b = torch.full((D,), 1.5, dtype=torch.bfloat16, device=DEV), torch.randn(D, device=DEV).to(torch.bfloat16)
    got = run_forward(x, w, b, 1e-5, False)
    assert torch.equal(got["mean"], values.float())
    assert torch.equal(got["y"], b.expand_as(x))
    check(got["rstd"], norm64(x, w, b, 1e-5, False)["rstd"], "rstd")
    got = run_forward(x, w, b, 0.0, False)
    assert bool(got["rstd"].isinf().all()) and bool(got["y"].isnan().all())


def test_a_row_that_is_not_finite_keeps_to_itself():
    x, w, b, gy = inputs(9, 500)
    clean = run_forward(x, w, b, 1e-5, False)
    grads = run_backward(gy, x, w, clean["mean"], clean["rstd"], False)
    for bad in (float("nan"), float("inf")):
        y = x.clone()
        y[4, 17] = bad
        got = run_forward(y, w, b, 1e-5, False)
        others = torch.arange(9, device=DEV) != 4
        assert torch.equal(got["y"][others], clean["y"][others]) and bool(got["y"][4].isnan().any())
        dx = run_backward(gy, y, w, got["mean"], got["rstd"], False)["grad_x"]
        assert torch.equal(dx[others], grads["grad_x"][others])


def test_captured_and_replayed_beside_eager_calls():
    """A captured forward and backward pass with workspaces of their own, replayed with other inputs and eager calls between."""
    T, D = 700, 1000
    sets = [inputs(T, D, seed=s) for s in range(3)]
    x, w, b, gy = (t.clone() for t in sets[0])
    y, mean, rstd = torch.empty_like(x), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    out = dict(grad_x=torch.empty_like(x), grad_weight=torch.empty_like(w), grad_bias=torch.empty_like(w))
    ws = torch.empty(npd.npd_layer_norm_workspace_bytes(T, D, grad_bias=True), dtype=torch.uint8, device=DEV)

    def call():
        npd.npd_layer_norm(x, w, bias=b, y_out=y, mean_out=mean, rstd_out=rstd)
        npd.npd_layer_norm_bwd(gy, x, w, mean=mean, rstd=rstd, workspace=ws, **out)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for s in (1, 2, 0, 1):
        for to, of in zip((x, w, b, gy), sets[s]):
            to.copy_(of)
        graph.replay()
        got = run_forward(*sets[s][:3], 1e-5, False)
        grads = run_backward(sets[s][3], *sets[s][:2], got["mean"], got["rstd"], False)
        torch.cuda.synchronize()
        assert torch.equal(y, got["y"]) and torch.equal(mean, got["mean"]) and torch.equal(rstd, got["rstd"])
        for n, v in out.items():
            assert torch.equal(v, grads[n]), n


def test_two_streams_at_once():
    T, D = 900, 2048
    sets = [inputs(T, D, seed=s) for s in range(2)]
    want = []
    for x, w, b, gy in sets:
        f = run_forward(x, w, b, 1e-5, False)
        want.append((f, run_backward(gy, x, w, f["mean"], f["rstd"], False)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[] for _ in sets]
    for _ in range(4):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                x, w, b, gy = sets[i]
                f = run_forward(x, w, b, 1e-5, False)
                got[i].append((f, run_backward(gy, x, w, f["mean"], f["rstd"], False)))
    torch.cuda.synchronize()
    for i in range(2):
        for f, g in got[i]:
            assert torch.equal(f["y"], want[i][0]["y"])
            for n in g:
                assert torch.equal(g[n], want[i][1][n])


def test_offsets_beyond_32_bits():
    """Rows whose elements lie more than 2^31 apart from the first."""
    T, D, stride = 3, 1000, (1 << 30) + 9
    memory = torch.empty(2 * stride + D, dtype=torch.bfloat16, device=DEV)
    x, w, b, gy = inputs(T, D)
    far = torch.as_strided(memory, (T, D), (stride, 1))
    far.copy_(x)
    got, want = run_forward(far, w, b, 1e-5, False), run_forward(x, w, b, 1e-5, False)
    assert torch.equal(got["y"], want["y"])
    a = run_backward(gy, far, w, got["mean"], got["rstd"], False)
    c = run_backward(gy, x, w, got["mean"], got["rstd"], False)
    assert all(torch.equal(a[n], c[n]) for n in a)
