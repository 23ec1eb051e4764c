"""Rows as 8-bit integers and the head's logits in them, against exact whole numbers and 64 bits.

Tolerances: the sums are exact.  With u = 2^-24 the sum's conversion to fp32, two factors and the bias are four roundings, 4 u (|x| + |bias|)
of the logit before its soft cap, whose slope is at most 1 and which is off by 2^-20 of itself; B = 2^-8 rounds the result to bf16.
"""
import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding

pytestmark = pytest.mark.gpu

B, U = 2.0 ** -8, 2.0 ** -24
DEV = "cuda:0"


# --------------------------------------------------------------------------------------------------------- whole numbers

def quantized(x):
    """Exact quotients 127 x / max in 64 bits (15 and 8 bits: what is half way between two whole numbers is exactly there)."""
    v = x.double()
    top = v.abs().amax(1)
    q = torch.round(127 * v / torch.where(top > 0, top, 1.0)[:, None])
    # (rounded once from 64 bits, where a quotient by 127 is never half way: torch divides by a number through its reciprocal)
    return q, (top / 127).float()


def quantize(x, pad=0):
    R, D = x.shape
    whole = torch.full((R, D + pad), 99, dtype=torch.int8, device=DEV)
    scale = torch.empty(R, device=DEV)
    npd.npd_quantize_rows(x, q_out=whole[:, :D], scale_out=scale)
    assert bool((whole[:, D:] == 99).all())
    return whole[:, :D], scale


SIZES = [(1, 1), (4, 7), (9, 8), (5, 100), (300, 512), (7, 513), (33, 1000), (6, 1024), (5, 1025), (17, 2048), (3, 2049), (9, 4096),
         (3, 5000), (4, 8192), (2, 8200), (2, 16384), (3, 20001), (1, 32768), (2, 65536)]


@pytest.mark.parametrize("R,D", SIZES)
def test_rows_are_exact(R, D):
    g = torch.Generator(device=DEV).manual_seed(R + D)
    whole = (torch.randn((R, D + 3), device=DEV, generator=g) * torch.exp(3 * torch.randn((R, 1), device=DEV, generator=g))).to(torch.bfloat16)
    x = whole[:, :D] if D % 2 else whole[:, 3:]
    q, scale = quantize(x, pad=5 if R % 2 else 0)
    want, want_scale = quantized(x)
    assert torch.equal(q.double(), want) and torch.equal(scale, want_scale)


@pytest.mark.parametrize("exponent", [-130, -126, -100, -8, 0, 3, 100, 120])
def test_quotients_half_way(exponent):
    """Largest values whose quotients are whole and half numbers: ties go to the even one, whatever the exponent."""
    halves = torch.arange(-254, 255, device=DEV).double() / 2
    rows = [halves * m for m in (1.0, 2.0)] + [torch.cat([halves[::2] * 0.5, torch.tensor([127.0] * 254, device=DEV).double()])]
    x64 = torch.stack([r[:509] for r in rows]) * 2.0 ** exponent
    x = x64.to(torch.bfloat16)
    q, scale = quantize(x)
    want, want_scale = quantized(x)
    assert torch.equal(q.double(), want)
    if exponent > -120:  # (below, 1 / 127 of them is not a normal number)
        assert torch.equal(scale, want_scale)


def test_every_pair_of_values():
    """All magnitudes of one exponent below all largest ones of it and the seven exponents above: every quotient there is."""
    tops = torch.arange(128, 256, device=DEV).double()
    values = torch.cat([torch.arange(128, 256, device=DEV).double() * 2.0 ** -e for e in range(9)])
    x = torch.cat([tops[:, None], torch.minimum(values[None, :], tops[:, None])], 1).to(torch.bfloat16)
    x[:, 1::2] *= -1
    q, scale = quantize(x)
    want, want_scale = quantized(x)
    assert torch.equal(q.double(), want) and torch.equal(scale, want_scale)


def test_rows_of_zeros_extremes_and_what_is_not_finite():
    x = torch.zeros((6, 300), dtype=torch.bfloat16, device=DEV)
    x[1, 5] = float("nan")
    x[2, 299] = float("-inf")
    x[3, 7] = -3.3895313892515355e38
    x[3, 8] = 1.0e38
    x[4, 0] = 9.2e-41  # the smallest one there is
    x[5] = -0.0
    q, scale = quantize(x)
    want, want_scale = quantized(torch.where(x.isfinite(), x, 0))
    assert bool(scale[1].isnan()) and bool(scale[2].isnan()) and not bool(q[1].any()) and not bool(q[2].any())
    for r in (0, 3, 4, 5):
        assert torch.equal(q[r].double(), want[r]), r
        assert float((scale[r] - want_scale[r]).abs()) <= 2.0 ** -149


# -------------------------------------------------------------------------------------------------------------- products

def operands(T, V, D, g, h_pad=0, w_pad=0, offset=0, most=127):
    def ints(rows, pad):
        m = torch.randint(-most, most + 1, (rows * (D + pad) + offset,), device=DEV, generator=g, dtype=torch.int8)
        return m[offset:].view(rows, D + pad)[:, :D]
    scales = [torch.exp(torch.randn(n, device=DEV, generator=g)) * 2e-3 for n in (T, V)]
    return ints(T, h_pad), scales[0], ints(V, w_pad), scales[1]


def logits64(h, hs, w, ws, bias, cap):
    x = (h.double() @ w.double().t()) * hs.double()[:, None] * ws.double()
    b = torch.zeros(w.shape[0], device=DEV).double() if bias is None else bias.double()
    tol = 4 * U * (x.abs() + b.abs())
    x = x + b
    if cap:
        x = cap * torch.tanh(x / cap)
        tol = tol + 2.0 ** -20 * x.abs()
    return x, tol * (1 + B) + B * x.abs()


def check(h, hs, w, ws, bias=None, cap=0.0, pad=0, **more):
    T, V = h.shape[0], w.shape[0]
    whole = torch.full((T, V + pad), 3.0, dtype=torch.bfloat16, device=DEV)
    npd.npd_head_logits_int8(h, hs, w, ws, bias=bias, softcap=cap, logits_out=whole[:, :V], **more)
    x, tol = logits64(h, hs, w, ws, bias, cap)
    off = (whole[:, :V].double() - x).abs()
    assert bool((off <= tol + 1e-30).all()), float((off / (tol + 1e-30)).max())
    assert bool((whole[:, V:] == 3.0).all())


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 31, 33, 47, 48, 49, 63, 64, 65, 130])
@pytest.mark.parametrize("V,D", [(1, 1), (7, 15), (33, 16), (130, 17), (500, 64), (1000, 100), (257, 255), (129, 256), (1025, 257),
                                 (300, 1000), (8200, 512)])
def test_few_and_more_rows(T, V, D):
    g = torch.Generator(device=DEV).manual_seed(T + 100 * V + D)
    bias = torch.randn(V, device=DEV, generator=g).to(torch.bfloat16) if (T + V) % 2 else None
    check(*operands(T, V, D, g), bias=bias, cap=30.0 if T % 3 == 0 else 0.0, pad=T % 2)


@pytest.mark.parametrize("T", [1, 6, 13, 40, 64, 100])
@pytest.mark.parametrize("h_pad,w_pad,offset", [(0, 1, 0), (16, 32, 0), (3, 8, 5), (0, 0, 1), (16, 0, 16)])
def test_rows_that_begin_anywhere(T, h_pad, w_pad, offset):
    for D in (304, 301):
        g = torch.Generator(device=DEV).manual_seed(T)
        check(*operands(T, 700, D, g, h_pad, w_pad, offset), pad=1)


@pytest.mark.parametrize("T", [1, 4, 8])
@pytest.mark.parametrize("V,D", [(2000, 2048), (1001, 2300), (33000, 2048), (5000, 4100)])
def test_rows_of_many_blocks(T, V, D):
    g = torch.Generator(device=DEV).manual_seed(T + V)
    check(*operands(T, V, D, g))


@pytest.mark.parametrize("T,V,D", [(16, 40000, 300), (64, 33001, 256), (48, 32768, 512), (33, 40000, 260)])
def test_wide_vocabularies_of_few_rows(T, V, D):
    g = torch.Generator(device=DEV).manual_seed(T + V)
    check(*operands(T, V, D, g), bias=torch.randn(V, device=DEV, generator=g).to(torch.bfloat16), cap=20.0)


@pytest.mark.parametrize("cap", [0.0, 30.0])
@pytest.mark.parametrize("T,V,D", [(65, 1000, 64), (128, 20000, 128), (100, 17003, 192), (129, 16500, 64), (300, 17001, 100), (2100, 2100, 208),
                                   (2305, 4100, 64), (700, 9000, 1024), (257, 70000, 160)])
def test_tiles(T, V, D, cap):
    g = torch.Generator(device=DEV).manual_seed(T + V + D)
    bias = torch.randn(V, device=DEV, generator=g).to(torch.bfloat16) if T % 2 else None
    check(*operands(T, V, D, g), bias=bias, cap=cap, pad=V % 2)


@pytest.mark.parametrize("T", [1, 8, 20, 64, 65, 300])
def test_largest_sums(T):
    """65,536 products of (-128)^2, the largest there are: 2^30."""
    D, V = 65536, 200 if T < 300 else 16640
    h, w = torch.full((T, D), -128, dtype=torch.int8, device=DEV), torch.full((V, D), -128, dtype=torch.int8, device=DEV)
    w[::2] = 127
    out = torch.empty((T, V), dtype=torch.bfloat16, device=DEV)
    npd.npd_head_logits_int8(h, torch.ones(T, device=DEV), w, torch.ones(V, device=DEV), logits_out=out)
    want = torch.tensor([-128.0 * 127 * D, 128.0 * 128 * D], device=DEV).to(torch.bfloat16)
    assert bool((out[:, ::2] == want[0]).all()) and bool((out[:, 1::2] == want[1]).all())


def test_scales_that_are_zero_large_small_or_not_finite():
    g = torch.Generator(device=DEV).manual_seed(1)
    for T in (3, 20, 90):
        h, hs, w, ws = operands(T, 200, 128, g)
        hs[0], ws[5] = 0.0, 0.0
        hs[1] = 1e30
        ws[7] = 1e-30
        check(h, hs, w, ws)
        hs[2] = float("nan")
        out = torch.empty((T, 200), dtype=torch.bfloat16, device=DEV)
        npd.npd_head_logits_int8(h, hs, w, ws, logits_out=out)
        assert bool(out[2].isnan().all()) and not bool(out[:2].isnan().any())


def test_weights_padded_to_sixteen_need_no_workspace():
    """What lies between the width and the stride is not part of the rows."""
    g = torch.Generator(device=DEV).manual_seed(3)
    T, V, D = 100, 1000, 1000
    assert npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOGITS_INT8, T, V, 1008) == 0
    assert npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOGITS_INT8, 64, V, D) == 0
    assert npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOGITS_INT8, T, V, D, hidden_stride=1008, weight_stride=1008) > 0
    check(*operands(T, V, D, g, 8, 8))
    check(*operands(T, V, 1008, g), workspace=torch.empty(0, dtype=torch.uint8, device=DEV))


def test_captured_streams_and_workspaces():
    """Two captured calls with workspaces of their own, replayed in turn and side by side with eager ones."""
    g = torch.Generator(device=DEV).manual_seed(4)
    T, V, D = 150, 3001, 333
    sets = [operands(T, V, D, g) for _ in range(2)]
    need = npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOGITS_INT8, T, V, D)
    want, graphs, outs = [], [], []
    for s in sets:
        ws = torch.empty(need, dtype=torch.uint8, device=DEV)
        out = torch.empty((T, V), dtype=torch.bfloat16, device=DEV)
        npd.npd_head_logits_int8(*s, logits_out=out, workspace=ws)
        want.append(out.clone())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            npd.npd_head_logits_int8(*s, logits_out=out, workspace=ws)
        graphs.append((graph, ws))
        outs.append(out)
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        for out in outs:
            out.zero_()
        torch.cuda.synchronize()
        for (graph, _), stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        eager = torch.empty_like(outs[0])
        npd.npd_head_logits_int8(*sets[0], logits_out=eager)
        torch.cuda.synchronize()
        assert torch.equal(eager, want[0]) and all(torch.equal(o, w) for o, w in zip(outs, want))


def test_rows_behind_the_last_are_left():
    """Rows of the logits that the call does not have stay as they were."""
    g = torch.Generator(device=DEV).manual_seed(6)
    for T in (3, 20, 70, 260):
        h, hs, w, ws = operands(T, 640, 64, g)
        out = torch.full((T + 3, 640), 3.0, dtype=torch.bfloat16, device=DEV)
        npd.npd_head_logits_int8(h, hs, w, ws, logits_out=out[:T])
        assert bool((out[T:] == 3.0).all())
