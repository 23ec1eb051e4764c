"""The kernels that large calls of the head operators run, at sizes that a 64-bit implementation still takes: tiles of 256 x 256 and
128 x 256, more of them than compute units (a workgroup then takes a second tile, whose first steps are requested under the
first one's last), loops of several rounds of the stages, contractions in pieces, sums of the weights' gradient over chunks."""
import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding
from head_util import bwd64, dev, head64, inputs, loss64, near
from test_gpu_head import NAN, check_loss, padded, run_loss, untouched

pytestmark = pytest.mark.gpu

# tiles of 256 rows: 2 x 274 forward and 274 of the weights' gradient, for 256 compute units; 7 steps of the width
# tiles of 128 rows: 157 (forward), hidden states' gradient in pieces of the vocabulary
SHAPES = [(300, 70001, 200), (100, 40000, 160), (300, 70016, 328)]


@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("cap,bias,k", [(0.0, True, 10), (30.0, False, 0)])
def test_loss_and_gradients(T, V, D, cap, bias, k):
    check_loss(inputs(T, V, D, k, bias, mask=0.9), cap=cap, grad_scale=0.9, ce=0.1)


@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("cap,bias", [(0.0, True), (30.0, False)])
def test_loss_forward_only(T, V, D, cap, bias):
    check_loss(inputs(T, V, D, 10, bias, seed=1, mask=0.9), cap=cap, grads=())


@pytest.mark.parametrize("T,V,D", SHAPES)
@pytest.mark.parametrize("cap,bias", [(0.0, True), (30.0, False)])
def test_logits(T, V, D, cap, bias):
    s = inputs(T, V, D, bias=bias)
    full, out = padded(T, V, V + 7)
    npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], softcap=cap, logits_out=out)
    torch.cuda.synchronize()
    untouched(full, out)
    x, _, dx = head64(s, cap)
    near(out, (x, dx + 2.0 ** -8 * (x.abs() + dx)), "logits")


@pytest.mark.parametrize("T,V,D", SHAPES + [(600, 70000, 104)])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_logits_backward(T, V, D, cap):
    s = inputs(T, V, D)
    g = (torch.randn((T, V), device=dev()) * 0.1).to(torch.bfloat16)
    y = (cap * torch.tanh(2 * torch.randn((T, V), device=dev()) / cap)).to(torch.bfloat16) if cap else None
    out = dict(grad_hidden=torch.full((T, D), NAN, dtype=torch.bfloat16, device=dev()),
               grad_weight=torch.full((V, D), NAN, dtype=torch.bfloat16, device=dev()),
               grad_bias=torch.full((V,), NAN, dtype=torch.bfloat16, device=dev()))
    npd.npd_head_logits_bwd(g, s["hidden"], s["weight"], logits=y, softcap=cap, **out)
    torch.cuda.synchronize()
    want = bwd64(g, s, y, cap)
    for name, v in out.items():
        near(v, want[name], name)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("scored", [2100, 700])
def test_weight_gradient_over_chunks(accumulate, scored):
    """Three chunks (or one, of three that were launched) of 258 tiles: first, middle and last forms take a second tile."""
    T, V, D = 2100, 66001, 40
    s = inputs(T, V, D, 6, True)
    s["mask"].fill_(1)
    s["mask"][scored:] = 0
    d = binding.HeadDesc(T, V, D, D, D, D, D, 0, 6, 15 if accumulate else 7, 1.0, 0.9, 0.1, 0.0)
    least = binding.load().npd_head_workspace_bytes(d, binding.NPD_HEAD_LOSS)
    assert least < binding.load().npd_head_workspace_bytes_preferred(d, binding.NPD_HEAD_LOSS)
    start = dict(grad_weight=torch.randn((V, D), device=dev()).to(torch.bfloat16),
                 grad_bias=torch.randn(V, device=dev()).to(torch.bfloat16)) if accumulate else {}
    want = loss64(s, grad_scale=0.9, ce=0.1)
    got = run_loss(s, grad_scale=0.9, ce=0.1, accumulate=start, workspace=torch.empty(least, dtype=torch.uint8, device=dev()))
    for n, v in got.items():
        value, t = want[n]
        if n in start:
            value = value + start[n].double()
            t = t + 2.0 ** -8 * value.abs()
        near(v, (value, t), n)


def test_one_chunk_accumulates():
    T, V, D = 300, 70001, 200
    s = inputs(T, V, D, 6, True)
    start = dict(grad_weight=torch.randn((V, D), device=dev()).to(torch.bfloat16))
    want = loss64(s, grad_scale=0.9, ce=0.1)["grad_weight"]
    got = run_loss(s, grad_scale=0.9, ce=0.1, grads=("hidden", "weight"), accumulate=start)
    value = want[0] + start["grad_weight"].double()
    near(got["grad_weight"], (value, want[1] + 2.0 ** -8 * value.abs()), "grad_weight")


def test_a_large_call_repeats_itself():
    s = inputs(300, 70001, 200, 9, True)
    a, b = (run_loss(s, grad_scale=0.9, ce=0.1) for _ in range(2))
    for name in a:
        assert torch.equal(a[name], b[name]), name


@pytest.mark.parametrize("T", [1, 3, 4, 6, 30])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_few_rows_of_a_large_vocabulary(T, cap):
    """More workgroups than a compute unit has room for three of: the other order of their loads."""
    V, D = 130001, 264
    s = inputs(T, V, D, 5, True)
    s["mask"][T // 2] = 1
    check_loss(s, cap=cap, grads=())
    check_loss(s, cap=cap, grad_scale=0.9, ce=0.1)
    full, out = padded(T, V, V + 2)
    npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], softcap=cap, logits_out=out)
    torch.cuda.synchronize()
    untouched(full, out)
    x, _, dx = head64(s, cap)
    near(out, (x, dx + 2.0 ** -8 * (x.abs() + dx)), "logits")
