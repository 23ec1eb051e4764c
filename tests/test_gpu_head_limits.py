"""The head operators at the ends of what a call may ask for: soft caps of any size, far temperatures, labels that are not used."""
import pytest
import torch

import head_util
import paper_2605_05940_amd as npd
from head_util import dev, head64, inputs, near
from paper_2605_05940_amd import binding
from test_gpu_head import check_loss

pytestmark = pytest.mark.gpu


def head64_relative(s, cap=0.0):
    """`head64` with a soft cap that is off by 2^-20 of itself: below |tanh| = 1/3 a product of five roundings and a polynomial fitted
    to 3.3e-8 (less than 2^-21 together), above it 1 - 2 / (1 + e) with errors of 2^-22 in all (e's and the reciprocal's 2^-23
    relative, at derivatives of at most 4/9 and 4/3, and two roundings); times cap 2^-24 more."""
    z, _, dx = head64(s)
    if not cap:
        return z, torch.ones_like(z), dx
    y = cap * torch.tanh(z / cap)
    return y, 1 - (y / cap) ** 2, dx + 2.0 ** -20 * y.abs()


@pytest.mark.parametrize("T", [1, 7, 40, 70, 150])
@pytest.mark.parametrize("cap", [5.0, 30.0, 1e3, 1e4, 1e6, 1e12])
def test_soft_caps_of_any_size(T, cap, monkeypatch):
    """A logit is as accurate below a high cap as below a low one: logits, scalars and gradients."""
    s = inputs(T, 1003, 64, 3, True, mask=0.9)
    s["hidden"][0] *= 2.0 ** -8          # logits far below the cap
    s["bias"][::2] *= 2.0 ** -8
    s["mask"][T // 2] = 1
    out = torch.empty((T, 1003), dtype=torch.bfloat16, device=dev())
    npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], softcap=cap, logits_out=out)
    torch.cuda.synchronize()
    x, _, dx = head64_relative(s, cap)
    near(out, (x, dx + 2.0 ** -8 * (x.abs() + dx)), "logits")
    monkeypatch.setattr(head_util, "head64", head64_relative)
    check_loss(s, cap=cap, grads=())
    check_loss(s, cap=cap, grad_scale=0.9, ce=0.1)


@pytest.mark.parametrize("tau", [1e10, 1e20, 1e30])
@pytest.mark.parametrize("cap", [0.0, 30.0, 1e-3])
@pytest.mark.parametrize("T,V", [(6, 300), (40, 1003), (100, 1003), (100, 1000), (300, 20001)])
def test_temperatures_that_leave_nothing_of_the_logits(T, V, cap, tau):
    """Every entry counts alike then, and entries behind the vocabulary do not count."""
    s = inputs(T, V, 40, 7, True, mask=0.9)
    s["mask"][T // 2] = 1
    check_loss(s, cap=cap, tau=tau, grads=())
    check_loss(s, cap=cap, tau=tau, grad_scale=tau)


@pytest.mark.parametrize("T", [20, 90])
@pytest.mark.parametrize("grads", [False, True])
def test_labels_that_nothing_uses_are_not_reported(T, grads):
    """Padding labels in a call for the KL alone: the status tells of the ids."""
    s = inputs(T, 400, 64, 4)
    s["mask"].fill_(1)
    s["idx"][11, 2] = 400
    kd, lse = (torch.empty(T, device=dev()) for _ in range(2))
    for labels in (-100, 400):
        s["labels"].fill_(labels)
        status = torch.zeros(1, dtype=torch.int32, device=dev())
        npd.npd_head_loss_fwd_bwd(s["hidden"], s["weight"], s["mask"], labels=s["labels"], teacher_idx=s["idx"],
                                  teacher_val=s["val"], kd_tok=kd, lse_tok=lse, dev_status=status,
                                  grad_hidden=torch.empty_like(s["hidden"]) if grads else None)
        torch.cuda.synchronize()
        assert status.item() == binding.NPD_DEV_BAD_TOPK_INDEX
        assert kd.isnan().nonzero().tolist() == [[11]] and bool(lse.isfinite().all())


@pytest.mark.parametrize("T", [1, 6, 40, 70, 200])
@pytest.mark.parametrize("cap", [0.0, 500.0])
def test_columns_between_a_far_label_and_the_top(T, cap):
    """A row's label lies 2^137 below its most likely entry, other entries 2^39 above the label: their share of 2^-98 is kept."""
    V = 520
    logits = torch.full((V,), -20.0, device=dev())
    logits[3:40] = 27.0
    logits[300] = 95.0
    weight = torch.zeros((V, 8), dtype=torch.bfloat16, device=dev())
    weight[:, 0] = logits.to(torch.bfloat16)
    weight[1] = 0.0   # the label's
    hidden = torch.zeros((T, 8), dtype=torch.bfloat16, device=dev())
    hidden[:, 0] = 1.0
    s = dict(hidden=hidden, weight=weight, labels=torch.ones(T, dtype=torch.int32, device=dev()),
             mask=torch.ones(T, dtype=torch.uint8, device=dev()), bias=None, idx=None, val=None)
    got = check_loss(s, cap=cap, ce=1.0)
    assert bool((got["grad_weight"][3:40, 0] > 0).all())


@pytest.mark.parametrize("T,V,D", [(3, 700, 40), (40, 333, 61), (200, 1003, 72)])
def test_logits_and_their_backward_pass_replay_from_a_graph(T, V, D):
    """One graph of both, replayed with other inputs and eager calls in between; workspaces of the graph's own."""
    s = inputs(T, V, D, bias=True)
    g = torch.zeros((T, V), dtype=torch.bfloat16, device=dev())
    out = [torch.empty((T, V), dtype=torch.bfloat16, device=dev()), torch.empty_like(s["hidden"]), torch.empty_like(s["weight"]),
           torch.empty(V, dtype=torch.bfloat16, device=dev())]

    def call():
        npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], softcap=20.0, logits_out=out[0])
        npd.npd_head_logits_bwd(g, s["hidden"], s["weight"], logits=out[0], softcap=20.0, grad_hidden=out[1], grad_weight=out[2],
                                grad_bias=out[3])

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        other = inputs(T, V, D, bias=True, seed=i + 1)
        for n in ("hidden", "weight", "bias"):
            s[n].copy_(other[n])
        g.copy_(0.1 * torch.randn((T, V), device=dev(), generator=torch.Generator(device=dev()).manual_seed(i)))
        got = []
        for run in (graph.replay, call):
            for t in out:
                t.fill_(float("nan"))
            run()
            torch.cuda.synchronize()
            got.append([t.clone() for t in out])
        for a, b in zip(*got):
            assert torch.equal(a, b) and bool(a.isfinite().all())


def test_logits_on_another_stream():
    s = inputs(150, 900, 61, bias=True)   # (rows that are copied into the call's own workspace)
    want = torch.empty((150, 900), dtype=torch.bfloat16, device=dev())
    npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], logits_out=want)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.empty_like(want) for _ in range(6)]
    for i, out in enumerate(outs):
        with torch.cuda.stream(streams[i % 2]):
            npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], logits_out=out)
    torch.cuda.synchronize()
    for out in outs:
        assert torch.equal(out, want)
