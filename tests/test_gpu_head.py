"""The head operators (npd_head_loss_fwd_bwd, npd_head_logits, npd_head_logits_bwd) on the GPU against plain 64-bit
implementations of their formulas (tests/head_util.py, which derives the tolerances)."""
import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding
from head_util import bwd64, dev, head64, inputs, loss64, near

pytestmark = pytest.mark.gpu
NAN = float("nan")


def padded(rows, cols, pitch, dtype=torch.bfloat16, offset=0):
    """A [rows, cols] view with `pitch` elements between rows and NaN around it, and the buffer it lies in."""
    full = torch.full((rows * pitch + 64 + offset,), NAN, dtype=dtype, device=dev())
    return full, full[32 + offset:32 + offset + rows * pitch].view(rows, pitch)[:, :cols]


def untouched(full, view):
    """Everything of the buffer outside the view is still NaN."""
    outside = torch.ones_like(full, dtype=torch.bool)
    outside[(view.data_ptr() - full.data_ptr()) // 2:][:view.shape[0] * view.stride(0)].view(
        view.shape[0], view.stride(0))[:, :view.shape[1]] = False
    assert bool(full[outside].isnan().all()), "written outside the tensor"


def run_loss(s, *, cap=0.0, tau=1.0, grad_scale=1.0, ce=0.0, grads=("hidden", "weight", "bias"), accumulate=None,
             workspace=None, pitch=None, status=0):
    """One call with padded outputs; returns {name: tensor}."""
    T, D = s["hidden"].shape
    V = s["weight"].shape[0]
    out, kept = {}, []
    if tau == 1.0:
        out["lse"] = torch.full((T,), NAN, device=dev())
        out["nll"] = torch.full((T,), NAN, device=dev())
    if s["idx"] is not None:
        out["kd"] = torch.full((T,), NAN, device=dev())
    shapes = dict(hidden=(T, D), weight=(V, D))
    for g in grads:
        if g == "bias":
            out["grad_bias"] = torch.full((V,), NAN, dtype=torch.bfloat16, device=dev())
        else:
            full, out["grad_" + g] = padded(*shapes[g], pitch or D)
            kept.append((full, out["grad_" + g]))
    if accumulate:
        for name, start in accumulate.items():
            out[name].copy_(start)
    st = torch.zeros(1, dtype=torch.int32, device=dev())
    npd.npd_head_loss_fwd_bwd(
        s["hidden"], s["weight"], s["mask"], bias=s["bias"], softcap=cap, labels=s["labels"], teacher_idx=s["idx"],
        teacher_val=s["val"], tau=tau, grad_scale=grad_scale, ce_grad_scale=ce, grad_hidden=out.get("grad_hidden"),
        grad_weight=out.get("grad_weight"), grad_bias=out.get("grad_bias"), accumulate=bool(accumulate),
        kd_tok=out.get("kd"), nll_tok=out.get("nll"), lse_tok=out.get("lse"), dev_status=st, workspace=workspace)
    torch.cuda.synchronize()
    assert st.item() == status
    for full, view in kept:
        untouched(full, view)
    return out


def check_loss(s, **kw):
    want = loss64(s, cap=kw.get("cap", 0.0), tau=kw.get("tau", 1.0), grad_scale=kw.get("grad_scale", 1.0), ce=kw.get("ce", 0.0))
    got = run_loss(s, **kw)
    for name, v in got.items():
        near(v, want[name], name)
    return got


# T, V, D, k, kd weight, ce weight, tau, bias, cap
SHAPES = [
    (1, 1, 1, 1, 1.0, 0.0, 1.0, False, 0.0),
    (1, 1000, 64, 0, 0.0, 1.0, 1.0, False, 0.0),
    (2, 33, 8, 5, 0.9, 0.1, 1.0, True, 0.0),
    (5, 8, 24, 8, 1.0, 0.0, 2.0, False, 0.0),
    (17, 129, 7, 3, 0.5, 0.5, 1.0, True, 5.0),
    (64, 256, 32, 10, 1.0, 0.0, 0.5, False, 0.0),
    (65, 257, 40, 7, 0.9, 0.1, 1.0, False, 30.0),
    (100, 4099, 260, 0, 0.0, 0.25, 1.0, True, 0.0),
    (129, 515, 100, 3, 0.9, 0.1, 1.0, True, 0.0),
    (257, 1024, 256, 10, 0.9, 0.1, 1.0, False, 0.0),
    (300, 2000, 1000, 64, 1.0, 0.0, 2.0, True, 0.0),
    (513, 1031, 520, 100, 0.9, 0.1, 1.0, False, 3.0),
    (900, 5003, 72, 20, 0.9, 0.1, 1.0, True, 0.0),
    (40, 40000, 128, 10, 0.9, 0.1, 1.0, False, 0.0),
]


@pytest.mark.parametrize("T,V,D,k,gs,ce,tau,bias,cap", SHAPES)
def test_loss_and_gradients(T, V, D, k, gs, ce, tau, bias, cap):
    s = inputs(T, V, D, k, bias)
    s["mask"][T // 2] = 1
    check_loss(s, cap=cap, tau=tau, grad_scale=gs, ce=ce)


@pytest.mark.parametrize("T,V,D,k,gs,ce,tau,bias,cap", SHAPES[:10])
def test_loss_forward_only(T, V, D, k, gs, ce, tau, bias, cap):
    check_loss(inputs(T, V, D, k, bias, seed=1), cap=cap, tau=tau, grads=())


@pytest.mark.parametrize("T", [3, 4, 5, 8, 9, 16, 17, 31, 33, 48, 49, 64])
@pytest.mark.parametrize("V,D,bias,cap", [(515, 129, True, 0.0), (33000, 40, False, 30.0), (1000, 256, True, 2.0)])
def test_few_rows(T, V, D, bias, cap):
    """Every number of rows that has a kernel of its own, both widths of its workgroups: scalars, gradients, logits."""
    s = inputs(T, V, D, 3, bias, mask=0.9)
    check_loss(s, cap=cap, grad_scale=0.9, ce=0.1)
    full, out = padded(T, V, V + 3)
    npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], softcap=cap, logits_out=out)
    torch.cuda.synchronize()
    untouched(full, out)
    x, _, dx = head64(s, cap)
    near(out, (x, dx + 2.0 ** -8 * (x.abs() + dx)), "logits")


@pytest.mark.parametrize("grads", [("hidden",), ("weight",), ("bias",), ("hidden", "bias")])
def test_loss_any_gradient_alone(grads):
    s = inputs(150, 777, 96, 12, True)
    check_loss(s, grad_scale=0.7, ce=0.3, grads=grads)


@pytest.mark.parametrize("mask", ["none", "one", "all", "last"])
def test_loss_masks(mask):
    s = inputs(300, 600, 64, 5, True)
    s["mask"].fill_(1 if mask == "all" else 0)
    if mask in ("one", "last"):
        s["mask"][0 if mask == "one" else -1] = 3
    got = check_loss(s, grad_scale=0.9, ce=0.1)
    if mask == "none":
        for v in got.values():
            assert not v.any()


def test_loss_masked_positions_are_not_read():
    s = inputs(200, 500, 64, 5)
    want = run_loss(s, grad_scale=0.9, ce=0.1)
    off = s["mask"] == 0
    s["hidden"][off] = NAN
    s["labels"][off] = -100
    s["idx"][off] = 1 << 30
    s["val"][off] = NAN
    got = run_loss(s, grad_scale=0.9, ce=0.1)
    for name in want:
        assert torch.equal(got[name], want[name]), name


@pytest.mark.parametrize("T", [1024, 1025, 2500, 2048 + 256])
def test_loss_in_chunks(T):
    """The least workspace holds 1,024 rows at a time where there are many more: gradients of the weights are summed over chunks."""
    s = inputs(T, 700, 72, 6, True, mask=0.95)
    d = binding.HeadDesc(T, 700, 72, 72, 72, 72, 72, 0, 6, 7, 1.0, 0.9, 0.1, 0.0)
    least = binding.load().npd_head_workspace_bytes(d, binding.NPD_HEAD_LOSS)
    most = binding.load().npd_head_workspace_bytes_preferred(d, binding.NPD_HEAD_LOSS)
    assert 0 < least <= most and (least < most) == (T > 2000)
    check_loss(s, grad_scale=0.9, ce=0.1, workspace=torch.empty(least, dtype=torch.uint8, device=dev()))
    s["mask"][300:] = 0   # chunks that turn out to be empty
    check_loss(s, grad_scale=0.9, ce=0.1, workspace=torch.empty(least, dtype=torch.uint8, device=dev()))


@pytest.mark.parametrize("scored", [2500, 200, 0])
def test_loss_in_chunks_accumulates(scored):
    T, V, D = 2500, 700, 72
    s = inputs(T, V, D, 6, True)
    s["mask"].fill_(1)
    s["mask"][scored:] = 0
    d = binding.HeadDesc(T, V, D, D, D, D, D, 0, 6, 15, 1.0, 0.9, 0.1, 0.0)
    ws = torch.empty(binding.load().npd_head_workspace_bytes(d, binding.NPD_HEAD_LOSS), dtype=torch.uint8, device=dev())
    start = dict(grad_weight=torch.randn((V, D), device=dev()).to(torch.bfloat16),
                 grad_bias=torch.randn(V, device=dev()).to(torch.bfloat16))
    want = loss64(s, grad_scale=0.9, ce=0.1)
    got = run_loss(s, grad_scale=0.9, ce=0.1, accumulate=start, workspace=ws)
    for n, a in start.items():
        v, t = want[n]
        v = v + a.double()
        near(got[n], (v, t + 2.0 ** -8 * v.abs()), n)
    near(got["grad_hidden"], want["grad_hidden"], "grad_hidden")


def test_a_workspace_of_every_size_between():
    """Chunks of 1,024, 2,048, 4,096 and 8,192 rows: the same results to rounding, nothing written behind the bytes asked for."""
    T, V, D = 9000, 200, 24
    s = inputs(T, V, D, 3, True, mask=0.9)
    d = binding.HeadDesc(T, V, D, D, D, D, D, 0, 3, 7, 1.0, 0.9, 0.1, 0.0)
    least = binding.load().npd_head_workspace_bytes(d, binding.NPD_HEAD_LOSS)
    most = binding.load().npd_head_workspace_bytes_preferred(d, binding.NPD_HEAD_LOSS)
    assert least < most
    for n in {least, (least + most) // 2, most - 1, most}:
        full = torch.full((n + 512,), 0x5a, dtype=torch.uint8, device=dev())
        check_loss(s, grad_scale=0.9 / T, ce=0.1 / T, workspace=full[:n])
        assert bool((full[n:] == 0x5a).all())


def test_loss_more_rows_than_a_preferred_chunk():
    s = inputs(9000, 300, 40, 4, mask=0.97)
    check_loss(s, grad_scale=0.9 / 9000, ce=0.1 / 9000)


@pytest.mark.parametrize("spread", [30.0, 300.0])
@pytest.mark.parametrize("cap", [0.0, 50.0])
def test_loss_far_logits(spread, cap):
    """Logits of hundreds and thousands: a row's columns lie far above its label's, parts of it take references of their own."""
    s = inputs(200, 1500, 64, 5, True, seed=1, spread=spread)
    s["labels"] = torch.randint(0, 1500, (200,), dtype=torch.int32, device=dev())
    check_loss(s, cap=cap, grad_scale=0.9, ce=0.1)


def test_loss_banned_entries():
    """A bias of -inf: probability 0, no gradient there; +inf where the teacher or the label asks for it."""
    s = inputs(60, 900, 64, 4, True)
    s["bias"][100:600] = -float("inf")
    s["idx"] = torch.stack([torch.randperm(100, device=dev())[:4] for _ in range(60)]).to(torch.int32)
    s["labels"] = torch.randint(600, 900, (60,), dtype=torch.int32, device=dev())
    s["mask"][0] = 1
    got = check_loss(s, grad_scale=0.9, ce=0.1)
    assert not got["grad_weight"][100:600].any() and not got["grad_bias"][100:600].any()
    s["labels"][0] = 200
    s["idx"][0, 1] = 300
    out = run_loss(s, grads=())
    assert out["nll"][0] == float("inf") and out["kd"][0] == float("inf")
    assert bool(out["nll"][1:].isfinite().all()) and bool(out["lse"].isfinite().all())
    s["val"][0, 1] = -float("inf")   # an entry without weight asks for nothing
    out = run_loss(s, grads=())
    near(out["kd"], loss64(s)["kd"], "kd")


def test_loss_not_a_number_stays_with_its_position():
    s = inputs(70, 400, 64, 4)
    s["mask"].fill_(1)
    want = run_loss(s, grad_scale=0.9, ce=0.1, grads=("hidden",))
    s["hidden"][13, 5] = NAN
    s["hidden"][40] = float("inf")
    got = run_loss(s, grad_scale=0.9, ce=0.1, grads=("hidden",))
    bad = torch.zeros(70, dtype=torch.bool, device=dev())
    bad[[13, 40]] = True
    for name in want:
        assert torch.equal(got[name][~bad], want[name][~bad]), name
        assert not bool(got[name][13].isfinite().any()), name


def test_loss_bad_labels_and_ids():
    s = inputs(80, 400, 64, 4, True)
    s["mask"].fill_(1)
    good = dict(s, mask=s["mask"].clone())
    good["mask"][[3, 50, 60]] = 0
    want = loss64(good, grad_scale=0.9, ce=0.1)
    s["labels"][3], s["labels"][50] = -1, 400
    s["idx"][60, 2] = 400
    got = run_loss(s, grad_scale=0.9, ce=0.1, status=binding.NPD_DEV_BAD_LABEL | binding.NPD_DEV_BAD_TOPK_INDEX)
    near(got["grad_weight"], want["grad_weight"], "grad_weight")
    near(got["grad_bias"], want["grad_bias"], "grad_bias")
    for name, rows in (("nll", [3, 50]), ("kd", [60]), ("grad_hidden", [3, 50, 60])):
        assert bool(got[name][rows].isnan().all()), name
        keep = torch.ones(80, dtype=torch.bool, device=dev())
        keep[[3, 50, 60]] = False
        near(got[name][keep], tuple(t[keep] for t in want[name]), name)


@pytest.mark.parametrize("D,pitch,offset", [(64, 72, 0), (64, 71, 0), (61, 64, 0), (64, 64, 3), (40, 40, 8)])
def test_loss_strides_and_alignment(D, pitch, offset):
    T, V = 90, 333
    s = inputs(T, V, D, 5, True)
    for name, n in (("hidden", T), ("weight", V)):
        _, view = padded(n, D, pitch, offset=offset)
        s[name] = view.copy_(s[name])
    check_loss(s, grad_scale=0.9, ce=0.1, pitch=pitch)


def test_loss_accumulates():
    s = inputs(140, 300, 64, 4, True)
    plain = run_loss(s, grad_scale=0.9, ce=0.1)
    start = {n: torch.randn_like(plain[n].float()).to(torch.bfloat16) for n in ("grad_weight", "grad_bias")}
    want = loss64(s, grad_scale=0.9, ce=0.1)
    got = run_loss(s, grad_scale=0.9, ce=0.1, accumulate=start)
    for n, a in start.items():
        v, t = want[n]
        v = v + a.double()
        near(got[n], (v, t + 2.0 ** -8 * v.abs()), n)
    assert torch.equal(got["grad_hidden"], plain["grad_hidden"])


def test_loss_is_reproducible():
    s = inputs(700, 3000, 136, 9, True)
    a, b = (run_loss(s, grad_scale=0.9, ce=0.1) for _ in range(2))
    for name in a:
        assert torch.equal(a[name], b[name]), name


def test_loss_against_differences():
    """A step of one hidden state along a coordinate, exact in bf16: the difference of the scalars against the gradient."""
    T, V, D = 6, 200, 32
    s = inputs(T, V, D, 5)
    s["mask"].fill_(1)
    step = 2.0 ** -5
    s["hidden"] = (torch.round(s["hidden"].float().clamp(-1.9, 1.9) / step) * step).to(torch.bfloat16)
    grad = run_loss(s, grad_scale=0.9, ce=0.1, grads=("hidden",))["grad_hidden"].double()
    scale = loss64(s, grad_scale=0.9, ce=0.1)["grad_hidden"][0].abs().amax()
    for d in (0, 7, 31):
        f = []
        for sign in (1, -1):
            t = dict(s, hidden=s["hidden"].clone())
            t["hidden"][:, d] += sign * step
            out = run_loss(t, grads=())
            f.append(0.9 * out["kd"].double() + 0.1 * out["nll"].double())
        # central differences: third derivatives of a log-sum-exp of weights below 2 give at most step^2 2^3 / 6; the scalars'
        # own errors (1e-5 here) are divided by twice the step
        got = (f[0] - f[1]) / (2 * step)
        assert (got - grad[:, d]).abs().max() <= step ** 2 * 8 / 6 + 1e-5 / step + 2.0 ** -7 * scale


def test_loss_replays_from_a_graph():
    s = inputs(400, 1200, 64, 6, True)
    s["mask"][0] = 1
    T, V, D = 400, 1200, 64
    out = [torch.empty((T, D), dtype=torch.bfloat16, device=dev()), torch.empty((V, D), dtype=torch.bfloat16, device=dev()),
           torch.empty(V, dtype=torch.bfloat16, device=dev()), *(torch.empty(T, device=dev()) for _ in range(3))]

    def call():
        npd.npd_head_loss_fwd_bwd(s["hidden"], s["weight"], s["mask"], bias=s["bias"], labels=s["labels"], teacher_idx=s["idx"],
                                  teacher_val=s["val"], grad_scale=0.9, ce_grad_scale=0.1, grad_hidden=out[0],
                                  grad_weight=out[1], grad_bias=out[2], kd_tok=out[3], nll_tok=out[4], lse_tok=out[5])

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        other = inputs(T, V, D, 6, True, seed=2 * i + 2, mask=0.2 + 0.2 * i)
        for n in s:
            s[n].copy_(other[n])
        for t in out:
            t.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for t in out:
            t.fill_(NAN)
        call()
        torch.cuda.synchronize()
        for a, b in zip(got, out):
            assert torch.equal(a, b)


def test_two_calls_at_once_on_two_streams():
    sets = [inputs(600, 2000, 64, 6, True, seed=i) for i in range(2)]
    want = [run_loss(s, grad_scale=0.9, ce=0.1) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [[torch.empty_like(w["grad_hidden"].contiguous()), torch.empty_like(w["grad_weight"].contiguous()),
             torch.empty_like(w["nll"])] for w in want]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, o, on in zip(sets, outs, streams):
            with torch.cuda.stream(on):
                npd.npd_head_loss_fwd_bwd(s["hidden"], s["weight"], s["mask"], bias=s["bias"], labels=s["labels"],
                                          teacher_idx=s["idx"], teacher_val=s["val"], grad_scale=0.9, ce_grad_scale=0.1,
                                          grad_hidden=o[0], grad_weight=o[1], nll_tok=o[2])
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        for a, n in zip(o, ("grad_hidden", "grad_weight", "nll")):
            assert torch.equal(a, w[n]), n


# ------------------------------------------------------------------------------------------------------------ the logits

@pytest.mark.parametrize("T,V,D,bias,cap", [(1, 1, 1, False, 0.0), (1, 5000, 128, True, 0.0), (3, 17, 9, True, 30.0),
                                            (64, 300, 64, False, 0.0), (65, 1027, 100, True, 2.0), (130, 512, 72, False, 30.0),
                                            (300, 3001, 136, True, 0.0), (513, 1024, 256, False, 0.0)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 0), (5, 0), (0, 1)])
def test_logits(T, V, D, bias, cap, pad, offset):
    s = inputs(T, V, D, bias=bias)
    full, out = padded(T, V, V + pad, offset=offset)
    npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], softcap=cap, logits_out=out)
    torch.cuda.synchronize()
    untouched(full, out)
    x, _, dx = head64(s, cap)
    near(out, (x, dx + 2.0 ** -8 * (x.abs() + dx)), "logits")


@pytest.mark.parametrize("T,V,D,bias,cap", [(1, 1, 1, True, 0.0), (1, 5000, 128, False, 0.0), (5, 24, 8, True, 0.0),
                                            (64, 256, 64, True, 30.0), (65, 1027, 100, True, 2.0), (130, 512, 72, False, 30.0),
                                            (300, 3001, 136, True, 0.0), (513, 1024, 256, False, 0.0),
                                            (1500, 1003, 64, True, 30.0)])
@pytest.mark.parametrize("pad,offset", [(0, 0), (8, 0), (5, 0), (0, 1)])
def test_logits_backward(T, V, D, bias, cap, pad, offset):
    s = inputs(T, V, D, bias=bias)
    _, g = padded(T, V, V + pad, offset=offset)
    g.copy_(torch.randn((T, V), device=dev()) * 0.1)
    y = None
    if cap:
        _, y = padded(T, V, V + pad)
        y.copy_(cap * torch.tanh(2 * torch.randn((T, V), device=dev()) / cap))
    out = dict(grad_hidden=torch.full((T, D), NAN, dtype=torch.bfloat16, device=dev()),
               grad_weight=torch.full((V, D), NAN, dtype=torch.bfloat16, device=dev()))
    if bias:
        out["grad_bias"] = torch.full((V,), NAN, dtype=torch.bfloat16, device=dev())
    d = binding.HeadDesc(T, V, D, D, D, D, D, V + pad, 0, 3 | (4 if bias else 0) | (16 if offset else 0), 1.0, 0.0, 0.0, cap)
    least = binding.load().npd_head_workspace_bytes(d, binding.NPD_HEAD_LOGITS_BWD)
    ws = torch.empty(least, dtype=torch.uint8, device=dev()) if T > 1024 else None   # two chunks, where rows are copied
    npd.npd_head_logits_bwd(g, s["hidden"], s["weight"], logits=y, softcap=cap, workspace=ws, **out)
    torch.cuda.synchronize()
    want = bwd64(g, s, y, cap)
    for name, v in out.items():
        near(v, want[name], name)


def test_the_operators_together():
    """Teacher logits and record, dense and top-k losses of the student from logits and from hidden states, per-sample means:
    the two ways to the same loss agree to the rounding of the logits they went through."""
    T, V, D = 320, 2000, 128
    student, teacher = inputs(T, V, D, mask=0.8), inputs(T, V, D, seed=1)
    mask, labels = student["mask"], student["labels"]
    logits = {n: torch.empty((T, V), dtype=torch.bfloat16, device=dev()) for n in ("student", "teacher")}
    for n, s in (("student", student), ("teacher", teacher)):
        npd.npd_head_logits(s["hidden"], s["weight"], logits_out=logits[n])
    idx = torch.empty((T, 16), dtype=torch.int32, device=dev())
    val = torch.empty((T, 16), device=dev())
    npd.npd_teacher_topk(logits["teacher"], 16, topk_idx=idx, topk_val=val, loss_mask=mask)
    g = torch.empty_like(logits["student"])
    a = [torch.empty(T, device=dev()) for _ in range(2)]
    npd.npd_kd_loss_fwd_bwd(logits["student"], mask, teacher_idx=idx, teacher_val=val, labels=labels, grad_scale=0.9,
                            ce_grad_scale=0.1, grad_out=g, kd_tok=a[0], nll_tok=a[1])
    by_logits = [torch.empty_like(student["hidden"]), torch.empty_like(student["weight"])]
    npd.npd_head_logits_bwd(g, student["hidden"], student["weight"], grad_hidden=by_logits[0], grad_weight=by_logits[1])
    b = [torch.empty(T, device=dev()) for _ in range(2)]
    direct = [torch.empty_like(t) for t in by_logits]
    npd.npd_head_loss_fwd_bwd(student["hidden"], student["weight"], mask, labels=labels, teacher_idx=idx, teacher_val=val,
                              grad_scale=0.9, ce_grad_scale=0.1, grad_hidden=direct[0], grad_weight=direct[1], kd_tok=b[0],
                              nll_tok=b[1])
    cu = torch.tensor([0, 100, 101, T], dtype=torch.int32, device=dev())
    means = [torch.empty(3, device=dev()) for _ in range(2)]
    for x, m in zip((a[1], b[1]), means):
        npd.npd_segment_reduce(x, mask, cu, seg_mean=m)
    torch.cuda.synchronize()
    # logits up to 32 in magnitude are off by 2^-8 of themselves where they are stored: two of them in each scalar
    top = logits["student"].abs().max().item()
    assert top < 32
    for x, y in zip(a, b):
        assert (x - y).abs().max().item() <= 2 * top * 2.0 ** -8
    assert (means[0] - means[1]).abs().max().item() <= 2 * top * 2.0 ** -8
    for x, y in zip(by_logits, direct):
        # (probabilities then differ by at most 2 top 2^-8 relative, and so does their part of the gradient)
        assert (x.float() - y.float()).norm() <= (2 * top * 2.0 ** -8 + 2.0 ** -7) * y.float().norm()
    full = loss64(dict(student, idx=idx, val=val), grad_scale=0.9, ce=0.1)
    for n, v in (("kd", b[0]), ("nll", b[1]), ("grad_hidden", direct[0]), ("grad_weight", direct[1])):
        near(v, full[n], n)


def placed(t, stride, offset):
    """`t` in rows `stride` apart, `offset` values behind an address of 16 bytes, with NaN around every row."""
    full = torch.full((offset + t.shape[0] * stride + 16,), NAN, dtype=t.dtype, device=t.device)
    at = full[offset:offset + t.shape[0] * stride].view(t.shape[0], stride)[:, :t.shape[1]]
    at.copy_(t)
    return at


@pytest.mark.parametrize("T", [1, 5, 8, 16, 40, 64])
@pytest.mark.parametrize("D", [3, 8, 9, 127, 129, 261])
@pytest.mark.parametrize("extra,offset", [(0, 0), (1, 0), (2, 1), (1, 1), (4, 2)])
def test_few_rows_wherever_they_begin(T, D, extra, offset):
    """Rows of the weights and of the hidden states on any multiple of two bytes; what is around a row is not seen."""
    s = inputs(T, 300, D, 3, True, mask=0.9)
    s["weight"] = placed(s["weight"], D + extra, offset)
    s["hidden"] = placed(s["hidden"], D + (extra + 1) % 3, offset // 2 * 2)
    full, out = padded(T, 300, 301)
    npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], softcap=4.0, logits_out=out)
    torch.cuda.synchronize()
    untouched(full, out)
    x, _, dx = head64(s, 4.0)
    near(out, (x, dx + 2.0 ** -8 * (x.abs() + dx)), "logits")
    check_loss(s, cap=4.0, grads=())


@pytest.mark.parametrize("T", [1, 4, 5, 8])
@pytest.mark.parametrize("V", [1, 31, 33, 64, 97, 1000])
@pytest.mark.parametrize("D", [1024, 1160, 1400])
def test_few_rows_of_a_small_vocabulary(T, V, D):
    """Workgroups whose waves share their columns: scalars, gradients, logits; parts that lie behind the vocabulary."""
    s = inputs(T, V, D, 1, True, mask=0.9)
    check_loss(s, grad_scale=0.9, ce=0.1)
    check_loss(s, tau=2.0, grads=())
    full, out = padded(T, V, V + 1)
    npd.npd_head_logits(s["hidden"], s["weight"], bias=s["bias"], logits_out=out)
    torch.cuda.synchronize()
    untouched(full, out)
    x, _, dx = head64(s, 0.0)
    near(out, (x, dx + 2.0 ** -8 * (x.abs() + dx)), "logits")
