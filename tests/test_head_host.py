"""Head operators on a machine without a GPU: the descriptor's layout, workspace queries, and every refusal of the C ABI (checked
before the first HIP call) and of the Python wrappers."""
import ctypes
import subprocess

import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding
from head_util import bwd64, inputs, loss64

OK, E_NULL, E_SHAPE, E_VALUE, E_ALIAS, E_UNSUP, E_WS, E_HIP = range(8)
LOSS, LOGITS, BWD = 0, 1, 2
GH, GW, GB, ACC, UNALIGNED = 1, 2, 4, 8, 16
T, V, D, K = 64, 200, 32, 4


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def desc(**kw):
    d = dict(n_tokens=T, vocab=V, width=D, hidden_stride=D, weight_stride=D, grad_hidden_stride=D, grad_weight_stride=D,
             logits_stride=V, topk=K, flags=GH | GW | GB, tau=1.0, grad_scale=0.9, ce_grad_scale=0.1, softcap=0.0)
    d.update(kw)
    return binding.HeadDesc(**d)


# addresses that are never followed: far apart, 256-byte aligned
BASE = 1 << 32
ARGS = {n: BASE + i * (1 << 26) for i, n in enumerate(
    ["hidden", "weight", "bias", "labels", "idx", "val", "mask", "gh", "gw", "gb", "kd", "nll", "lse", "status", "ws", "logits",
     "glogits"])}


def loss(lib, d, ws_bytes=None, **kw):
    a = dict(ARGS, **kw)
    if ws_bytes is None:
        ws_bytes = lib.npd_head_workspace_bytes(d, LOSS)
    return lib.npd_head_loss_fwd_bwd(d, a["hidden"], a["weight"], a["bias"], a["labels"], a["idx"], a["val"], a["mask"], a["gh"],
                                     a["gw"], a["gb"], a["kd"], a["nll"], a["lse"], a["status"], a["ws"], ws_bytes, None)


def logits(lib, d, ws_bytes=0, **kw):
    a = dict(ARGS, **kw)
    return lib.npd_head_logits(d, a["hidden"], a["weight"], a["bias"], a["logits"], a["ws"], ws_bytes, None)


def backward(lib, d, ws_bytes=None, **kw):
    a = dict(ARGS, logits=None)
    a.update(kw)
    if ws_bytes is None:
        ws_bytes = lib.npd_head_workspace_bytes(d, BWD)
    return lib.npd_head_logits_bwd(d, a["glogits"], a["logits"], a["hidden"], a["weight"], a["gh"], a["gw"], a["gb"], a["ws"],
                                   ws_bytes, None)


def test_the_descriptor_is_the_headers(tmp_path):
    src = tmp_path / "use.c"
    fields = [f for f, _ in binding.HeadDesc._fields_]
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "npd.h"\nint main(void) {\n' +
                   'printf("%zu", sizeof(npd_head_desc));\n' +
                   "".join(f'printf(" %zu", offsetof(npd_head_desc, {f}));\n' for f in fields) + "return 0; }\n")
    root = __import__("os").path.dirname(__import__("os").path.dirname(__import__("os").path.abspath(__file__)))
    exe = tmp_path / "use"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", f"-I{root}/include", "-o", str(exe), str(src)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, check=True, text=True).stdout.split()]
    assert got == [ctypes.sizeof(binding.HeadDesc)] + [getattr(binding.HeadDesc, f).offset for f in fields]


@pytest.mark.parametrize("bad,status", [
    (dict(n_tokens=0), E_SHAPE), (dict(vocab=0), E_SHAPE), (dict(width=0), E_SHAPE), (dict(n_tokens=-3), E_SHAPE),
    (dict(n_tokens=(1 << 30) + 1), E_UNSUP), (dict(vocab=(1 << 21) + 1, logits_stride=(1 << 21) + 1), E_UNSUP),
    (dict(width=(1 << 16) + 1), E_UNSUP), (dict(hidden_stride=D - 1), E_SHAPE), (dict(weight_stride=D - 1), E_SHAPE),
    (dict(grad_hidden_stride=D - 1), E_SHAPE), (dict(grad_weight_stride=0), E_SHAPE),
    (dict(hidden_stride=(1 << 21) + 8), E_UNSUP), (dict(weight_stride=1 << 40), E_UNSUP),
    (dict(topk=-1), E_SHAPE), (dict(topk=V + 1), E_SHAPE), (dict(vocab=8192, topk=4097), E_UNSUP),
    (dict(tau=0.0), E_VALUE), (dict(tau=float("nan")), E_VALUE), (dict(tau=float("inf")), E_VALUE),
    (dict(grad_scale=float("inf")), E_VALUE), (dict(ce_grad_scale=float("nan")), E_VALUE),
    (dict(softcap=-1.0), E_VALUE), (dict(softcap=float("inf")), E_VALUE), (dict(softcap=float("nan")), E_VALUE),
    (dict(flags=32), E_VALUE), (dict(flags=ACC), E_VALUE), (dict(flags=ACC | GH), E_VALUE),
    (dict(flags=0), E_VALUE),                                    # a CE gradient without one
    (dict(topk=0, ce_grad_scale=0.0), E_VALUE),                  # nothing to differentiate
    (dict(tau=2.0), E_UNSUP),                                    # CE at a temperature
    (dict(ce_grad_scale=-0.1), E_UNSUP),                         # weights of opposite sign
])
def test_loss_refuses_bad_descriptors(lib, bad, status):
    d = desc(**bad)
    assert lib.npd_head_workspace_bytes(d, LOSS) == lib.npd_head_workspace_bytes_preferred(d, LOSS) == 0
    assert loss(lib, d, 1 << 25) == status


def test_null_descriptor_and_unknown_operation(lib):
    assert loss(lib, None, 0) == logits(lib, None) == backward(lib, None, 0) == E_NULL
    assert lib.npd_head_workspace_bytes(None, LOSS) == lib.npd_head_workspace_bytes(desc(), 7) == 0


@pytest.mark.parametrize("bad,status", [
    (dict(hidden=None), E_NULL), (dict(weight=None), E_NULL), (dict(mask=None), E_NULL), (dict(labels=None), E_NULL),
    (dict(idx=None), E_NULL), (dict(val=None), E_NULL), (dict(gh=None), E_NULL), (dict(gw=None), E_NULL), (dict(gb=None), E_NULL),
    (dict(hidden=BASE + 1), E_VALUE), (dict(hidden=BASE + 2), E_VALUE), (dict(weight=ARGS["weight"] + 8), E_VALUE),
    (dict(bias=ARGS["bias"] + 1), E_VALUE), (dict(labels=ARGS["labels"] + 2), E_VALUE), (dict(idx=ARGS["idx"] + 1), E_VALUE),
    (dict(val=ARGS["val"] + 2), E_VALUE), (dict(gh=ARGS["gh"] + 1), E_VALUE), (dict(gw=ARGS["gw"] + 1), E_VALUE),
    (dict(gb=ARGS["gb"] + 1), E_VALUE), (dict(kd=ARGS["kd"] + 2), E_VALUE), (dict(nll=ARGS["nll"] + 1), E_VALUE),
    (dict(lse=ARGS["lse"] + 2), E_VALUE), (dict(status=ARGS["status"] + 2), E_VALUE),
    (dict(ws=None), E_WS), (dict(ws=ARGS["ws"] + 128), E_WS), (dict(ws_bytes=1000), E_WS),
    (dict(gh=ARGS["hidden"]), E_ALIAS), (dict(gw=ARGS["weight"]), E_ALIAS), (dict(gw=ARGS["gh"] + 64), E_ALIAS),
    (dict(kd=ARGS["nll"]), E_ALIAS), (dict(lse=ARGS["val"] + 16), E_ALIAS), (dict(ws=ARGS["weight"]), E_ALIAS),
    (dict(status=ARGS["mask"] + 4), E_ALIAS), (dict(gb=ARGS["bias"]), E_ALIAS), (dict(ws=ARGS["gw"]), E_ALIAS),
])
def test_loss_refuses_bad_arguments(lib, bad, status):
    assert loss(lib, desc(), **bad) == status


def test_loss_refuses_what_does_not_go_together(lib):
    assert loss(lib, desc(flags=GH), gw=None) == E_VALUE                       # a gradient without its flag
    none = dict(idx=None, val=None, kd=None)
    assert loss(lib, desc(topk=0), **dict(none, kd=ARGS["kd"])) == E_VALUE     # a KL without a teacher
    assert loss(lib, desc(topk=0), **dict(none, idx=ARGS["idx"])) == E_VALUE
    quiet = dict(gh=None, gw=None, gb=None)
    warm = desc(flags=0, tau=2.0, ce_grad_scale=0.0)
    assert loss(lib, warm, **quiet) == E_UNSUP                                 # NLL and log-sum-exp belong to tau = 1
    assert loss(lib, warm, nll=None, **quiet) == E_UNSUP
    assert loss(lib, warm, lse=None, **quiet) == E_UNSUP
    # tensors at any address, once the flag says so: refused for what is wrong besides
    odd = desc(flags=GH | GW | GB | UNALIGNED)
    assert loss(lib, odd, hidden=BASE + 2, ws=None) == E_WS
    assert loss(lib, odd, hidden=BASE + 1) == E_VALUE


@pytest.mark.parametrize("bad,status", [
    (dict(flags=GH), E_VALUE), (dict(logits_stride=V - 1), E_SHAPE), (dict(logits_stride=(1 << 21) + 1), E_UNSUP),
    (dict(hidden_stride=1), E_SHAPE), (dict(weight_stride=1), E_SHAPE), (dict(softcap=-2.0), E_VALUE), (dict(vocab=-1), E_SHAPE)])
def test_logits_refuse_bad_descriptors(lib, bad, status):
    assert logits(lib, desc(**dict(dict(flags=0), **bad))) == status


@pytest.mark.parametrize("bad,status", [
    (dict(hidden=None), E_NULL), (dict(weight=None), E_NULL), (dict(logits=None), E_NULL), (dict(hidden=BASE + 8), E_VALUE),
    (dict(weight=ARGS["weight"] + 2), E_VALUE), (dict(logits=ARGS["logits"] + 1), E_VALUE), (dict(bias=ARGS["bias"] + 1), E_VALUE),
    (dict(logits=ARGS["weight"] + 256), E_ALIAS), (dict(logits=ARGS["hidden"]), E_ALIAS)])
def test_logits_refuse_bad_arguments(lib, bad, status):
    assert logits(lib, desc(flags=0), **bad) == status


def test_logits_of_unaligned_tensors_need_a_workspace(lib):
    d = desc(flags=UNALIGNED, n_tokens=100)
    need = lib.npd_head_workspace_bytes(d, LOGITS)
    assert need >= (100 + V) * D * 2
    assert logits(lib, d, need - 1, hidden=BASE + 2) == E_WS
    assert logits(lib, d, need, hidden=BASE + 2, ws=None) == E_WS
    assert lib.npd_head_workspace_bytes(desc(flags=0, n_tokens=100), LOGITS) == 0
    # few rows read the weights where they lie
    assert lib.npd_head_workspace_bytes(desc(flags=UNALIGNED, n_tokens=64), LOGITS) == 0


@pytest.mark.parametrize("bad,status", [
    (dict(flags=0), E_VALUE), (dict(logits_stride=V - 1), E_SHAPE), (dict(grad_hidden_stride=1), E_SHAPE),
    (dict(grad_weight_stride=1), E_SHAPE), (dict(hidden_stride=1), E_SHAPE), (dict(weight_stride=1), E_SHAPE),
    (dict(flags=GH | GW | GB | 64), E_VALUE), (dict(softcap=float("nan")), E_VALUE)])
def test_backward_refuses_bad_descriptors(lib, bad, status):
    assert backward(lib, desc(**bad), 1 << 25) == status


@pytest.mark.parametrize("bad,status", [
    (dict(glogits=None), E_NULL), (dict(hidden=None), E_NULL), (dict(weight=None), E_NULL), (dict(gh=None), E_NULL),
    (dict(gb=None), E_NULL), (dict(logits=ARGS["logits"]), E_VALUE), (dict(glogits=ARGS["glogits"] + 4), E_VALUE),
    (dict(hidden=BASE + 2), E_VALUE), (dict(weight=ARGS["weight"] + 2), E_VALUE), (dict(gw=ARGS["gw"] + 1), E_VALUE),
    (dict(gh=ARGS["glogits"]), E_ALIAS), (dict(gw=ARGS["hidden"]), E_ALIAS), (dict(gb=ARGS["gw"]), E_ALIAS),
    (dict(ws=None), E_WS), (dict(ws_bytes=100), E_WS), (dict(ws=ARGS["glogits"]), E_ALIAS)])
def test_backward_refuses_bad_arguments(lib, bad, status):
    assert backward(lib, desc(), **bad) == status


def test_backward_with_a_soft_cap_needs_the_logits(lib):
    assert backward(lib, desc(softcap=30.0)) == E_NULL
    assert backward(lib, desc(softcap=30.0), logits=ARGS["gw"]) == E_ALIAS
    # strides and pointers of tensors that a call does not have are not looked at
    assert backward(lib, desc(flags=GB, hidden_stride=0, weight_stride=0), hidden=None, weight=None, gh=None, gw=None,
                    glogits=ARGS["glogits"] + 1) == E_VALUE


@pytest.mark.parametrize("op", [LOSS, BWD])
def test_workspace_sizes(lib, op):
    """The least is what the shortest useful chunks take, the preferred amount what 8,192 rows do; neither grows with the rows
    beyond that but for the list of positions."""
    def sizes(n, **kw):
        d = desc(n_tokens=n, vocab=5003, logits_stride=5003, **kw)
        return lib.npd_head_workspace_bytes(d, op), lib.npd_head_workspace_bytes_preferred(d, op)
    for n in (1, 1000, 1024, 1025, 8192, 8193, 100000):
        least, most = sizes(n)
        assert 0 < least <= most
    a, b = sizes(20000)[1], sizes(40000)[1]
    assert b - a <= 20000 * 4 + 512
    # forward only: no copy of the gradient, 5,003 x 2 bytes a row
    if op == LOSS:
        assert sizes(8192)[1] - sizes(8192, flags=0, ce_grad_scale=0.0)[1] >= 8192 * 5003 * 2


def test_the_wrappers_refuse(monkeypatch):
    h, w = torch.zeros((4, 16), dtype=torch.bfloat16), torch.zeros((50, 16), dtype=torch.bfloat16)
    m = torch.ones(4, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device tensors"):
        npd.npd_head_loss_fwd_bwd(h, w, m)
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype=None: None if t is None else t.data_ptr())
    with pytest.raises(ValueError, match="weight"):
        npd.npd_head_loss_fwd_bwd(h, w[:, :8], m)
    with pytest.raises(ValueError, match="teacher_idx"):
        npd.npd_head_loss_fwd_bwd(h, w, m, teacher_idx=torch.zeros((4, 3), dtype=torch.int32))
    with pytest.raises(ValueError, match="teacher_idx"):
        npd.npd_head_loss_fwd_bwd(h, w, m, teacher_idx=torch.zeros((3, 3), dtype=torch.int32), teacher_val=torch.zeros((3, 3)))
    with pytest.raises(ValueError, match="hidden"):
        npd.npd_head_logits(h.T, w[:, :4].contiguous(), logits_out=torch.zeros((16, 50), dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="row stride"):
        npd.npd_head_logits_bwd(torch.zeros((4, 50)), h, w, logits=torch.zeros((4, 60))[:, :50], softcap=1.0)


def test_the_formulas_against_differences():
    """The 64-bit gradients that the GPU tests compare with are those of the 64-bit loss (central differences)."""
    s = inputs(5, 40, 12, 4, True, device="cpu")
    s["mask"] = torch.tensor([1, 0, 1, 1, 0], dtype=torch.uint8)
    for cap, tau, gs, ce in ((0.0, 1.0, 0.9, 0.1), (3.0, 1.0, 0.9, 0.1), (0.0, 2.0, 1.0, 0.0), (3.0, 0.5, 1.0, 0.0)):
        want = loss64(s, cap=cap, tau=tau, grad_scale=gs, ce=ce)

        def value(t):
            o = loss64(t, cap=cap, tau=tau)
            return (gs * o["kd"][0] + (ce * o["nll"][0] if ce else 0.0)).sum().item()

        step = 1e-5
        for name, key in (("hidden", "grad_hidden"), ("weight", "grad_weight"), ("bias", "grad_bias")):
            g = want[key][0].reshape(-1)
            for i in range(0, g.numel(), max(1, g.numel() // 17)):
                f = []
                for sign in (1, -1):
                    t = dict(s, **{name: s[name].double().clone()})
                    t[name].view(-1)[i] += sign * step
                    f.append(value(t))
                assert abs((f[0] - f[1]) / (2 * step) - g[i].item()) <= 1e-7 + 1e-6 * abs(g[i].item()), (name, i)


def test_the_backward_formula_against_differences():
    s = inputs(4, 30, 10, 0, True, device="cpu")
    cap, r = 2.0, torch.randn((4, 30), dtype=torch.float64)
    r = r.to(torch.bfloat16)

    def out(t):
        z = t["hidden"].double() @ t["weight"].double().T + t["bias"].double()
        return cap * torch.tanh(z / cap)

    want = bwd64(r, s, out(s), cap)
    step = 1e-5
    for name, key in (("hidden", "grad_hidden"), ("weight", "grad_weight"), ("bias", "grad_bias")):
        g = want[key][0].reshape(-1)
        for i in range(0, g.numel(), max(1, g.numel() // 11)):
            f = []
            for sign in (1, -1):
                t = dict(s, **{name: s[name].double().clone()})
                t[name].view(-1)[i] += sign * step
                f.append((r.double() * out(t)).sum().item())
            assert abs((f[0] - f[1]) / (2 * step) - g[i].item()) <= 1e-7 + 1e-6 * abs(g[i].item()), (name, i)
