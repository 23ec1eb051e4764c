"""The norm, the 8-bit head and the drawing of tokens on a machine without a GPU: the descriptors' layouts, workspace queries, every
refusal of the C ABI (checked before the first HIP call), and what the Python wrappers refuse before the library is called."""
import ctypes
import os
import subprocess

import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding

OK, E_NULL, E_SHAPE, E_VALUE, E_ALIAS, E_UNSUP, E_WS, E_HIP = range(8)
RMS, GX, GW, GB, ACC = 1, 2, 4, 8, 16
UNALIGNED, INT8 = 16, 3
T, V, D = 64, 200, 32
NAN, INF = float("nan"), float("inf")

# addresses that are never followed: far apart, 256-byte aligned
BASE = 1 << 32
ARGS = {n: BASE + i * (1 << 26) for i, n in enumerate(
    ["x", "w", "b", "y", "mean", "rstd", "gx", "gw", "gb", "ws", "q", "scale", "h", "hs", "weight", "wscale", "logits", "u", "mask", "tau", "k",
     "p", "m", "token", "logprob", "nll", "kept", "status"])}


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def norm_desc(**kw):
    d = dict(n_tokens=T, x_stride=D, y_stride=D, grad_x_stride=D, width=D, flags=0, eps=1e-5)
    d.update(kw)
    return binding.NormDesc(**d)


def norm(lib, d, **kw):
    a = dict(ARGS, **kw)
    return lib.npd_layer_norm(d, a["x"], a["w"], a["b"], a["y"], a["mean"], a["rstd"], None)


def norm_bwd(lib, d, ws_bytes=None, **kw):
    a = dict(ARGS, **kw)
    if ws_bytes is None:
        ws_bytes = lib.npd_layer_norm_workspace_bytes(d)
    return lib.npd_layer_norm_bwd(d, a["y"], a["x"], a["w"], a["mean"], a["rstd"], a["gx"], a["gw"], a["gb"], a["ws"], ws_bytes, None)


def quantize(lib, rows=T, width=D, x_stride=D, q_stride=D, **kw):
    a = dict(ARGS, **kw)
    return lib.npd_quantize_rows(rows, width, x_stride, q_stride, a["x"], a["q"], a["scale"], None)


def head_desc(**kw):
    d = dict(n_tokens=T + 1, vocab=V, width=D, hidden_stride=D, weight_stride=D, logits_stride=V)
    d.update(kw)
    return binding.HeadDesc(**d)


def int8(lib, d, ws_bytes=0, **kw):
    a = dict(ARGS, **kw)
    return lib.npd_head_logits_int8(d, a["h"], a["hs"], a["weight"], a["wscale"], a["b"], a["logits"], a["ws"], ws_bytes, None)


def sample_desc(**kw):
    d = dict(n_tokens=T, logits_stride=V, vocab=V, temperature=1.0, top_p=1.0)
    d.update(kw)
    return binding.SampleDesc(**d)


def sample(lib, d, ws_bytes=0, **kw):
    a = dict(ARGS, tau=None, k=None, p=None, m=None)
    a.update(kw)
    return lib.npd_sample_tokens(d, a["logits"], a["u"], a["mask"], a["tau"], a["k"], a["p"], a["m"], a["token"], a["logprob"], a["nll"],
                                 a["kept"], a["status"], a["ws"], ws_bytes, None)


def test_the_descriptors_are_the_headers(tmp_path):
    src = tmp_path / "t.c"
    exe = tmp_path / "t"
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = {"npd_norm_desc": binding.NormDesc, "npd_sample_desc": binding.SampleDesc}
    lines = [f'printf("%zu\\n", sizeof({n}));' + "".join(f'printf("%zu\\n", offsetof({n}, {f}));' for f, _ in c._fields_) for n, c in fields.items()]
    consts = ["NPD_NORM_RMS", "NPD_NORM_GRAD_X", "NPD_NORM_GRAD_WEIGHT", "NPD_NORM_GRAD_BIAS", "NPD_NORM_ACCUMULATE", "NPD_HEAD_LOGITS_INT8",
              "NPD_DEV_BAD_SAMPLING", "NPD_DEV_BAD_LOGITS"]
    lines += [f'printf("%d\\n", (int){c});' for c in consts]
    src.write_text(f'#include <stdio.h>\n#include "{root}/include/npd.h"\nint main(void) {{ {"".join(lines)} return 0; }}\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-o", str(exe), str(src)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for c in fields.values():
        want += [ctypes.sizeof(c)] + [getattr(c, f).offset for f, _ in c._fields_]
    assert got == want + [getattr(binding, c) for c in consts]


# ------------------------------------------------------------------------------------------------------------- the norm

def test_norm_refusals(lib):
    assert norm(lib, None) == E_NULL
    for name in ("x", "y"):
        assert norm(lib, norm_desc(), **{name: None}) == E_NULL
    for kw in (dict(n_tokens=0), dict(width=0), dict(n_tokens=-1), dict(x_stride=D - 1), dict(y_stride=D - 1), dict(x_stride=1 << 60),
               dict(y_stride=1 << 60)):
        assert norm(lib, norm_desc(**kw)) == E_SHAPE, kw
    for kw in (dict(n_tokens=(1 << 30) + 1), dict(width=(1 << 16) + 1, x_stride=1 << 17, y_stride=1 << 17)):
        assert norm(lib, norm_desc(**kw)) == E_UNSUP, kw
    for kw in (dict(eps=-1e-9), dict(eps=NAN), dict(eps=INF), dict(flags=GX), dict(flags=32)):
        assert norm(lib, norm_desc(**kw)) == E_VALUE, kw
    assert norm(lib, norm_desc(flags=RMS)) == E_VALUE          # a mean that is not taken
    for name, n in (("x", 1), ("w", 1), ("b", 1), ("y", 1), ("mean", 2), ("rstd", 2)):
        assert norm(lib, norm_desc(), **{name: ARGS[name] + n}) == E_VALUE, name
    for out in ("y", "mean", "rstd"):
        for other in ("x", "w", "b", "y", "mean", "rstd"):
            if out != other:
                assert norm(lib, norm_desc(), **{out: ARGS[other] + 4}) == E_ALIAS, (out, other)


def test_norm_backward_refusals(lib):
    every = GX | GW | GB
    assert norm_bwd(lib, None, 0) == E_NULL
    for name in ("x", "y", "mean", "rstd", "gx", "gw", "gb"):
        assert norm_bwd(lib, norm_desc(flags=every), **{name: None}) == E_NULL, name
    for flags, name in ((GX | GW, "gb"), (GX | GB, "gw"), (GW | GB, "gx")):
        assert norm_bwd(lib, norm_desc(flags=flags)) == E_VALUE, name
    for flags in (0, RMS, every | 32):
        assert norm_bwd(lib, norm_desc(flags=flags), 1 << 30) == E_VALUE
    assert norm_bwd(lib, norm_desc(flags=GX | ACC), gw=None, gb=None) == E_VALUE   # nothing that is added to
    assert norm_bwd(lib, norm_desc(flags=every | RMS)) == E_VALUE                  # a mean
    for kw in (dict(grad_x_stride=D - 1), dict(grad_x_stride=1 << 60), dict(x_stride=3), dict(n_tokens=0)):
        assert norm_bwd(lib, norm_desc(flags=every, **kw), 1 << 30) == E_SHAPE, kw
    for name, n in (("x", 1), ("w", 1), ("y", 1), ("mean", 2), ("rstd", 1), ("gx", 1), ("gw", 1), ("gb", 1)):
        assert norm_bwd(lib, norm_desc(flags=every), **{name: ARGS[name] + n}) == E_VALUE, name
    need = lib.npd_layer_norm_workspace_bytes(norm_desc(flags=every))
    assert norm_bwd(lib, norm_desc(flags=every), need - 1) == E_WS
    assert norm_bwd(lib, norm_desc(flags=every), need, ws=None) == E_WS
    assert norm_bwd(lib, norm_desc(flags=every), need, ws=ARGS["ws"] + 128) == E_WS
    for out in ("gx", "gw", "gb", "ws"):
        for other in ("x", "w", "y", "mean", "rstd", "gx", "gw", "gb", "ws"):
            if out != other:
                shift = 0 if out == "ws" else 4
                assert norm_bwd(lib, norm_desc(flags=every), **{out: ARGS[other] + shift}) == E_ALIAS, (out, other)


def test_norm_workspace(lib):
    size = lib.npd_layer_norm_workspace_bytes
    assert size(None) == size(norm_desc(flags=0)) == size(norm_desc(flags=GW, width=0)) == 0
    assert size(norm_desc(flags=GX)) == 0
    one = size(norm_desc(flags=GW))
    assert one > 0 and size(norm_desc(flags=GW | GB)) == 2 * one == size(norm_desc(flags=GX | GW | GB | RMS | ACC))
    large = dict(n_tokens=1 << 30, width=1 << 16, x_stride=1 << 16, y_stride=1 << 16, flags=GW | GB)
    assert size(norm_desc(**large)) == 2 * 512 * (1 << 16) * 4
    assert npd.npd_layer_norm_workspace_bytes(T, D, grad_bias=True) == 2 * one
    assert npd.npd_layer_norm_workspace_bytes(T, D, grad_weight=False) == 0
    assert npd.npd_layer_norm_workspace_bytes(T, 1 << 40) == 0


# ------------------------------------------------------------------------------------------------------- 8-bit integers

def test_quantize_refusals(lib):
    for name in ("x", "q", "scale"):
        assert quantize(lib, **{name: None}) == E_NULL
    for kw in (dict(rows=0), dict(rows=-3), dict(width=0), dict(x_stride=D - 1), dict(q_stride=D - 1), dict(x_stride=1 << 60), dict(q_stride=1 << 60)):
        assert quantize(lib, **kw) == E_SHAPE, kw
    for kw in (dict(rows=(1 << 30) + 1), dict(width=(1 << 16) + 1, x_stride=1 << 17, q_stride=1 << 17)):
        assert quantize(lib, **kw) == E_UNSUP, kw
    assert quantize(lib, x=ARGS["x"] + 1) == quantize(lib, scale=ARGS["scale"] + 2) == E_VALUE
    for out in ("q", "scale"):
        for other in ("x", "q", "scale"):
            if out != other:
                assert quantize(lib, **{out: ARGS[other] + 4}) == E_ALIAS


def test_int8_refusals(lib):
    assert int8(lib, None) == E_NULL
    for name in ("h", "hs", "weight", "wscale", "logits"):
        assert int8(lib, head_desc(), **{name: None}) == E_NULL, name
    for kw in (dict(n_tokens=0), dict(vocab=0), dict(width=-1), dict(hidden_stride=D - 1), dict(weight_stride=0), dict(logits_stride=V - 1)):
        assert int8(lib, head_desc(**kw)) == E_SHAPE, kw
    big = 1 << 22
    for kw in (dict(n_tokens=(1 << 30) + 1), dict(vocab=big, logits_stride=big), dict(width=1 << 17, hidden_stride=1 << 17, weight_stride=1 << 17),
               dict(hidden_stride=big), dict(weight_stride=big), dict(logits_stride=big)):
        assert int8(lib, head_desc(**kw)) == E_UNSUP, kw
    for kw in (dict(flags=1), dict(flags=8), dict(softcap=-1.0), dict(softcap=NAN), dict(softcap=INF), dict(softcap=1e-39)):
        assert int8(lib, head_desc(**kw)) == E_VALUE, kw
    for name, n in (("hs", 2), ("wscale", 2), ("b", 1), ("logits", 1), ("h", 8), ("weight", 4)):
        assert int8(lib, head_desc(), **{name: ARGS[name] + n}) == E_VALUE, name
    for other in ("h", "hs", "weight", "wscale", "b"):
        assert int8(lib, head_desc(), logits=ARGS[other] + 2) == E_ALIAS, other


def test_int8_workspace(lib):
    def size(**kw):
        d = head_desc(**kw)
        assert lib.npd_head_workspace_bytes(d, INT8) == lib.npd_head_workspace_bytes_preferred(d, INT8)
        return lib.npd_head_workspace_bytes(d, INT8)
    assert size() == size(hidden_stride=48, weight_stride=64) == size(n_tokens=10, flags=UNALIGNED) == size(vocab=0) == 0
    assert lib.npd_head_workspace_bytes(None, INT8) == 0
    h, w = 65 * 32, 200 * 32
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    assert size(flags=UNALIGNED) == size(width=31) == size(hidden_stride=33, weight_stride=35) == up(h) + up(w)
    assert size(hidden_stride=40) == up(h) and size(weight_stride=40) == up(w)
    for kw, need in ((dict(flags=UNALIGNED), up(h) + up(w)), (dict(width=20), up(h) + up(w))):
        d = head_desc(**kw)
        assert int8(lib, d, need - 1) == int8(lib, d, need, ws=None) == int8(lib, d, need, ws=ARGS["ws"] + 16) == E_WS
        assert int8(lib, d, need, ws=ARGS["weight"]) == int8(lib, d, need, ws=ARGS["logits"]) == E_ALIAS
    assert size(n_tokens=40, width=31) == 0   # few rows are read at any alignment
    assert npd.npd_head_workspace_bytes(INT8, 65, 200, 31) == up(h) + up(w)


# --------------------------------------------------------------------------------------------------------------- tokens

def test_sample_refusals(lib):
    assert sample(lib, None) == E_NULL
    for name in ("logits", "u", "token"):
        assert sample(lib, sample_desc(), **{name: None}) == E_NULL, name
    for kw in (dict(n_tokens=0), dict(vocab=0), dict(logits_stride=V - 1), dict(logits_stride=1 << 60)):
        assert sample(lib, sample_desc(**kw)) == E_SHAPE, kw
    for kw in (dict(n_tokens=1 << 31), dict(vocab=(1 << 26) + 1, logits_stride=1 << 27)):
        assert sample(lib, sample_desc(**kw)) == E_UNSUP, kw
    bad = [dict(flags=1), dict(top_k=-1)] + [dict(temperature=v) for v in (-0.5, NAN, INF)]
    bad += [{n: v} for n in ("top_p", "min_p") for v in (-0.1, 1.1, NAN, INF)]
    for kw in bad:
        assert sample(lib, sample_desc(**kw)) == E_VALUE, kw
    # what rows have of their own is not looked at here: the next refusal is another one's
    for kw, own in ((dict(temperature=NAN), "tau"), (dict(top_k=-1), "k"), (dict(top_p=2.0), "p"), (dict(min_p=-1.0), "m")):
        assert sample(lib, sample_desc(**kw), **{own: ARGS[own], "token": ARGS["logits"]}) == E_ALIAS
    for name in ("u", "tau", "k", "p", "m", "token", "logprob", "nll", "kept", "status"):
        assert sample(lib, sample_desc(), **{name: ARGS[name] + 2}) == E_VALUE, name
    assert sample(lib, sample_desc(), logits=ARGS["logits"] + 1) == E_VALUE
    for out in ("token", "logprob", "nll", "kept", "status"):
        for other in ("logits", "u", "mask", "token", "logprob", "nll", "kept"):
            if out != other:
                assert sample(lib, sample_desc(), **{out: ARGS[other]}) == E_ALIAS, (out, other)


def test_sample_workspace(lib):
    size = npd.npd_sample_workspace_bytes
    assert size(T, V) == size(1, 98303) == size(86, 1 << 20) == size(0, 100) == size(1, 1 << 40) == 0
    part = 4 * (7936 + 4 + 256)
    assert size(1, 98304) == 3 * part and size(1, 1 << 26) == 8 * part and size(85, 1 << 18) == 255 * part and size(40, 151936) == 160 * part
    d = sample_desc(n_tokens=4, vocab=100000, logits_stride=100000)
    need = lib.npd_sample_workspace_bytes(d)
    assert need == 12 * part
    assert sample(lib, d, need, ws=ARGS["ws"] + 128) == E_WS
    assert sample(lib, d, need, ws=ARGS["logits"]) == sample(lib, d, need, ws=ARGS["token"]) == E_ALIAS


# ---------------------------------------------------------------------------------------------------- the Python wrappers

class OnDevice(torch.Tensor):
    """A host tensor that says it is on a device."""
    index = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.index))


def tensor(*shape, dtype=torch.bfloat16, index=0):
    t = torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)
    t.index = index
    return t


@pytest.fixture
def no_device(monkeypatch):
    """The library's calls are counted, not made."""
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *a: calls.append(name) or 0

    monkeypatch.setattr(binding, "load", Library)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return calls


def arguments():
    f, i, b = torch.float32, torch.int32, torch.int8
    ws = dict(workspace=tensor(1 << 16, dtype=torch.uint8))
    return {
        npd.npd_layer_norm: dict(x=tensor(T, D), weight=tensor(D), bias=tensor(D), y_out=tensor(T, D), mean_out=tensor(T, dtype=f),
                                 rstd_out=tensor(T, dtype=f)),
        npd.npd_layer_norm_bwd: dict(grad_y=tensor(T, D), x=tensor(T, D), weight=tensor(D), mean=tensor(T, dtype=f), rstd=tensor(T, dtype=f),
                                     grad_x=tensor(T, D), grad_weight=tensor(D), grad_bias=tensor(D), **ws),
        npd.npd_quantize_rows: dict(x=tensor(T, D), q_out=tensor(T, D, dtype=b), scale_out=tensor(T, dtype=f)),
        npd.npd_head_logits_int8: dict(hidden=tensor(T, D, dtype=b), hidden_scale=tensor(T, dtype=f), weight=tensor(V, D, dtype=b),
                                       weight_scale=tensor(V, dtype=f), bias=tensor(V), logits_out=tensor(T, V), **ws),
        npd.npd_sample_tokens: dict(logits=tensor(T, V), uniform=tensor(T, dtype=f), tokens_out=tensor(T, dtype=i), temperature=tensor(T, dtype=f),
                                    top_k=tensor(T, dtype=i), top_p=tensor(T, dtype=f), min_p=tensor(T, dtype=f),
                                    loss_mask=tensor(T, dtype=torch.uint8), logprob_out=tensor(T, dtype=f), nll_out=tensor(T, dtype=f),
                                    kept_out=tensor(T, dtype=i), dev_status=tensor(1, dtype=i), **ws),
    }


CALLS = [(f, n) for f, a in arguments().items() for n in a]


@pytest.mark.parametrize("call", arguments(), ids=lambda f: f.__name__)
def test_the_calls_that_these_are_made_from(call, no_device):
    call(**arguments()[call])
    assert no_device == [call.__name__]


@pytest.mark.parametrize("call,name", CALLS, ids=lambda x: x if isinstance(x, str) else x.__name__)
def test_a_tensor_on_another_device(call, name, no_device):
    a = arguments()[call]
    a[name].index = 1
    with pytest.raises(ValueError, match="cuda:1"):
        call(**a)
    assert not no_device


@pytest.mark.parametrize("call,name", CALLS, ids=lambda x: x if isinstance(x, str) else x.__name__)
def test_a_tensor_of_another_kind(call, name, no_device):
    """A type, a size or a layout that the call does not take; a tensor in host memory."""
    if name == "workspace":
        bad = [tensor(1 << 13, dtype=torch.uint8)[::2]]
    else:
        t = arguments()[call][name]
        shape = list(t.shape)
        other = torch.float64
        bad = [tensor(*shape, dtype=other), tensor(*(shape[:-1] + [2 * shape[-1]]), dtype=t.dtype)[..., ::2], torch.zeros(shape, dtype=t.dtype)]
        if (call, name) not in ((npd.npd_layer_norm, "x"), (npd.npd_quantize_rows, "x"), (npd.npd_sample_tokens, "logits")) and name not in (
                "hidden", "weight") or t.dim() == 1:
            bad.append(tensor(*(shape[:-1] + [shape[-1] + 1]), dtype=t.dtype))
    for t in bad:
        if name == "dev_status" and t.dtype is torch.int32 and t.is_contiguous() and isinstance(t, OnDevice) and t.numel() == 1:
            continue
        with pytest.raises(ValueError):
            call(**dict(arguments()[call], **{name: t}))
    assert not [n for n in no_device if n == call.__name__]


def test_sizes_beyond_the_descriptors_fields(monkeypatch):
    """2^32 + 5 columns are not five."""
    monkeypatch.setattr(binding, "_matrix", lambda name, t, shape, dtype=None: None if t is None else 4096)
    monkeypatch.setattr(binding, "_array", lambda name, t, n, dtype: None if t is None else 4096)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    n = (1 << 32) + 5
    wide = tensor(1, 1).expand(T, n)
    f = torch.float32
    calls = [lambda: npd.npd_layer_norm(wide, y_out=wide), lambda: npd.npd_quantize_rows(wide, q_out=wide, scale_out=tensor(T, dtype=f)),
             lambda: npd.npd_layer_norm_bwd(wide, wide, rstd=tensor(T, dtype=f), rms=True, grad_x=wide),
             lambda: npd.npd_head_logits_int8(wide, tensor(T, dtype=f), wide, tensor(T, dtype=f), logits_out=tensor(T, T)),
             lambda: npd.npd_sample_tokens(wide, tensor(T, dtype=f), tokens_out=tensor(T, dtype=torch.int32))]
    for call in calls:
        with pytest.raises(binding.NpdError) as e:
            call()
        assert e.value.status in (E_UNSUP, E_SHAPE)


@pytest.mark.parametrize("kw", [dict(temperature=-1.0), dict(temperature=NAN), dict(top_k=-5), dict(top_k=-(1 << 40)), dict(top_p=1.5), dict(min_p=-0.1)])
def test_sampling_numbers_out_of_range(kw, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    with pytest.raises(binding.NpdError) as e:
        npd.npd_sample_tokens(tensor(T, V), tensor(T, dtype=torch.float32), tokens_out=tensor(T, dtype=torch.int32), **kw)
    assert e.value.status == E_VALUE
