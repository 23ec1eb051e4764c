"""The Python wrappers of the head operators without a GPU: what they refuse before the library is called."""
import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding

T, V, D, K = 4, 50, 16, 3
LOAD = binding.load


class OnDevice(torch.Tensor):
    """A host tensor that says it is on a device."""
    index = 0
    is_cuda = property(lambda self: True)
    device = property(lambda self: torch.device("cuda", self.index))


def tensor(*shape, dtype=torch.bfloat16, index=0):
    t = torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)
    t.index = index
    return t


@pytest.fixture(autouse=True)
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
    f, i = torch.float32, torch.int32
    scalars = {n: tensor(T, dtype=f) for n in ("kd_tok", "nll_tok", "lse_tok")}
    bias, ws = dict(bias=tensor(V)), dict(workspace=tensor(1 << 20, dtype=torch.uint8))
    grads = dict(grad_hidden=tensor(T, D), grad_weight=tensor(V, D), grad_bias=tensor(V))
    both = dict(hidden=tensor(T, D), weight=tensor(V, D))
    return {
        npd.npd_head_loss_fwd_bwd: dict(**both, loss_mask=tensor(T, dtype=torch.uint8), labels=tensor(T, dtype=i),
                                        teacher_idx=tensor(T, K, dtype=i), teacher_val=tensor(T, K, dtype=f),
                                        dev_status=tensor(1, dtype=i), **bias, **grads, **scalars, **ws),
        npd.npd_head_logits: dict(**both, logits_out=tensor(T, V), **bias, **ws),
        npd.npd_head_logits_bwd: dict(grad_logits=tensor(T, V), **both, logits=tensor(T, V), softcap=30.0, **grads, **ws),
    }


CALLS = [(f, n) for f, a in arguments().items() for n, t in a.items() if isinstance(t, torch.Tensor)]


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


def test_logits_that_a_call_has_no_use_for(no_device):
    a = arguments()[npd.npd_head_logits_bwd]
    a.update(softcap=0.0)
    a["logits"].index = 1
    npd.npd_head_logits_bwd(**a)
    assert no_device == ["npd_head_logits_bwd"]


@pytest.mark.parametrize("call", arguments(), ids=lambda f: f.__name__)
def test_a_workspace_in_pieces(call, no_device):
    """What counts is the memory behind a workspace's address, not its number of elements."""
    for ws in (tensor(256, dtype=torch.uint8).expand(1 << 12, 256), tensor(1 << 13, dtype=torch.uint8)[::2]):
        with pytest.raises(ValueError, match="workspace"):
            call(**dict(arguments()[call], workspace=ws))
    assert not no_device


@pytest.mark.parametrize("call", arguments(), ids=lambda f: f.__name__)
@pytest.mark.parametrize("V,D", [((1 << 32) + 5, 1), (5, (1 << 32) + 3)])
def test_sizes_beyond_the_descriptors_fields(call, V, D, monkeypatch):
    """2^32 + 5 rows are not five."""
    monkeypatch.setattr(binding, "load", LOAD)

    def matrix(rows, cols):
        return tensor(1, 1).expand(rows, cols) if max(rows, cols) > 1 << 31 else tensor(rows, cols)

    monkeypatch.setattr(binding, "_matrix", lambda name, t, shape: None if t is None else 4096)
    weight, hidden = matrix(V, D), matrix(T, D)
    monkeypatch.setattr(binding, "_array", lambda name, t, n, dtype: None if t is None else 4096)
    a = dict(hidden=hidden, weight=weight)
    if call is npd.npd_head_loss_fwd_bwd:
        a.update(loss_mask=tensor(T, dtype=torch.uint8), lse_tok=tensor(T, dtype=torch.float32))
    elif call is npd.npd_head_logits:
        a.update(logits_out=matrix(T, V))
    else:
        a.update(grad_logits=matrix(T, V), grad_bias=tensor(5))
    with pytest.raises(binding.NpdError) as e:
        call(**a)
    assert e.value.status == 5   # not supported


def test_a_record_beyond_the_descriptors_field(monkeypatch):
    monkeypatch.setattr(binding, "load", LOAD)
    a = arguments()[npd.npd_head_loss_fwd_bwd]
    k = (1 << 32) + 2
    for name, dtype in (("teacher_idx", torch.int32), ("teacher_val", torch.float32)):
        a[name] = tensor(1, 1, dtype=dtype).expand(T, k)
        monkeypatch.setattr(OnDevice, "is_contiguous", lambda self: True, raising=False)
    with pytest.raises(binding.NpdError) as e:
        npd.npd_head_loss_fwd_bwd(**a)
    assert e.value.status == 2   # more ids than the vocabulary has


def test_the_workspace_that_a_call_takes(monkeypatch):
    """The function's answers are those for the descriptors that the calls make: one byte less is refused as too small."""
    L = LOAD()

    class Library:
        """Host checks alone: a call that would be made on the device ends here."""
        def __getattr__(self, name):
            f = getattr(L, name)
            return (lambda *a: f(*a[:-1], None) if a[-2] < need else 0) if name == call.__name__ else f

    monkeypatch.setattr(binding, "load", Library)
    ops = {npd.npd_head_loss_fwd_bwd: binding.NPD_HEAD_LOSS, npd.npd_head_logits: binding.NPD_HEAD_LOGITS,
           npd.npd_head_logits_bwd: binding.NPD_HEAD_LOGITS_BWD}
    n, w = 100, 13   # (rows that are copied)
    for call, op in ops.items():
        a = arguments()[call]
        for name, t in a.items():
            if isinstance(t, torch.Tensor) and name != "workspace":
                shape = [n if s == T else w if s == D else s for s in t.shape]
                a[name] = tensor(*shape, dtype=t.dtype)
        flags = 0 if op == binding.NPD_HEAD_LOGITS else 7
        if any(isinstance(t, torch.Tensor) and t.data_ptr() & 15 for t in a.values()):
            flags |= binding.NPD_HEAD_UNALIGNED
        how = dict(topk=K if op == binding.NPD_HEAD_LOSS else 0, flags=flags, softcap=a.get("softcap", 0.0))
        need = npd.npd_head_workspace_bytes(op, n, V, w, **how)
        assert 0 < need <= npd.npd_head_workspace_bytes(op, n, V, w, preferred=True, **how)
        room = torch.zeros(need + 256, dtype=torch.uint8)
        room = room[-room.data_ptr() % 256:][:need].as_subclass(OnDevice)
        call(**dict(a, workspace=room))
        with pytest.raises(binding.NpdError) as e:
            call(**dict(a, workspace=room[:-1]))
        assert e.value.status == 6
    assert npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOSS, 0, V, D) == 0


def test_one_row_has_no_stride(monkeypatch):
    """As in the calls: the rows of a padded buffer, one of which is taken."""
    monkeypatch.setattr(binding, "load", LOAD)
    size = npd.npd_head_workspace_bytes
    for op in (binding.NPD_HEAD_LOSS, binding.NPD_HEAD_LOGITS, binding.NPD_HEAD_LOGITS_BWD):
        flags = 0 if op == binding.NPD_HEAD_LOGITS else 7
        one = size(op, 1, 1000, 64, flags=flags)
        assert size(op, 1, 1000, 64, flags=flags, hidden_stride=67, logits_stride=1003) == one
        assert size(op, 100, 1, 64, flags=flags, weight_stride=67) == size(op, 100, 1, 64, flags=flags)
