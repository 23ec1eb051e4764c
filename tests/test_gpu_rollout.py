"""The operators around the head together, as a program calls them: a step of a rollout (norm, 8-bit hidden states, 8-bit head, token),
and a training step through the norm and the head's loss.

The rollout's tokens are checked against those drawn, in 64 bits, from the logits that the call left (which other tests check), the
training step's gradients against the loss in 64 bits of the same bf16 inputs and the hidden states that the norm left.
"""
import numpy as np
import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding
from sample_util import draw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B = 2.0 ** -8


def model(V, D, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    weight = (torch.randn((V, D), device=DEV, generator=g) * (3 / D ** 0.5)).to(torch.bfloat16)
    norm = (1 + 0.2 * torch.randn(D, device=DEV, generator=g)).to(torch.bfloat16)
    return weight, norm, g


class Rollout:
    """The buffers of a step for T sequences: the head's 8-bit weights, in rows that begin on 16 bytes, are laid out once."""

    def __init__(self, weight, norm, T):
        V, D = weight.shape
        S = (D + 15) // 16 * 16
        self.norm = norm
        self.weight_q = torch.empty((V, S), dtype=torch.int8, device=DEV)[:, :D]
        self.weight_scale = torch.empty(V, device=DEV)
        npd.npd_quantize_rows(weight, q_out=self.weight_q, scale_out=self.weight_scale)
        self.y = torch.empty((T, D), dtype=torch.bfloat16, device=DEV)
        self.q = torch.empty((T, S), dtype=torch.int8, device=DEV)[:, :D]
        self.scale = torch.empty(T, device=DEV)
        self.logits = torch.empty((T, V), dtype=torch.bfloat16, device=DEV)
        self.tokens = torch.empty(T, dtype=torch.int32, device=DEV)
        self.nll, self.logprob = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        self.kept = torch.empty(T, dtype=torch.int32, device=DEV)
        self.int8_ws = torch.empty(npd.npd_head_workspace_bytes(binding.NPD_HEAD_LOGITS_INT8, T, V, D, hidden_stride=S, weight_stride=S),
                                   dtype=torch.uint8, device=DEV)
        self.sample_ws = torch.empty(npd.npd_sample_workspace_bytes(T, V), dtype=torch.uint8, device=DEV)

    def step(self, x, u, mask):
        npd.npd_layer_norm(x, self.norm, y_out=self.y, rms=True, eps=1e-6)
        npd.npd_quantize_rows(self.y, q_out=self.q, scale_out=self.scale)
        npd.npd_head_logits_int8(self.q, self.scale, self.weight_q, self.weight_scale, logits_out=self.logits, workspace=self.int8_ws)
        npd.npd_sample_tokens(self.logits, u, temperature=0.8, top_k=40, top_p=0.95, loss_mask=mask, tokens_out=self.tokens,
                              logprob_out=self.logprob, nll_out=self.nll, kept_out=self.kept, workspace=self.sample_ws)

    def outputs(self):
        return [t.clone() for t in (self.logits, self.tokens, self.nll, self.logprob, self.kept)]


@pytest.mark.parametrize("T,V,D", [(1, 100000, 512), (7, 3000, 200), (70, 1000, 1000), (300, 5000, 64)])
def test_a_step_of_a_rollout(T, V, D):
    weight, norm, g = model(V, D)
    x = torch.randn((T, D), device=DEV, generator=g).to(torch.bfloat16)
    u = torch.rand(T, device=DEV, generator=g)
    mask = (torch.rand(T, device=DEV, generator=g) < 0.8).to(torch.uint8)
    mask[0] = 1
    r = Rollout(weight, norm, T)
    r.step(x, u, mask)
    rows, us, on = r.logits.double().cpu().numpy(), u.double().cpu().numpy(), mask.cpu().numpy()
    for t in range(T):
        got = (int(r.tokens[t]), int(r.kept[t]))
        if not on[t]:
            assert got == (-1, 0) and float(r.nll[t]) == 0
            continue
        token, kept, logprob, nll = draw(rows[t], us[t], float(np.float32(0.8)), 40, float(np.float32(0.95)), 0.0)
        assert got == (token, kept)
        assert abs(float(r.nll[t]) - nll) <= 2.0 ** -24 * nll + 1e-11
    # the logits against 64-bit ones of the unquantised head: of 127 steps to a row's largest value each operand is off by half a step at
    # most, over D products of independent signs; five standard deviations of (a / 254)^2 |w|^2 + |h|^2 (b / 254)^2, and bf16
    h, w = r.y.double(), weight.double()
    exact = h @ w.t()
    a, b = h.abs().amax(1, keepdim=True) / 254, w.abs().amax(1)[None] / 254
    deviation = torch.sqrt((a * w.norm(dim=1)[None]) ** 2 + (b * h.norm(dim=1)[:, None]) ** 2 + D * (a * b) ** 2)
    assert bool(((r.logits.double() - exact).abs() <= 5 * deviation + B * exact.abs() + 1e-6).all())


@pytest.mark.parametrize("T", [1, 40, 130])
def test_captured_steps(T):
    """Two steps captured with buffers of their own, replayed with other inputs, side by side, and with eager steps between."""
    V, D = 99000, 300
    weight, norm, g = model(V, D)
    sets = [(torch.randn((T, D), device=DEV, generator=g).to(torch.bfloat16), torch.rand(T, device=DEV, generator=g)) for _ in range(3)]
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    eager = Rollout(weight, norm, T)
    want = []
    for x, u in sets:
        eager.step(x, u, mask)
        want.append(eager.outputs())
    held = []
    for _ in range(2):
        r, x, u = Rollout(weight, norm, T), sets[0][0].clone(), sets[0][1].clone()
        r.step(x, u, mask)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            r.step(x, u, mask)
        held.append((r, x, u, graph, torch.cuda.Stream()))
    for a, b in ((0, 1), (2, 0), (1, 1), (0, 2)):
        for (_, x, u, _, _), i in zip(held, (a, b)):
            x.copy_(sets[i][0])
            u.copy_(sets[i][1])
        torch.cuda.synchronize()
        for _, _, _, graph, stream in held:
            with torch.cuda.stream(stream):
                graph.replay()
        eager.step(*sets[a], mask)
        torch.cuda.synchronize()
        for (r, _, _, _, _), i in zip(held, (a, b)):
            assert all(torch.equal(p, q) for p, q in zip(r.outputs(), want[i]))
        assert all(torch.equal(p, q) for p, q in zip(eager.outputs(), want[a]))


@pytest.mark.parametrize("rms", [False, True])
def test_a_training_step_through_norm_and_head(rms):
    T, V, D = 96, 1500, 256
    weight, norm_w, g = model(V, D)
    norm_b = None if rms else (0.1 * torch.randn(D, device=DEV, generator=g)).to(torch.bfloat16)
    x = torch.randn((T, D), device=DEV, generator=g).to(torch.bfloat16)
    labels = torch.randint(0, V, (T,), device=DEV, generator=g, dtype=torch.int32)
    mask = (torch.rand(T, device=DEV, generator=g) < 0.7).to(torch.uint8)
    n = int(mask.sum())
    h = torch.empty_like(x)
    mean, rstd = None if rms else torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    npd.npd_layer_norm(x, norm_w, bias=norm_b, rms=rms, eps=1e-6, y_out=h, mean_out=mean, rstd_out=rstd)
    grad_h, grad_w = torch.empty_like(h), torch.empty_like(weight)
    nll = torch.empty(T, device=DEV)
    npd.npd_head_loss_fwd_bwd(h, weight, mask, labels=labels, ce_grad_scale=1.0 / n, grad_hidden=grad_h, grad_weight=grad_w, nll_tok=nll)
    out = dict(grad_x=torch.empty_like(x), grad_weight=torch.empty_like(norm_w))
    if not rms:
        out["grad_bias"] = torch.empty_like(norm_b)
    npd.npd_layer_norm_bwd(grad_h, x, norm_w, mean=mean, rstd=rstd, rms=rms, **out)

    xs, ws = x.double().requires_grad_(), norm_w.double().requires_grad_()
    bs = None if rms else norm_b.double().requires_grad_()
    c = xs if rms else xs - xs.mean(1, keepdim=True)
    y = c * torch.rsqrt((c * c).mean(1, keepdim=True) + 1e-6) * ws
    y = y if rms else y + bs
    y = y + (h.double() - y).detach()          # the hidden states as they were rounded
    z = y @ weight.double().t()
    loss = (torch.nn.functional.cross_entropy(z, labels.long(), reduction="none") * mask).sum() / n
    loss.backward()
    # a gradient's relative error (in its norm): the hidden states' gradient is within .004 of itself (operands and result rounded
    # to bf16, B each at most), which the norm's backward pass, linear in it, passes on, and rounds once more
    for name, want in (("grad_x", xs.grad), ("grad_weight", ws.grad), ("grad_bias", None if rms else bs.grad)):
        if want is not None:
            assert float((out[name].double() - want).norm() / want.norm()) <= 4 * B, name
    assert abs(float((nll.double() * mask).sum() / n) - float(loss.detach())) <= 1e-5 * float(loss.detach())


def test_the_norms_backward_pass_is_captured_beside_an_eager_graph():
    """A captured backward pass of leaves that an eager autograd graph holds alive: the calls take no part in autograd."""
    T, D = 50, 128
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn((T, D), device=DEV, generator=g).to(torch.bfloat16).requires_grad_()
    w = torch.ones(D, dtype=torch.bfloat16, device=DEV, requires_grad=True)
    alive = (x * w).sum()
    gy, rstd, gx, gw = torch.ones_like(x), torch.empty(T, device=DEV), torch.empty_like(x), torch.empty_like(w)
    y = torch.empty_like(x)
    ws = torch.empty(npd.npd_layer_norm_workspace_bytes(T, D), dtype=torch.uint8, device=DEV)

    def call():
        npd.npd_layer_norm(x, w, rms=True, y_out=y, rstd_out=rstd)
        npd.npd_layer_norm_bwd(gy, x, w, rstd=rstd, rms=True, grad_x=gx, grad_weight=gw, workspace=ws)

    call()
    torch.cuda.synchronize()
    want = gx.clone(), gw.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        gx.zero_()
        gw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(gx, want[0]) and torch.equal(gw, want[1])
    alive.backward()
    assert x.grad is not None and w.grad is not None


def _calls(seed=0):
    """Every wrapper's call with each of its arguments: (call, outputs)."""
    T, V, D = 70, 600, 130
    weight, norm, g = model(V, D, seed)
    f = dict(device=DEV)
    x = torch.randn((T, D), device=DEV, generator=g).to(torch.bfloat16)
    bias = torch.randn(V, device=DEV, generator=g).to(torch.bfloat16)
    y, mean, rstd = torch.empty_like(x), torch.empty(T, **f), torch.empty(T, **f)
    gx, gw, gb = torch.empty_like(x), torch.ones_like(norm), torch.ones_like(norm)
    q, scale = torch.empty((T, D), dtype=torch.int8, **f), torch.empty(T, **f)
    wq, wscale = torch.empty((V, D), dtype=torch.int8, **f), torch.empty(V, **f)
    logits = torch.empty((T, V), dtype=torch.bfloat16, **f)
    tokens, kept, status = (torch.zeros(n, dtype=torch.int32, **f) for n in (T, T, 1))
    logprob, nll = torch.empty(T, **f), torch.empty(T, **f)
    u, r = torch.rand(T, device=DEV, generator=g), torch.rand(T, device=DEV, generator=g)
    mask = (r < 0.9).to(torch.uint8)
    ws = [torch.empty(1 << 20, dtype=torch.uint8, **f) for _ in range(3)]
    own = dict(temperature=0.5 + r, top_k=(50 * r).to(torch.int32), top_p=1 - 0.2 * r, min_p=0.1 * r)
    return [
        (lambda: npd.npd_layer_norm(x, norm, bias=norm, eps=1e-4, y_out=y, mean_out=mean, rstd_out=rstd), [y, mean, rstd]),
        (lambda: npd.npd_layer_norm(x, y_out=y, rms=True, rstd_out=rstd), [y, rstd]),
        (lambda: npd.npd_layer_norm_bwd(y, x, norm, mean=mean, rstd=rstd, grad_x=gx, grad_weight=gw, grad_bias=gb, accumulate=True), [gx, gw, gb]),
        (lambda: npd.npd_layer_norm_bwd(y, x, rstd=rstd, rms=True, grad_weight=gw, workspace=ws[0]), [gw]),
        (lambda: npd.npd_quantize_rows(x, q_out=q, scale_out=scale), [q, scale]),
        (lambda: npd.npd_quantize_rows(weight, q_out=wq, scale_out=wscale), [wq, wscale]),
        (lambda: npd.npd_head_logits_int8(q, scale, wq, wscale, bias=bias, softcap=20.0, logits_out=logits), [logits]),
        (lambda: npd.npd_head_logits_int8(q, scale, wq, wscale, logits_out=logits, workspace=ws[1]), [logits]),
        (lambda: npd.npd_sample_tokens(logits, u, tokens_out=tokens, temperature=0.7, top_k=20, top_p=0.9, min_p=0.01, loss_mask=mask,
                                       logprob_out=logprob, nll_out=nll, kept_out=kept, dev_status=status), [tokens, logprob, nll, kept, status]),
        (lambda: npd.npd_sample_tokens(logits, u, tokens_out=tokens, logprob_out=logprob, kept_out=kept, workspace=ws[2], **own),
         [tokens, logprob, kept]),
        (lambda: npd.npd_sample_tokens(logits, u, tokens_out=tokens, top_k=None, kept_out=kept), [tokens, kept]),
    ]


def test_native_and_python_marshalling_make_the_same_calls(monkeypatch):
    assert binding._host is not None
    native, python = [], []
    for call, outputs in _calls():
        call()
        native.append([t.clone() for t in outputs])
    monkeypatch.setattr(binding, "_host", None)
    for call, outputs in _calls():
        call()
        python.append([t.clone() for t in outputs])
    for a, b in zip(native, python):
        assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("host", [True, False])
def test_refusals_are_the_same_with_either(host, monkeypatch):
    if not host:
        monkeypatch.setattr(binding, "_host", None)
    x, f = torch.zeros((4, 40), dtype=torch.bfloat16, device=DEV), torch.zeros(4, device=DEV)
    q, i = torch.zeros((4, 40), dtype=torch.int8, device=DEV), torch.zeros(4, dtype=torch.int32, device=DEV)
    for call in (lambda: npd.npd_layer_norm(x, y_out=x), lambda: npd.npd_layer_norm(x, y_out=x.clone(), eps=-1.0),
                 lambda: npd.npd_layer_norm_bwd(x, x, rstd=f, rms=True), lambda: npd.npd_layer_norm_bwd(x, x, rstd=f, grad_x=x.clone()),
                 lambda: npd.npd_quantize_rows(x, q_out=x.view(torch.int8)[:, :40], scale_out=f),
                 lambda: npd.npd_head_logits_int8(q, f, q, f, logits_out=x[:, :4], softcap=float("nan")),
                 lambda: npd.npd_sample_tokens(x, f, tokens_out=i, temperature=-1.0), lambda: npd.npd_sample_tokens(x, f, tokens_out=i, top_k=-1),
                 lambda: npd.npd_sample_tokens(x, f, tokens_out=f.view(torch.int32))):
        with pytest.raises(binding.NpdError):
            call()
    for call in (lambda: npd.npd_layer_norm(x.float(), y_out=x.clone()), lambda: npd.npd_layer_norm(x, y_out=x.clone()[:, :39]),
                 lambda: npd.npd_layer_norm(x.t(), y_out=x.t()), lambda: npd.npd_layer_norm(x, f, y_out=x.clone()),
                 lambda: npd.npd_quantize_rows(x, q_out=i, scale_out=f), lambda: npd.npd_quantize_rows(x, q_out=q, scale_out=f[:3]),
                 lambda: npd.npd_head_logits_int8(q, f, x, f, logits_out=x[:, :4].clone()),
                 lambda: npd.npd_sample_tokens(x, i, tokens_out=i), lambda: npd.npd_sample_tokens(x, f, tokens_out=i, top_p=i),
                 lambda: npd.npd_sample_tokens(x, f.cpu(), tokens_out=i)):
        with pytest.raises(ValueError):
            call()
