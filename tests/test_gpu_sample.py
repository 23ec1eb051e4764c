"""Tokens drawn from logits against the 64-bit definition: tokens and counts are equal, logarithms are off by one rounding to fp32 (2^-24
of themselves) and what two 64-bit computations of sums of up to 2^18 terms differ by (below 1e-11)."""
import numpy as np
import pytest
import torch

import paper_2605_05940_amd as npd
from paper_2605_05940_amd import binding
from sample_util import draw

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def logits(T, V, seed=0, spread=3.0, offset=0, pad=0):
    g = torch.Generator(device=DEV).manual_seed(seed + 31 * T + V)
    memory = torch.full((offset + T * (V + pad),), 1e4, dtype=torch.bfloat16, device=DEV)
    x = memory[offset:].view(T, V + pad)[:, :V]
    x.copy_(spread * torch.randn((T, V), device=DEV, generator=g))
    return x, torch.rand(T, device=DEV, generator=g)


def call(x, u, **settings):
    T = x.shape[0]
    out = dict(tokens_out=torch.full((T,), -9, dtype=torch.int32, device=DEV), kept_out=torch.full((T,), -9, dtype=torch.int32, device=DEV),
               logprob_out=torch.full((T,), 9.0, device=DEV), nll_out=torch.full((T,), 9.0, device=DEV))
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    npd.npd_sample_tokens(x, u, dev_status=status, **out, **settings)
    return {n: v.cpu().numpy() for n, v in out.items()}, int(status.item())


def check(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    got, status = call(x, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    assert status == 0
    if npd.npd_sample_workspace_bytes(*x.shape):  # rows in parts, and whole: the same bit by bit
        whole, status = call(x, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p,
                             workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
        assert status == 0 and all((whole[n] == got[n]).all() for n in got)
    T = x.shape[0]

    def setting(v):
        v = v.cpu().numpy() if isinstance(v, torch.Tensor) else np.full(T, v, np.float32 if isinstance(v, float) else np.int64)
        return v

    tau, k, p, m = (setting(v) for v in (temperature, top_k, top_p, min_p))
    rows, us = x.double().cpu().numpy(), u.double().cpu().numpy()
    for r in range(T):
        token, kept, logprob, nll = draw(rows[r], us[r], float(tau[r]), int(k[r]), float(p[r]), float(m[r]))
        assert (got["tokens_out"][r], got["kept_out"][r]) == (token, kept), (r, got["tokens_out"][r], token, got["kept_out"][r], kept)
        for name, want in (("logprob_out", logprob), ("nll_out", nll)):
            assert abs(float(got[name][r]) - want) <= 2.0 ** -24 * abs(want) + 1e-11, (r, name)


SETTINGS = [dict(), dict(temperature=0.7), dict(temperature=0.0), dict(top_k=1), dict(top_k=50), dict(top_p=0.9), dict(min_p=0.05),
            dict(temperature=1.5, top_k=200, top_p=0.95, min_p=0.01), dict(top_p=0.0), dict(min_p=1.0), dict(top_k=10 ** 6, top_p=0.5),
            dict(temperature=0.3, top_p=0.999, top_k=37)]


@pytest.mark.parametrize("settings", SETTINGS, ids=str)
@pytest.mark.parametrize("T,V,offset,pad", [(1, 1, 0, 0), (5, 2, 1, 0), (9, 7, 3, 2), (40, 100, 0, 0), (33, 1000, 1, 1), (17, 4099, 0, 0),
                                            (12, 8192, 0, 0), (10, 32001, 5, 0), (5, 98304, 0, 0), (2, 131073, 1, 2), (6, 50003, 0, 0), (3, 151936, 0, 64)])
def test_against_the_definition(T, V, offset, pad, settings):
    check(*logits(T, V, offset=offset, pad=pad), **settings)


@pytest.mark.parametrize("spread", [0.0, 1e-3, 0.1, 30.0, 1e3, 1e30])
def test_logits_of_every_size(spread):
    """Equal ones, values that are closer than 2^-23 (no counter of their own) and far beyond 256 (likewise)."""
    for settings in (dict(), dict(top_k=20), dict(top_p=0.8), dict(temperature=0.0), dict(temperature=2.0, min_p=0.3, top_p=0.9)):
        check(*logits(8, 3000, spread=spread), **settings)


@pytest.mark.parametrize("V", [2000, 100003])
@pytest.mark.parametrize("n", [1, 2, 8, 9, 254, 255, 256, 300])
def test_entries_close_to_zero(n, V):
    """Numbers below 2^-23, some of them equal, zeros of both signs among them: listed, or too many for the list."""
    x, u = logits(24, V, spread=0.3)
    g = torch.Generator(device=DEV).manual_seed(n)
    tiny = torch.randint(1, 1 + 3 * n, (24, n), device=DEV, generator=g) * torch.randint(0, 2, (24, n), device=DEV, generator=g).mul(2).sub(1)
    x[:, torch.arange(100, 100 + n) * (V // 1000) % V] = (tiny.float() * 2.0 ** -40).to(torch.bfloat16)
    x[::2, 1900:1907] = 0.0
    x[::3, 1907:1911] = -0.0
    for settings in (dict(), dict(top_k=1000), dict(temperature=2.0 ** -40), dict(temperature=2.0 ** -39, min_p=0.2, top_p=0.9), dict(top_p=0.5)):
        check(x, u, **settings)
    x.masked_fill_(x.float().abs() > 2.0 ** -23, float("-inf"))
    x[:, 50] = torch.finfo(torch.bfloat16).tiny
    x[::2, 1900] = 0.0
    for settings in (dict(), dict(temperature=2.0 ** -39), dict(temperature=2.0 ** -39, min_p=0.7), dict(temperature=0.0), dict(min_p=1.0)):
        check(x, u, **settings)


@pytest.mark.parametrize("scale", [2.0 ** -40, 2.0 ** -24, 2.0 ** -22, 100.0, 1e4, 1e35])
def test_temperatures_as_large_as_the_logits(scale):
    x, u = logits(8, 2000, spread=scale)
    check(x, u, temperature=float(np.float32(scale)))
    check(x, u, temperature=float(np.float32(scale)), top_k=100, top_p=0.9, min_p=0.01)


@pytest.mark.parametrize("V,offset", [(40, 3), (2000, 1), (8191, 0), (65535, 5), (65600, 0), (524280, 2), (524287, 0), (524288, 0), (600001, 1),
                                      (4300003, 3)])
def test_the_entry_wherever_it_is(V, offset):
    """A value that occurs once, at the ends of the row, of its parts and of what is looked at together, and another that does twice."""
    T = 40
    g = torch.Generator(device=DEV).manual_seed(V)
    memory = torch.full((offset + T * V + 8,), 1e4, dtype=torch.bfloat16, device=DEV)
    x = memory[offset:offset + T * V].view(T, V)
    x.copy_((0.5 * torch.randn((T, V), device=DEV, generator=g)).clamp(-2, 2))
    places = [0, 1, 5, 7, 8, 9, V - 1, V - 2, V - 8, V - 9, V // 2, V // 3, V // 8, V // 8 - 1, V // 8 // 8 * 8, 16383 % V, 16384 % V, 24575 % V,
              24576 % V, 49151 % V, 49152 % V] + torch.randint(0, V, (T,), device=DEV, generator=g).tolist()
    rows = torch.arange(T, device=DEV)
    at = torch.tensor(places[:T], device=DEV)
    x[rows, at] = 30.0                                   # all the weight there is
    u = torch.rand(T, device=DEV, generator=g)
    for how in (dict(), dict(workspace=torch.empty(256, dtype=torch.uint8, device=DEV))):
        tokens = torch.empty(T, dtype=torch.int32, device=DEV)
        for few in (T, 2):
            npd.npd_sample_tokens(x[:few], u[:few], temperature=0.5, tokens_out=tokens[:few], **how)
            assert torch.equal(tokens[:few].long(), at[:few])
    also = (at + 1 + torch.randint(0, V - 1, (T,), device=DEV, generator=g)) % V
    x[rows, also] = 30.0
    want = torch.where(u < 0.5, torch.minimum(at, also), torch.maximum(at, also))
    for few in (T, 2):
        tokens = torch.empty(few, dtype=torch.int32, device=DEV)
        npd.npd_sample_tokens(x[:few], u[:few], temperature=0.5, tokens_out=tokens)
        assert torch.equal(tokens.long(), want[:few])


def test_few_values_and_many_ties():
    """Bf16 logits of two bits: every draw ends among equal entries, and in the middle of them what is kept ends."""
    x, u = logits(64, 5000, spread=1.0)
    x.copy_(torch.round(x.float()))
    for settings in (dict(), dict(top_k=777), dict(top_p=0.6), dict(top_k=3000, top_p=0.7, min_p=0.05), dict(temperature=0.0)):
        check(x, u, **settings)


@pytest.mark.parametrize("V,offset", [(1024, 0), (1025, 1), (5003, 3), (20000, 0), (151936, 0), (100001, 1)])
@pytest.mark.parametrize("value", [0.0, -1.5, 2.0 ** -30, 300.0])
def test_rows_of_equal_entries(V, offset, value):
    """The list of the ids of a value is as long as a list may be, longer, and far longer."""
    x, u = logits(7, V, offset=offset)
    x.fill_(value)
    x[3:, ::7] = value - 1
    check(x, u)
    check(x, u, top_k=V // 2, top_p=0.9)


def test_zeros_of_either_sign_are_equal():
    x = torch.zeros((6, 300), dtype=torch.bfloat16, device=DEV)
    x[:, ::2] = -0.0
    x[3:, 7] = 2.0 ** -30  # a row without a counter for every entry
    u = torch.tensor([0.0, 0.5, 0.999, 0.0, 0.4, 0.999], device=DEV)
    check(x, u)
    check(x, u, top_k=100)
    check(x, u, temperature=0.0)


@pytest.mark.parametrize("V", [64, 3001, 40000, 120001])
def test_entries_of_minus_infinity(V):
    x, u = logits(12, V)
    g = torch.Generator(device=DEV).manual_seed(8)
    x.masked_fill_(torch.rand(x.shape, device=DEV, generator=g) < 0.9, float("-inf"))
    x[:, 5] = 1.0
    x[7:10] = float("-inf")
    x[7:10, 6] = torch.tensor([-300.0, 0.0, 2.0 ** -40], device=DEV)  # one that is left, in either kind of row
    for settings in SETTINGS:
        check(x, u, **settings)


@pytest.mark.parametrize("V", [2000, 99000])
def test_the_lowest_number_as_a_mask(V):
    x, u = logits(8, V)
    g = torch.Generator(device=DEV).manual_seed(9)
    x.masked_fill_(torch.rand(x.shape, device=DEV, generator=g) < 0.7, torch.finfo(torch.bfloat16).min)
    x[4:] = torch.finfo(torch.bfloat16).min  # nothing else left: equal entries
    for settings in SETTINGS:
        check(x, u, **settings)


@pytest.mark.parametrize("V", [1500, 110001])
def test_numbers_below_minus_256(V):
    x, u = logits(8, V)
    x[:, ::3] = -400.0
    x[4:] -= 250.0  # the rest not far above
    for settings in SETTINGS + [dict(temperature=100.0), dict(top_k=1400), dict(min_p=1e-38), dict(temperature=30.0, min_p=1e-30)]:
        check(x, u, **settings)


@pytest.mark.parametrize("u", [0.0, 2.0 ** -149, 2.0 ** -24, 0.5, 1 - 2.0 ** -24])
def test_random_numbers_at_the_ends(u):
    x, _ = logits(9, 6000)
    us = torch.full((9,), u, device=DEV)
    for settings in SETTINGS:
        check(x, us, **settings)


def test_settings_of_every_row():
    T, V = 60, 9000
    x, u = logits(T, V)
    g = torch.Generator(device=DEV).manual_seed(11)
    r = torch.rand((4, T), device=DEV, generator=g)
    rows = dict(temperature=(2 * r[0]) * (r[0] > 0.2), top_k=(300 * r[1]).to(torch.int32) * (r[1] > 0.3).to(torch.int32),
                top_p=torch.where(r[2] > 0.3, r[2], 1.0), min_p=torch.where(r[3] > 0.5, 0.2 * r[3], 0.0))
    check(x, u, **rows)
    check(x, u, temperature=rows["temperature"], top_k=5)


@pytest.mark.parametrize("V", [700, 120000])
def test_rows_that_are_not_drawn_from(V):
    x, u = logits(10, V)
    mask = torch.ones(10, dtype=torch.uint8, device=DEV)
    mask[3] = 0
    x[3] = float("nan")
    got, status = call(x, u, loss_mask=mask)
    assert status == 0
    assert [got[n][3] for n in ("tokens_out", "kept_out", "logprob_out", "nll_out")] == [-1, 0, 0, 0]
    clean, _ = call(torch.where(x.isnan(), 0, x), u)
    others = np.arange(10) != 3
    assert all((got[n][others] == clean[n][others]).all() for n in got)


@pytest.mark.parametrize("V", [900, 120000])
@pytest.mark.parametrize("bad", ["nan", "-nan", "inf", "empty"])
def test_logits_that_cannot_be_drawn_from(bad, V):
    x, u = logits(6, V)
    clean, _ = call(x, u)
    if bad == "empty":
        x[2] = float("-inf")
    else:
        x[2, V - 1] = float("inf") if bad == "inf" else float("nan")
        if bad == "-nan":
            x.view(torch.int16)[2, V - 1] = -1
    got, status = call(x, u)
    assert status == binding.NPD_DEV_BAD_LOGITS
    assert got["tokens_out"][2] == -1 and got["kept_out"][2] == 0 and np.isnan(got["logprob_out"][2]) and np.isnan(got["nll_out"][2])
    others = np.arange(6) != 2
    assert all((got[n][others] == clean[n][others]).all() for n in got)


@pytest.mark.parametrize("name,value", [("temperature", -1.0), ("temperature", float("nan")), ("temperature", float("inf")), ("top_k", -1),
                                        ("top_p", -0.1), ("top_p", 1.5), ("top_p", float("nan")), ("min_p", 2.0), ("min_p", float("nan")),
                                        ("uniform", 1.0), ("uniform", -0.1), ("uniform", float("nan"))])
def test_settings_out_of_range_on_the_device(name, value):
    x, u = logits(5, 800)
    fine = dict(temperature=1.0, top_k=10, top_p=0.9, min_p=0.01)
    clean, _ = call(x, u, **fine)
    if name == "uniform":
        u[1] = value
    else:
        fine[name] = torch.full((5,), fine[name], device=DEV, dtype=torch.int32 if name == "top_k" else torch.float32)
        fine[name][1] = value
    got, status = call(x, u, **fine)
    assert status == binding.NPD_DEV_BAD_SAMPLING
    assert got["tokens_out"][1] == -1 and got["kept_out"][1] == 0 and np.isnan(got["logprob_out"][1]) and np.isnan(got["nll_out"][1])
    others = np.arange(5) != 1
    assert all((got[n][others] == clean[n][others]).all() for n in got)


def test_tokens_alone():
    x, u = logits(20, 3000)
    want, _ = call(x, u, top_p=0.9)
    tokens = torch.empty(20, dtype=torch.int32, device=DEV)
    npd.npd_sample_tokens(x, u, top_p=0.9, tokens_out=tokens)
    assert (tokens.cpu().numpy() == want["tokens_out"]).all()


def test_more_rows_than_workgroups_of_one_launch():
    T, V = 70000, 24
    x, u = logits(T, V)
    got, status = call(x, u, top_k=5)
    assert status == 0
    rows, us = x.double().cpu().numpy(), u.double().cpu().numpy()
    for r in list(range(0, T, 997)) + [65535, 65536, T - 1]:
        assert (got["tokens_out"][r], got["kept_out"][r]) == draw(rows[r], us[r], 1.0, 5, 1.0, 0.0)[:2]


def test_offsets_beyond_32_bits():
    V, stride = 1000, (1 << 30) + 11
    x, u = logits(3, V)
    far = torch.as_strided(torch.empty(2 * stride + V, dtype=torch.bfloat16, device=DEV), (3, V), (stride, 1))
    far.copy_(x)
    check(far, u, top_p=0.8)


@pytest.mark.parametrize("T,V", [(30, 20000), (3, 140000)])
def test_captured_and_replayed(T, V):
    ws = torch.empty(npd.npd_sample_workspace_bytes(T, V), dtype=torch.uint8, device=DEV)
    sets = [logits(T, V, seed=s) for s in range(3)]
    x, u = (t.clone() for t in sets[0])
    tau = torch.full((T,), 0.8, device=DEV)
    tokens, nll = torch.empty(T, dtype=torch.int32, device=DEV), torch.empty(T, device=DEV)

    def run(x, u, tokens, nll, **how):
        npd.npd_sample_tokens(x, u, temperature=tau, top_k=100, top_p=0.95, tokens_out=tokens, nll_out=nll, **how)

    run(x, u, tokens, nll, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(x, u, tokens, nll, workspace=ws)
    for s in (1, 0, 2, 1):
        x.copy_(sets[s][0])
        u.copy_(sets[s][1])
        graph.replay()
        want = torch.empty_like(tokens), torch.empty_like(nll)
        run(*sets[s], *want)
        torch.cuda.synchronize()
        assert torch.equal(tokens, want[0]) and torch.equal(nll, want[1])


@pytest.mark.parametrize("T", [50, 5])
def test_two_streams_at_once(T):
    sets = [logits(T, 100000, seed=s) for s in range(2)]
    want = [call(x, u, top_p=0.9)[0] for x, u in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    outs = []
    torch.cuda.synchronize()
    for _ in range(3):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                tokens = torch.empty(T, dtype=torch.int32, device=DEV)
                npd.npd_sample_tokens(*sets[i], top_p=0.9, tokens_out=tokens)
                outs.append((i, tokens))
    torch.cuda.synchronize()
    for i, tokens in outs:
        assert (tokens.cpu().numpy() == want[i]["tokens_out"]).all()
