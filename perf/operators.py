"""Performance cases of the head operators: the language-model head (hidden states times the vocabulary's weights) with
the loss behind it, as a distillation program calls them through the Python entry points.

  loss        one training step's loss from hidden states: npd_head_loss_fwd_bwd with gradients of hidden states, weights
              and bias; hard labels, a top-k teacher record, or both (Eq. 1)
  score       the same call forward only: per-position NLL, log-sum-exp and KL (Delta-IFD, perplexity, monitors)
  logits      npd_head_logits: bf16 logits, with bias and soft cap, for the calls that take logits
  logits_bwd  npd_head_logits_bwd: gradients of hidden states, weights and bias from the bf16 gradient of the logits

`tokens` are positions, `scored` the share of them that the mask keeps, `vocab` the rows and `width` the columns of the
weights, `k` the entries of the teacher's record (0: none), `lam` the weight of the KD term of Eq. 1 (0: hard labels
only), `cap` the soft cap (0: none).
"""
import math

import torch

DEVICE = "cuda:0"
own = False

CHUNK = 1 << 28                          # logits that the plain form and the exact one hold at a time
MAX_PRODUCT = 32768 * 151936 * 2048      # tokens * vocab * width of the largest listed case


def listed():
    return [
        # A whole training step at a 1B student's vocabulary: one pack of 32,768 positions, composite loss against the
        # stored top 64; prompts and padding are not scored.
        dict(name="loss_32k_topk64", op="loss", tokens=32768, scored=0.7, vocab=151936, width=2048, k=64, lam=0.9,
             tau=1.0, bias=False, cap=0.0),
        # Supervised fine-tuning at the largest vocabulary, soft-capped logits, hard labels alone.
        dict(name="loss_wide_vocab_ce", op="loss", tokens=8192, scored=0.8, vocab=262144, width=1152, k=0, lam=0.0,
             tau=1.0, bias=False, cap=30.0),
        # A micro-batch at a temperature, a vocabulary that nobody padded, a head with bias.
        dict(name="loss_odd_tau2", op="loss", tokens=1500, scored=0.6, vocab=50003, width=1000, k=10, lam=1.0, tau=2.0,
             bias=True, cap=0.0),
        # The smallest training call: launches and latency count.
        dict(name="loss_tiny", op="loss", tokens=512, scored=0.75, vocab=1024, width=256, k=10, lam=0.9, tau=1.0,
             bias=False, cap=0.0),
        # Data selection: the NLL of every response position of two packs.
        dict(name="score_16k", op="score", tokens=16384, scored=0.7, vocab=151936, width=1536, k=0, lam=0.0, tau=1.0,
             bias=False, cap=0.0),
        # One token of a rollout: the log-probability of what was sampled.
        dict(name="score_one_token", op="score", tokens=1, scored=1.0, vocab=151936, width=2048, k=0, lam=0.0, tau=1.0,
             bias=False, cap=0.0),
        # A monitor on a few positions against a teacher's record; width and vocabulary as odd as they come.
        dict(name="score_48_odd", op="score", tokens=48, scored=0.9, vocab=50003, width=1004, k=10, lam=1.0, tau=1.0,
             bias=True, cap=0.0),
        # A teacher's logits for the dense loss or its top-k record.
        dict(name="logits_4k", op="logits", tokens=4096, scored=1.0, vocab=151936, width=2048, k=0, lam=0.0, tau=1.0,
             bias=False, cap=0.0),
        # The next token's logits of one sequence, soft-capped.
        dict(name="logits_one_token", op="logits", tokens=1, scored=1.0, vocab=262144, width=1152, k=0, lam=0.0,
             tau=1.0, bias=False, cap=30.0),
        # A short prompt, rows of the logits at any even byte, bias and soft cap.
        dict(name="logits_odd", op="logits", tokens=333, scored=1.0, vocab=50003, width=1000, k=0, lam=0.0, tau=1.0,
             bias=True, cap=30.0),
        # The backward pass behind the dense-teacher loss.
        dict(name="logits_bwd_4k", op="logits_bwd", tokens=4096, scored=0.7, vocab=151936, width=2048, k=0, lam=0.0,
             tau=1.0, bias=False, cap=0.0),
        # The same for a short prompt, unpadded rows, bias and soft cap.
        dict(name="logits_bwd_odd", op="logits_bwd", tokens=333, scored=0.8, vocab=50003, width=1000, k=0, lam=0.0,
             tau=1.0, bias=True, cap=30.0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["loss", "loss", "loss", "score", "score", "logits", "logits_bwd"])
    vocab = _log_uniform(rng, 1000, 262144)
    vocab = max(64, vocab // 64 * 64) if rng.random() < 0.5 else vocab | 1
    width = _log_uniform(rng, 64, 4096)
    how = rng.random()
    width = width // 64 * 64 if how < 0.6 else width // 8 * 8 if how < 0.9 else width
    tokens = min(_log_uniform(rng, 1 if op in ("score", "logits") else 16, 32768), MAX_PRODUCT // (vocab * width))
    if op in ("logits", "logits_bwd"):
        tokens = min(tokens, 1_000_000_000 // vocab)
    k, lam, tau = 0, 0.0, 1.0
    if op in ("loss", "score") and rng.random() < 0.6:
        k, lam = _log_uniform(rng, 5, 100), rng.choice([1.0, 0.9])
        tau = rng.choice([1.0, 2.0]) if lam == 1.0 else 1.0
    return dict(op=op, tokens=tokens, scored=round(rng.uniform(0.5, 1.0), 2), vocab=vocab, width=width, k=k, lam=lam,
                tau=tau, bias=rng.random() < 0.3, cap=rng.choice([0.0, 0.0, 30.0]))


def prepare(case, seed):
    T, V, D, k = case["tokens"], case["vocab"], case["width"], case["k"]
    g = torch.Generator(device=DEVICE).manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, device=DEVICE, generator=g)

    state = dict(case=case)
    # logits of a random position spread over a few units; the head's input is a normalised activation
    weight = torch.empty((V, D), dtype=torch.bfloat16, device=DEVICE)
    for a in range(0, V, 65536):
        weight[a:a + 65536] = randn(min(65536, V - a), D) * (3.0 / math.sqrt(D))
    state["weight"] = weight
    state["bias"] = (0.5 * randn(V)).to(torch.bfloat16) if case["bias"] else None
    hidden = randn(T, D)
    mask = (torch.rand(T, device=DEVICE, generator=g) < case["scored"]).to(torch.uint8)
    mask[T // 2] = 1
    state["mask"] = mask
    if case["op"] in ("loss", "score"):
        # labels from hardly expected to nearly certain
        labels = torch.randint(0, V, (T,), device=DEVICE, generator=g)
        hidden += (0.4 + 1.6 * torch.rand((T, 1), device=DEVICE, generator=g)) * weight[labels].float()
        state["labels"] = labels.to(torch.int32)
        if k:
            # the teacher's record: distinct ids, the label among them, a few of which the student expects as well
            step = torch.randint(1, max(2, V // k), (T, 1), device=DEVICE, generator=g)
            idx = (labels[:, None] + step * torch.arange(k, device=DEVICE)) % V
            for j in range(1, min(k, 4)):
                hidden += 0.8 / j * weight[idx[:, j]].float()
            val = torch.sort(1.5 * randn(T, k), dim=1, descending=True).values
            state["idx"] = idx.to(torch.int32)
            state["val"] = val - torch.logsumexp(val, dim=1, keepdim=True)
    state["hidden"] = hidden.to(torch.bfloat16)
    # sums of a gradient are means over the scored positions, as a training program folds them into its weights
    n = max(1, round(T * case["scored"]))
    state["grad_scale"], state["ce_scale"] = case["lam"] / n, (1.0 - case["lam"]) / n
    if case["op"] == "logits_bwd":
        # the logit gradient of a loss: small everywhere, large at the label, zero rows where nothing is scored
        dlogits = torch.empty((T, V), dtype=torch.bfloat16, device=DEVICE)
        logits = torch.empty_like(dlogits) if case["cap"] else None
        rows = max(1, CHUNK // V)
        for a in range(0, T, rows):
            b = min(T, a + rows)
            z = 3.0 * randn(b - a, V)
            if logits is not None:
                logits[a:b] = case["cap"] * torch.tanh(z / case["cap"])
            p = torch.softmax(z, 1)
            p[torch.arange(b - a, device=DEVICE), torch.randint(0, V, (b - a,), device=DEVICE, generator=g)] -= 1.0
            dlogits[a:b] = p * mask[a:b, None]
        state["dlogits"], state["logits"] = dlogits, logits
    return state


# ------------------------------------------------------------------------------------------------------ the plain forms

def _plain_logits(h, wt, bias, cap):
    x = h @ wt
    if bias is not None:
        x += bias
    return cap * torch.tanh(x / cap) if cap else x


def _plain_loss(s, grads):
    c = s["case"]
    T, V = c["tokens"], c["vocab"]
    w = s["weight"].float()
    bias = None if s["bias"] is None else s["bias"].float()
    rows_all = torch.nonzero(s["mask"]).flatten()
    out = dict(nll=torch.zeros(T, device=w.device), lse=torch.zeros(T, device=w.device)) if c["tau"] == 1.0 else {}
    if c["k"]:
        out["kd"] = torch.zeros(T, device=w.device)
    if grads:
        out["grad_hidden"] = torch.zeros_like(s["hidden"])
        dw = torch.zeros_like(w)
        db = torch.zeros(V, device=w.device)
    for rows in rows_all.split(max(1, CHUNK // V)):
        h = s["hidden"][rows].float()
        x = _plain_logits(h, w.t(), bias, c["cap"])
        u = x / c["tau"]
        top = u.amax(1, keepdim=True)
        e = torch.exp(u - top)
        z = e.sum(1, keepdim=True)
        lse = (top + torch.log(z))[:, 0]
        y = s["labels"][rows].long()
        if "nll" in out:
            out["lse"][rows] = lse
            out["nll"][rows] = lse - x.gather(1, y[:, None])[:, 0]
        if c["k"]:
            ids = s["idx"][rows].long()
            v = s["val"][rows] / c["tau"]
            v = v - v.amax(1, keepdim=True)
            logp = v - torch.log(torch.exp(v).sum(1, keepdim=True))
            out["kd"][rows] = (torch.exp(logp) * (logp - u.gather(1, ids) + lse[:, None])).sum(1)
        if not grads:
            continue
        kd, ce = (s["grad_scale"] / c["tau"], s["ce_scale"])
        d = e * ((kd + ce) / z)
        if c["k"]:
            d.scatter_add_(1, ids, -kd * torch.exp(logp))
        if ce:
            d.scatter_add_(1, y[:, None], torch.full_like(z, -ce))
        if c["cap"]:
            d *= 1.0 - (x / c["cap"]) ** 2
        out["grad_hidden"][rows] = (d @ w).to(torch.bfloat16)
        dw += d.t() @ h
        db += d.sum(0)
    if grads:
        out["grad_weight"] = dw.to(torch.bfloat16)
        if bias is not None:
            out["grad_bias"] = db.to(torch.bfloat16)
    return out


def _plain_head_logits(s):
    c = s["case"]
    w = s["weight"].float()
    bias = None if s["bias"] is None else s["bias"].float()
    out = torch.empty((c["tokens"], c["vocab"]), dtype=torch.bfloat16, device=w.device)
    rows = max(1, CHUNK // c["vocab"])
    for a in range(0, c["tokens"], rows):
        out[a:a + rows] = _plain_logits(s["hidden"][a:a + rows].float(), w.t(), bias, c["cap"]).to(torch.bfloat16)
    return dict(logits=out)


def _plain_logits_bwd(s):
    c = s["case"]
    w = s["weight"].float()
    out = dict(grad_hidden=torch.empty_like(s["hidden"]))
    dw = torch.zeros_like(w)
    db = torch.zeros(c["vocab"], device=w.device)
    rows = max(1, CHUNK // c["vocab"])
    for a in range(0, c["tokens"], rows):
        d = s["dlogits"][a:a + rows].float()
        if c["cap"]:
            d *= 1.0 - (s["logits"][a:a + rows].float() / c["cap"]) ** 2
        out["grad_hidden"][a:a + rows] = (d @ w).to(torch.bfloat16)
        dw += d.t() @ s["hidden"][a:a + rows].float()
        db += d.sum(0)
    out["grad_weight"] = dw.to(torch.bfloat16)
    if s["bias"] is not None:
        out["grad_bias"] = db.to(torch.bfloat16)
    return out


# ------------------------------------------------------------------------------------------------ the framework's calls

def _own(s):
    import paper_2605_05940_amd as npd
    c = s["case"]
    T, V = c["tokens"], c["vocab"]
    hidden, weight, bias = s["hidden"], s["weight"], s["bias"]
    if c["op"] == "logits":
        logits = torch.empty((T, V), dtype=torch.bfloat16, device=DEVICE)
        npd.npd_head_logits(hidden, weight, bias=bias, softcap=c["cap"], logits_out=logits)
        return dict(logits=logits)
    out = {}
    if c["op"] != "score":
        out["grad_hidden"], out["grad_weight"] = torch.empty_like(hidden), torch.empty_like(weight)
        if bias is not None:
            out["grad_bias"] = torch.empty_like(bias)
    if c["op"] == "logits_bwd":
        npd.npd_head_logits_bwd(s["dlogits"], hidden, weight, logits=s["logits"], softcap=c["cap"],
                                grad_hidden=out["grad_hidden"], grad_weight=out["grad_weight"],
                                grad_bias=out.get("grad_bias"))
        return out
    scalars = {}
    if c["tau"] == 1.0:
        scalars = dict(nll=torch.empty(T, device=DEVICE), lse=torch.empty(T, device=DEVICE))
    if c["k"]:
        scalars["kd"] = torch.empty(T, device=DEVICE)
    training = c["op"] == "loss"
    npd.npd_head_loss_fwd_bwd(
        hidden, weight, s["mask"], bias=bias, softcap=c["cap"], labels=s["labels"], teacher_idx=s.get("idx"),
        teacher_val=s.get("val"), tau=c["tau"], grad_scale=s["grad_scale"] if training else 1.0,
        ce_grad_scale=s["ce_scale"] if training else 0.0, grad_hidden=out.get("grad_hidden"),
        grad_weight=out.get("grad_weight"), grad_bias=out.get("grad_bias"), nll_tok=scalars.get("nll"),
        lse_tok=scalars.get("lse"), kd_tok=scalars.get("kd"))
    return {**scalars, **out}


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "logits":
        return _plain_head_logits(state)
    if op == "logits_bwd":
        return _plain_logits_bwd(state)
    return _plain_loss(state, op == "loss")


# ------------------------------------------------------------------------------------------------------- work and truth

def work(case):
    T, V, D, k = case["tokens"], case["vocab"], case["width"], case["k"]
    n = max(1, round(T * case["scored"]))
    op = case["op"]
    head = 2 * V * D + (2 * V if case["bias"] else 0)
    if op == "logits":
        return dict(bytes=head + 2 * T * D + 2 * T * V, flops=2 * T * V * D)
    if op == "logits_bwd":
        return dict(bytes=2 * head + 4 * T * D + (4 if case["cap"] else 2) * T * V, flops=4 * T * V * D)
    scalars = T * (1 + 4 + (8 if case["tau"] == 1.0 else 0) + (4 if k else 0)) + 8 * n * k
    if op == "score":
        return dict(bytes=head + 2 * n * D + scalars, flops=2 * n * V * D)
    return dict(bytes=2 * head + 2 * n * D + 2 * T * D + scalars, flops=6 * n * V * D)


def exact(case, seed):
    s = prepare(case, seed)
    T, V, op, cap, tau = case["tokens"], case["vocab"], case["op"], case["cap"], case["tau"]
    f64 = torch.float64
    W, H = s["weight"].to(f64), s["hidden"].to(f64)
    b = s["bias"].to(f64) if case["bias"] else torch.zeros((), dtype=f64, device=W.device)
    step = max(1, CHUNK // 2 // V)
    dev = W.device

    def head(a, e):
        y = torch.addmm(b.expand(V), H[a:e], W.T)
        return torch.tanh(y.div_(cap)).mul_(cap) if cap else y

    if op == "logits":
        # rounded as the output is: 64-bit logits of every position would not fit
        if T * V > 1 << 30:
            return dict(logits=None)
        return dict(logits=torch.cat([head(a, min(T, a + step)) for a in range(0, T, step)]))
    dH, dW = torch.zeros_like(H), torch.zeros_like(W)
    dB = torch.zeros(V, dtype=f64, device=dev)
    nll, lse, kd = (torch.zeros(T, dtype=f64, device=dev) for _ in range(3))
    for a in range(0, T, step):
        e = min(T, a + step)
        if op == "logits_bwd":
            D = s["dlogits"][a:e].to(f64)
            if cap:
                D = D * (1 - torch.square(s["logits"][a:e].to(f64) / cap))
        else:
            on = s["mask"][a:e].to(f64)
            x = head(a, e)
            L = torch.logsumexp(x / tau, 1)
            i = torch.arange(e - a, device=dev)
            y = s["labels"][a:e].long()
            lse[a:e], nll[a:e] = L * on, (L - x[i, y]) * on
            P = torch.exp(x / tau - L[:, None])
            D = P * (s["grad_scale"] / tau + s["ce_scale"])
            if case["k"]:
                ids = s["idx"][a:e].long()
                q = torch.log_softmax(s["val"][a:e].to(f64) / tau, 1)
                kd[a:e] = on * torch.sum(q.exp() * (q - x.gather(1, ids) / tau + L[:, None]), 1)
                D.scatter_add_(1, ids, q.exp() * (-s["grad_scale"] / tau))
            D[i, y] -= s["ce_scale"]
            if cap:
                D *= 1 - torch.square(x / cap)
            D *= on[:, None]
        if op != "score":
            dH[a:e] = D @ W
            dW.addmm_(D.T, H[a:e])
            dB += D.sum(0)
    out = {}
    if op != "logits_bwd":
        if tau == 1.0:
            out = dict(nll=nll, lse=lse)
        if case["k"]:
            out["kd"] = kd
    if op != "score":
        out["grad_hidden"], out["grad_weight"] = dH, dW
        if case["bias"]:
            out["grad_bias"] = dB
    return out
