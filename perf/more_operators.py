"""Gated linear layer, token scores and distillation, and what their speed is judged by.

Three operators beside the linear layer and the vocabulary loss, each forward
only and as a training step:

* ``gated``         y = act(x wg^T + bg) * (x wu^T + bu): both projections of a
                    gated feed-forward block, the activation and the product;
                    w holds the d_hidden rows of wg, then those of wu
* ``gated_train``   the same, then the gradients of x, w and bias for a given dy
* ``scores``        per row of logits / temperature the log probability of a
                    given token, the entropy of the distribution and the
                    ``top`` most likely entries with their log probabilities
* ``scores_train``  the same, then the gradient of the logits for given
                    gradients of log probability and entropy
* ``distill``       divergence of the student's distribution h w^T / temperature
                    from a teacher's, of which the logits of its ``top`` most
                    likely entries are known
* ``distill_train`` the same, then the gradients of h and w

``own`` selects between the plain form (elementary torch operations in 32
bits, rounded once at the end) and the library's calls.

``excluded`` names a vocabulary entry that is never predicted (the mask token);
-1 for none. A row of the distillation counts where its weight is not zero; the
others (tokens that a masked objective left visible) have loss 0 and no
gradient. A teacher's entry -1 stands for none: a row may have fewer than
``top``.

Sizes: width 448 and 832, MLP ratio 4, 8 x 2048 tokens and blocks of 256 are
those of this library's layers; vocabularies are generic.
"""

import math

import torch

own = False

GELU_A = math.sqrt(2.0 / math.pi)
GELU_B = 0.044715
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token through a gated block while serving: latency, and the weights read once
        dict(name="gated_token", kind="gated", rows=1, d_in=832, d_hidden=3328, act="silu", bias=False, dtype="bf16",
             strided=False),
        # a denoising block of 256 tokens
        dict(name="gated_block", kind="gated", rows=256, d_in=832, d_hidden=3328, act="silu", bias=False,
             dtype="bf16", strided=False),
        # training step over a batch of 8 x 2048 tokens
        dict(name="gated_train_16k", kind="gated_train", rows=16384, d_in=832, d_hidden=3328, act="silu", bias=False,
             dtype="bf16", strided=False),
        # fp32 training step of ragged sizes with biases, x and dy slices of wider buffers
        dict(name="gated_train_odd_f32", kind="gated_train", rows=1001, d_in=451, d_hidden=1189, act="gelu",
             bias=True, dtype="f32", strided=True),
        # the sampler after one token's fp32 logits: confidence and the likeliest alternatives
        dict(name="scores_token", kind="scores", rows=1, vocab=50304, top=8, temperature=0.7, excluded=-1, token=False,
             dtype="f32", strided=False),
        # a denoising step chooses which tokens of a block of 256 to keep by their log probability and entropy; logits
        # of odd width inside wider rows
        dict(name="scores_block", kind="scores", rows=256, vocab=50021, top=1, temperature=1.0, excluded=50020,
             token=True, dtype="bf16", strided=True),
        # a teacher's likeliest entries for a training batch of 8 x 2048 tokens
        dict(name="scores_16k", kind="scores", rows=16384, vocab=50304, top=16, temperature=1.0, excluded=50303,
             token=True, dtype="bf16", strided=False),
        # a policy step: log probabilities of the sampled tokens with an entropy bonus, and the gradient of the logits
        dict(name="scores_train", kind="scores_train", rows=4096, vocab=32000, top=0, temperature=1.0, excluded=-1,
             token=True, dtype="f32", strided=False),
        # how far a student is from its teacher on a short answer
        dict(name="distill_answer", kind="distill", rows=24, d_model=832, vocab=50304, top=16, temperature=1.0,
             counted=1.0, excluded=-1, ragged=False, dtype="bf16"),
        # one training block of 256 tokens, half of them masked, over a vocabulary of odd size
        dict(name="distill_train_block", kind="distill_train", rows=256, d_model=448, vocab=50021, top=8,
             temperature=1.0, counted=0.5, excluded=50020, ragged=True, dtype="bf16"),
        # a training batch of 8 x 2048 tokens, half of them masked, softened distributions
        dict(name="distill_train_16k", kind="distill_train", rows=16384, d_model=832, vocab=50304, top=32,
             temperature=2.0, counted=0.5, excluded=50303, ragged=False, dtype="bf16"),
        # fp32, every row counted, a small vocabulary, many entries
        dict(name="distill_train_f32", kind="distill_train", rows=1000, d_model=448, vocab=8191, top=64,
             temperature=1.0, counted=1.0, excluded=-1, ragged=True, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size over the logarithm of the range: as it comes, or a multiple of 64 (of 8 below that)."""
    n = _log(rng, lo, hi)
    step = rng.choice((1, 8, 64))
    return n if step == 1 else min(hi, max(lo, (n + step - 1) // step * step))


def draw(rng):
    kind = rng.choice(("gated", "gated_train", "gated_train", "scores", "scores", "scores_train", "distill",
                       "distill_train", "distill_train"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    most = [work(c) for c in listed()]
    while True:
        if kind.startswith("gated"):
            case = dict(kind=kind, rows=_size(rng, 1, 16384), d_in=_size(rng, 64, 1664), d_hidden=_size(rng, 64, 3328),
                        act=rng.choice(("silu", "silu", "gelu", "none")), bias=rng.random() < 0.4, dtype=dtype,
                        strided=rng.random() < 0.25)
        elif kind.startswith("scores"):
            vocab = _size(rng, 500, 131072)
            case = dict(kind=kind, rows=_size(rng, 1, 16384), vocab=vocab,
                        top=0 if rng.random() < 0.25 else _size(rng, 1, 64),
                        temperature=rng.choice((1.0, rng.uniform(0.5, 2.0))), excluded=rng.choice((-1, vocab - 1)),
                        token=kind == "scores_train" or rng.random() < 0.7, dtype=rng.choice((dtype, "f32")),
                        strided=rng.random() < 0.25)
        else:
            vocab = _size(rng, 500, 50304)
            case = dict(kind=kind, rows=_size(rng, 1, 16384), d_model=_size(rng, 64, 1664), vocab=vocab,
                        top=_size(rng, 1, 64), temperature=rng.choice((1.0, rng.uniform(0.5, 4.0))),
                        counted=rng.choice((1.0, rng.uniform(0.05, 1.0))), excluded=rng.choice((-1, vocab - 1)),
                        ragged=rng.random() < 0.5, dtype=dtype)
        w = work(case)
        if w["flops"] <= max(m["flops"] for m in most) and w["bytes"] <= max(m["bytes"] for m in most):
            return case


def _counted(case):
    return max(1, int(round(case["rows"] * case["counted"])))


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    t = case["rows"]
    if case["kind"].startswith("gated"):
        k, n = case["d_in"], case["d_hidden"]
        b = 2 * n * e if case["bias"] else 0
        data = t * k * e + 2 * n * k * e + b + t * n * e
        flops = 4 * t * k * n
        if case["kind"] == "gated_train":
            # dy read, the gradients of x, w and bias written
            data += t * n * e + t * k * e + 2 * n * k * e + b
            flops *= 3
        return {"bytes": data, "flops": flops}
    if case["kind"].startswith("scores"):
        v, k = case["vocab"], case["top"]
        # the logits; per row its entropy, the token and its log probability, and the likeliest entries
        data = t * v * e + t * (4 + (8 + 4 if case["token"] else 0) + k * (8 + 4))
        flops = 4 * t * v
        if case["kind"] == "scores_train":
            data += t * v * e + t * 8
            flops *= 2
        return {"bytes": data, "flops": flops}
    k, v, n = case["d_model"], case["vocab"], case["top"]
    c = _counted(case)
    # the rows that count, the weights, the teacher's entries, the weight, loss and log sum of each row
    data = c * k * e + v * k * e + c * n * (8 + 4) + t * (4 + 4 + 4)
    flops = 2 * c * k * v
    if case["kind"] == "distill_train":
        data += t * 4 + t * k * e + v * k * e
        flops *= 3
    return {"bytes": data, "flops": flops}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(shape, std, dtype):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

    def uniform(shape):
        return torch.rand(shape, generator=g, device="cuda")

    s = {"case": case, "kept": {}}
    dt, t = TYPES[case["dtype"]], case["rows"]
    if case["kind"].startswith("gated"):
        k, n = case["d_in"], case["d_hidden"]
        # activations after a norm; weights as at initialisation, so that x w^T is near N(0, 1)
        s["x"] = normal((t, k + 64 if case["strided"] else k), 1.0, dt)[:, :k]
        s["w"] = normal((2 * n, k), 1.0 / math.sqrt(k), dt)
        s["bias"] = normal((2 * n,), 0.3, dt) if case["bias"] else None
        if case["kind"] == "gated_train":
            s["dy"] = normal((t, n + 64 if case["strided"] else n), 1.0, dt)[:, :n]
        return s
    v = case["vocab"]
    if case["kind"].startswith("scores"):
        # logits of a trained head: a spread of a few units, and in most rows one entry that stands out, which is
        # also the token asked for
        z = torch.empty((t, v + 7 if case["strided"] else v), device="cuda", dtype=dt)[:, :v]
        for a in range(0, t, 4096):
            z[a:a + 4096] = torch.randn((min(4096, t - a), v), generator=g, device="cuda") * 2.5
        token = torch.randint(0, v - 1, (t,), generator=g, device="cuda")  # never the last entry
        z[torch.arange(t, device="cuda"), token] += (uniform((t,)) * 14.0).to(dt)
        s["logits"], s["token"] = z, token if case["token"] else None
        if case["kind"] == "scores_train":
            # advantages over the batch, and the weight of an entropy bonus
            s["dlogp"] = normal((t,), 1.0, torch.float32)
            s["dentropy"] = 0.01 + 0.01 * uniform((t,))
        return s
    k, n = case["d_model"], case["top"]
    s["h"] = normal((t, k), 1.0, dt)
    s["w"] = normal((v, k), 2.0 / math.sqrt(k), dt)
    # the teacher's entries: distinct, never the last one, their logits falling
    first = torch.randint(0, v - 1, (t, 1), generator=g, device="cuda")
    step = torch.randint(1, max(2, (v - 1) // n), (t, 1), generator=g, device="cuda")
    j = torch.arange(n, device="cuda")
    s["ids"] = (first + step * j) % (v - 1)
    s["teacher"] = (12.0 + normal((t, n), 2.0, torch.float32)).sort(1, descending=True).values
    if case["ragged"]:
        have = torch.randint(1, n + 1, (t, 1), generator=g, device="cuda")
        s["ids"] = torch.where(j < have, s["ids"], torch.full_like(s["ids"], -1))
    # a masked objective: the rows that count are the masked tokens, weighted by 1 / (mask ratio)
    c = _counted(case)
    rows = torch.randperm(t, generator=g, device="cuda")[:c]
    ratio = uniform((t,)) * 0.9 + 0.1
    weight = torch.zeros((t,), device="cuda")
    weight[rows] = 1.0 / ratio[rows] / t
    s["weight"] = weight
    if case["kind"] == "distill_train":
        s["dloss"] = torch.ones((t,), device="cuda")
    return s


# ---------------------------------------------------------------------------
# plain form: elementary operations in 32 bits, one rounding at the end
# ---------------------------------------------------------------------------
def _act(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "silu":
        sg = torch.sigmoid(z)
        return z * sg, sg * (1 + z * (1 - sg))
    th = torch.tanh(GELU_A * (z + GELU_B * z * z * z))
    return 0.5 * z * (1 + th), 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * GELU_A * (1 + 3 * GELU_B * z * z)


def _plain_gated(s):
    case = s["case"]
    dt, n = TYPES[case["dtype"]], case["d_hidden"]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    a, d = _act(z[:, :n], case["act"])
    up = z[:, n:]
    r = {"y": (a * up).to(dt)}
    if case["kind"] == "gated":
        return r
    dy = s["dy"].float()
    dz = torch.cat((dy * up * d, dy * a), 1)
    r["dx"] = (dz @ w).to(dt)
    r["dw"] = (dz.t() @ x).to(dt)
    if s["bias"] is not None:
        r["dbias"] = dz.sum(0).to(dt)
    return r


def _plain_scores(s):
    case = s["case"]
    z = s["logits"].float() * (1.0 / case["temperature"])
    t, v = z.shape
    if case["excluded"] >= 0:
        z[:, case["excluded"]] = -math.inf
    r = {}
    if case["top"] > 0:
        # 64-bit keys that order by value, then by lower index: the bits of a float as an integer of the same order
        # (0 added: there is one zero), the index below them
        bits = (z + 0.0).view(torch.int32)
        bits = bits ^ ((bits >> 31) & 0x7FFFFFFF)
        keys = bits.long() * (1 << 32) + (v - 1 - torch.arange(v, device=z.device))
        ids = v - 1 - (torch.topk(keys, min(case["top"], v), dim=1).values & 0xFFFFFFFF)
        top = torch.gather(z, 1, ids)
        ids = torch.where(top == -math.inf, torch.full_like(ids, -1), ids)
        del bits, keys
    m = z.amax(1, keepdim=True)
    z = z.sub_(m)
    p = z.exp()
    total = p.sum(1, keepdim=True)
    log_total = total.log()
    r["entropy"] = (log_total - torch.where(p > 0, p * z, 0.0).sum(1, keepdim=True) / total).squeeze(1)
    if case["top"] > 0:
        r["ids"], r["top"] = ids, top - m - log_total
    if s["token"] is None:
        return r
    r["logp"] = (torch.gather(z, 1, s["token"][:, None]) - log_total).squeeze(1)
    if case["kind"] == "scores":
        return r
    p = p.div_(total)
    logp = torch.where(p > 0, z.sub_(log_total), 0.0)
    g = logp.add_(r["entropy"][:, None]).mul_(-s["dentropy"][:, None]).sub_(s["dlogp"][:, None]).mul_(p)
    g.scatter_add_(1, s["token"][:, None], s["dlogp"][:, None])
    r["dlogits"] = (g * (1.0 / case["temperature"])).to(TYPES[case["dtype"]])
    return r


def _plain_distill(s):
    case = s["case"]
    dt, scale = TYPES[case["dtype"]], 1.0 / case["temperature"]
    h, w = s["h"].float(), s["w"].float()
    z = (h @ w.t()) * scale
    if case["excluded"] >= 0:
        z[:, case["excluded"]] = -math.inf
    known = (s["ids"] >= 0) & (s["ids"] != case["excluded"])
    ids = torch.where(known, s["ids"], torch.zeros_like(s["ids"]))
    counts = (s["weight"] != 0) & known.any(1)
    teacher = torch.where(known, s["teacher"] * scale, torch.full_like(s["teacher"], -math.inf))
    q = (teacher - teacher.amax(1, keepdim=True)).exp()
    total_q = q.sum(1, keepdim=True)
    log_q = teacher - teacher.amax(1, keepdim=True) - total_q.log()
    q = q / total_q
    m = z.amax(1, keepdim=True)
    log_p = torch.gather(z, 1, ids) - m
    p = z.sub_(m).exp_()
    total = p.sum(1, keepdim=True)
    log_p = log_p - total.log()
    zero = torch.zeros_like(s["weight"])
    loss = torch.where(known, q * (log_q - log_p), 0.0).sum(1)
    r = {"loss": torch.where(counts, loss * s["weight"], zero),
         "lse": torch.where(counts, (m + total.log()).squeeze(1), zero)}
    if case["kind"] == "distill":
        return r
    g = torch.where(counts, s["weight"] * s["dloss"], zero)[:, None] * scale
    p = p.mul_(g / total)
    p.scatter_add_(1, ids, -g * torch.where(known, q, 0.0))
    r["dh"] = (p @ w).to(dt)
    r["dw"] = (p.t() @ h).to(dt)
    return r


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _own_gated(s):
    from paper_2607_02805_gb300.dense import GatedLinear
    case, op = s["case"], s["kept"].get("op")
    if op is None:
        op = s["kept"]["op"] = GatedLinear(case["rows"], case["d_in"], case["d_hidden"], act=case["act"],
                                           dtype=TYPES[case["dtype"]])
    r = {"y": op.forward(s["x"], s["w"], s["bias"])}
    if case["kind"] == "gated_train":
        r["dx"], r["dw"], dbias = op.backward(s["x"], s["w"], s["dy"], s["bias"])
        if dbias is not None:
            r["dbias"] = dbias
    return r


def _own_scores(s):
    from paper_2607_02805_gb300.dense import TokenScores
    case, op = s["case"], s["kept"].get("op")
    if op is None:
        op = s["kept"]["op"] = TokenScores(case["rows"], case["vocab"], top=case["top"], dtype=TYPES[case["dtype"]],
                                           excluded=case["excluded"], temperature=case["temperature"])
    logp, entropy, ids, top = op.forward(s["logits"], s["token"])
    r = {"entropy": entropy}
    if case["top"] > 0:
        r["ids"], r["top"] = ids, top
    if logp is not None:
        r["logp"] = logp
    if case["kind"] == "scores_train":
        r["dlogits"] = op.backward(s["logits"], s["token"], s["dlogp"], s["dentropy"])
    return r


def _own_distill(s):
    from paper_2607_02805_gb300.dense import DistillLoss
    case, op = s["case"], s["kept"].get("op")
    if op is None:
        op = s["kept"]["op"] = DistillLoss(case["rows"], case["d_model"], case["vocab"], case["top"],
                                           dtype=TYPES[case["dtype"]], excluded=case["excluded"],
                                           temperature=case["temperature"])
    loss, lse = op.forward(s["h"], s["w"], s["ids"], s["teacher"], s["weight"])
    r = {"loss": loss, "lse": lse}
    if case["kind"] == "distill_train":
        r["dh"], r["dw"] = op.backward(s["h"], s["w"], s["ids"], s["teacher"], s["weight"], s["dloss"])
    return r


def run(state):
    kind = state["case"]["kind"].split("_")[0]
    if own:
        return {"gated": _own_gated, "scores": _own_scores, "distill": _own_distill}[kind](state)
    return {"gated": _plain_gated, "scores": _plain_scores, "distill": _plain_distill}[kind](state)


# ---------------------------------------------------------------------------
# 64-bit values, from the definitions
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"].split("_")[0]
    with torch.enable_grad():
        return {"gated": _exact_gated, "scores": _exact_scores, "distill": _exact_distill}[kind](case, s)


def _exact_gated(case, s):
    x = s["x"].double().requires_grad_(True)
    w = s["w"].double().requires_grad_(True)
    b = s["bias"].double().requires_grad_(True) if s["bias"] is not None else None
    gate, up = torch.einsum("tk,jnk->jtn", x, w.view(2, case["d_hidden"], case["d_in"]))
    if b is not None:
        gate, up = gate + b.view(2, 1, -1)[0], up + b.view(2, 1, -1)[1]
    if case["act"] == "silu":
        y = up * gate / (1 + torch.exp(-gate))
    elif case["act"] == "gelu":  # 0.5 (1 + tanh u) = 1 / (1 + exp(-2 u))
        y = up * gate / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (gate + 0.044715 * gate ** 3)))
    else:
        y = up * gate
    r = {"y": y.detach()}
    if case["kind"] == "gated":
        return r
    grads = torch.autograd.grad(y, [x, w] + ([b] if b is not None else []), s["dy"].double())
    r["dx"], r["dw"] = grads[0], grads[1]
    if b is not None:
        r["dbias"] = grads[2]
    return r


def _exact_scores(case, s):
    t, v, k = case["rows"], case["vocab"], case["top"]
    parts = []
    for a in range(0, t, 1024):
        x = s["logits"][a:a + 1024].double().requires_grad_(True)
        hide = torch.zeros(v, dtype=torch.bool, device="cuda")
        if case["excluded"] >= 0:
            hide[case["excluded"]] = True
        z = (x / case["temperature"]).masked_fill(hide[None, :], -math.inf)
        logp = torch.log_softmax(z, 1)
        safe = logp.masked_fill(hide[None, :], 0.0)
        entropy = -(safe.exp().masked_fill(hide[None, :], 0.0) * safe).sum(1)
        r = {"entropy": entropy.detach()}
        if k > 0:
            best, ids = torch.sort(logp.detach(), dim=1, descending=True, stable=True)
            # equal logits have equal log probabilities; different ones may too after rounding, so the logits decide
            order = torch.sort(z.detach(), dim=1, descending=True, stable=True).indices[:, :k]
            r["ids"] = torch.where(best[:, :k] == -math.inf, torch.full_like(ids[:, :k], -1), order)
            r["top"] = best[:, :k]
            del best, ids, order
        if s["token"] is not None:
            chosen = logp[torch.arange(x.shape[0], device="cuda"), s["token"][a:a + 1024]]
            r["logp"] = chosen.detach()
            if case["kind"] == "scores_train":
                of = (chosen * s["dlogp"][a:a + 1024].double() + entropy * s["dentropy"][a:a + 1024].double()).sum()
                r["dlogits"] = torch.autograd.grad(of, x)[0]
        parts.append(r)
    return {name: torch.cat([p[name] for p in parts]) for name in parts[0]}


def _exact_distill(case, s):
    t = case["rows"]
    w = s["w"].double()
    keep = torch.ones(case["vocab"], dtype=torch.bool, device="cuda")
    if case["excluded"] >= 0:
        keep[case["excluded"]] = False
    rows = torch.nonzero(s["weight"]).squeeze(1)
    loss = torch.zeros(t, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(loss)
    train = case["kind"] == "distill_train"
    if train:
        dh = torch.zeros(t, case["d_model"], dtype=torch.float64, device="cuda")
        dw = torch.zeros_like(w)
    for part in rows.split(2048):
        h = s["h"][part].double()
        z = torch.einsum("tk,vk->tv", h, w) / case["temperature"]
        z = torch.where(keep[None, :], z, torch.full_like(z, -math.inf))
        l = torch.logsumexp(z, 1)
        lse[part] = l
        # the teacher's distribution over the whole vocabulary, zero where it is not known
        ids, known = s["ids"][part], s["ids"][part] >= 0
        q = torch.softmax(torch.where(known, s["teacher"][part].double() / case["temperature"], -math.inf), 1)
        full = torch.zeros_like(z).scatter_add_(1, ids.clamp(min=0), q)
        n = torch.nonzero(full, as_tuple=True)
        terms = torch.zeros_like(z)
        terms[n] = full[n] * (full[n].log() - z[n] + l[n[0]])
        wt = s["weight"][part].double()
        loss[part] = wt * terms.sum(1)
        if train:
            dz = torch.exp(z - l[:, None]) - full
            dz *= (wt * s["dloss"][part].double() / case["temperature"])[:, None]
            dh[part] = torch.einsum("tv,vk->tk", dz, w)
            dw += torch.einsum("tv,tk->vk", dz, h)
    r = {"loss": loss, "lse": lse}
    if train:
        r["dh"], r["dw"] = dh, dw
    return r
