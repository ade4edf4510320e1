"""The dense operators around the mixers, and what their speed is judged by.

Two operators, each forward only and as a training step:

* ``linear``      y = residual + act(x w^T + bias): the MLP of a block, the
                  projections around a mixer, and the logits of single tokens
* ``linear_train`` the same, then the gradients of x, w and bias for a given dy
* ``loss``        weighted softmax cross entropy of h w^T over the vocabulary
                  at the rows that count, without keeping the logits
* ``loss_train``  the same, then the gradients of h and w

``own`` selects between the plain form (elementary torch operations in 32
bits, rounded once at the end) and the library's calls.

A row of the loss counts where its target is in the vocabulary and its weight
is not zero; the others (the tokens that a masked objective left visible) have
loss 0 and no gradient. ``excluded`` names a vocabulary entry that is never
predicted (the mask token); -1 for none.

Sizes: width 448 and 832, MLP ratio 4, 8 x 2048 tokens and the block sizes are
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
        # one token through an up projection while serving: latency, and the weights read once
        dict(name="linear_token", kind="linear", rows=1, d_in=832, d_out=3328, act="gelu", bias=True, residual=False,
             dtype="bf16", out="bf16", strided=False),
        # the logits of one token: the largest weight matrix there is, in fp32 for the sampler
        dict(name="linear_logits_token", kind="linear", rows=1, d_in=832, d_out=50304, act="none", bias=False,
             residual=False, dtype="bf16", out="f32", strided=False),
        # a denoising block of 32 tokens through the down projection, added to the residual stream; few rows, long sum
        dict(name="linear_block_down", kind="linear", rows=32, d_in=3328, d_out=832, act="none", bias=True,
             residual=True, dtype="bf16", out="bf16", strided=False),
        # the up projection over a training batch of 8 x 2048 tokens, read from a slice of a wider buffer
        dict(name="linear_up_16k", kind="linear", rows=16384, d_in=832, d_out=3328, act="gelu", bias=True,
             residual=False, dtype="bf16", out="bf16", strided=True),
        # ragged sizes in fp32, the precision of the smallest configurations
        dict(name="linear_odd_f32", kind="linear", rows=777, d_in=451, d_out=1789, act="silu", bias=True,
             residual=True, dtype="f32", out="f32", strided=False),
        # training step of the up projection
        dict(name="linear_train_up_16k", kind="linear_train", rows=16384, d_in=832, d_out=3328, act="gelu", bias=True,
             residual=False, dtype="bf16", out="bf16", strided=False),
        # training step of a down projection of ragged sizes with its residual
        dict(name="linear_train_odd", kind="linear_train", rows=3001, d_in=1789, d_out=451, act="silu", bias=True,
             residual=True, dtype="bf16", out="bf16", strided=False),
        # fp32 training step at the smaller width
        dict(name="linear_train_f32", kind="linear_train", rows=2048, d_in=448, d_out=1792, act="gelu", bias=True,
             residual=False, dtype="f32", out="f32", strided=False),
        # log likelihoods of a short answer: few rows over the whole vocabulary
        dict(name="loss_answer", kind="loss", rows=24, d_model=832, vocab=50304, counted=1.0, excluded=-1,
             dtype="bf16"),
        # one training block of 256 tokens, half of them masked, over a vocabulary of odd size
        dict(name="loss_train_block", kind="loss_train", rows=256, d_model=448, vocab=50021, counted=0.5,
             excluded=50020, dtype="bf16"),
        # the loss of a training batch of 8 x 2048 tokens, half of them masked
        dict(name="loss_train_16k", kind="loss_train", rows=16384, d_model=832, vocab=50304, counted=0.5,
             excluded=50303, dtype="bf16"),
        # fp32, every row counted, a small vocabulary
        dict(name="loss_train_f32", kind="loss_train", rows=1000, d_model=448, vocab=8191, counted=1.0, excluded=-1,
             dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size over the logarithm of the range: as it comes, or a multiple of 64 (of 8 below that)."""
    n = _log(rng, lo, hi)
    step = rng.choice((1, 8, 64))
    return n if step == 1 else min(hi, max(lo, (n + step - 1) // step * step))


def draw(rng):
    kind = rng.choice(("linear", "linear", "linear_train", "linear_train", "loss", "loss_train", "loss_train"))
    dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
    while True:
        if kind.startswith("linear"):
            case = dict(kind=kind, rows=_size(rng, 1, 16384), d_in=_size(rng, 64, 3328), d_out=_size(rng, 64, 3328),
                        act=rng.choice(("none", "silu", "gelu")), bias=rng.random() < 0.7,
                        residual=rng.random() < 0.4, dtype=dtype, out=dtype, strided=rng.random() < 0.25)
            if kind == "linear" and dtype == "bf16" and rng.random() < 0.2:
                case["out"] = "f32"
        else:
            vocab = _size(rng, 500, 50304)
            case = dict(kind=kind, rows=_size(rng, 1, 16384), d_model=_size(rng, 64, 1664), vocab=vocab,
                        counted=rng.choice((1.0, rng.uniform(0.05, 1.0))),
                        excluded=rng.choice((-1, vocab - 1)), dtype=dtype)
        if work(case)["flops"] <= work(listed()[10])["flops"]:
            return case


def _counted(case):
    return max(1, int(round(case["rows"] * case["counted"])))


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["kind"].startswith("linear"):
        t, k, n = case["rows"], case["d_in"], case["d_out"]
        o = 4 if case["out"] == "f32" else 2
        b = n * e if case["bias"] else 0
        data = t * k * e + n * k * e + b + t * n * o * (2 if case["residual"] else 1)
        flops = 2 * t * k * n
        if case["kind"] == "linear_train":
            # dy read, the gradients of x, w and bias written
            data += t * n * o + t * k * e + n * k * e + b
            flops *= 3
        return {"bytes": data, "flops": flops}
    t, k, v = case["rows"], case["d_model"], case["vocab"]
    c = _counted(case)
    # the rows that count, the weights, targets and weights of the rows, loss and log sum of each row
    data = c * k * e + v * k * e + t * (8 + 4) + t * (4 + 4)
    flops = 2 * c * k * v
    if case["kind"] == "loss_train":
        data += t * 4 + t * k * e + v * k * e
        flops *= 3
    return {"bytes": data, "flops": flops}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))

    def normal(shape, std, dtype):
        return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)

    s = {"case": case, "kept": {}}
    dt = TYPES[case["dtype"]]
    if case["kind"].startswith("linear"):
        t, k, n = case["rows"], case["d_in"], case["d_out"]
        out = TYPES[case["out"]]
        # activations after a norm; weights as at initialisation, so that x w^T is near N(0, 1)
        x = normal((t, k + 64 if case["strided"] else k), 1.0, dt)
        s["x"] = x[:, :k]
        s["w"] = normal((n, k), 1.0 / math.sqrt(k), dt)
        s["bias"] = normal((n,), 0.3, dt) if case["bias"] else None
        s["residual"] = normal((t, n), 1.0, out) if case["residual"] else None
        if case["kind"] == "linear_train":
            s["dy"] = normal((t, n), 1.0, out)
        return s
    t, k, v = case["rows"], case["d_model"], case["vocab"]
    s["h"] = normal((t, k), 1.0, dt)
    s["w"] = normal((v, k), 2.0 / math.sqrt(k), dt)
    s["target"] = torch.randint(0, v - 1, (t,), generator=g, device="cuda")  # never the last entry
    # a masked objective: the rows that count are the masked tokens, weighted by 1 / (mask ratio)
    c = _counted(case)
    rows = torch.randperm(t, generator=g, device="cuda")[:c]
    ratio = torch.rand((t,), generator=g, device="cuda") * 0.9 + 0.1
    weight = torch.zeros((t,), device="cuda")
    weight[rows] = 1.0 / ratio[rows] / t
    s["weight"] = weight
    if case["kind"] == "loss_train":
        s["dloss"] = torch.ones((t,), device="cuda")
    return s


# ---------------------------------------------------------------------------
# plain form: elementary operations in 32 bits, one rounding at the end
# ---------------------------------------------------------------------------
def _act(z, act):
    """The activation and its derivative."""
    if act == "none":
        return z, None
    if act == "silu":
        sg = torch.sigmoid(z)
        return z * sg, sg * (1 + z * (1 - sg))
    th = torch.tanh(GELU_A * (z + GELU_B * z * z * z))
    return 0.5 * z * (1 + th), 0.5 * (1 + th) + 0.5 * z * (1 - th * th) * GELU_A * (1 + 3 * GELU_B * z * z)


def _plain_linear(s):
    case = s["case"]
    dt, out = TYPES[case["dtype"]], TYPES[case["out"]]
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    if s["bias"] is not None:
        z = z + s["bias"].float()
    y, d = _act(z, case["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if case["kind"] == "linear":
        return {"y": y.to(out)}
    dz = s["dy"].float()
    if d is not None:
        dz = dz * d
    r = {"y": y.to(out), "dx": (dz @ w).to(dt), "dw": (dz.t() @ x).to(dt)}
    if s["bias"] is not None:
        r["dbias"] = dz.sum(0).to(dt)
    return r


def _plain_loss(s):
    case = s["case"]
    dt = TYPES[case["dtype"]]
    h, w, target = s["h"].float(), s["w"].float(), s["target"]
    z = h @ w.t()
    if case["excluded"] >= 0:
        z[:, case["excluded"]] = -math.inf
    m = z.amax(1, keepdim=True)
    counts = s["weight"] != 0
    at = torch.gather(z, 1, target[:, None])
    p = z.sub_(m).exp_()
    total = p.sum(1, keepdim=True)
    lse = (m + total.log()).squeeze(1)
    zero = torch.zeros_like(lse)
    r = {"loss": torch.where(counts, (lse - at.squeeze(1)) * s["weight"], zero), "lse": torch.where(counts, lse, zero)}
    if case["kind"] == "loss":
        return r
    g = torch.where(counts, s["weight"] * s["dloss"], zero)[:, None]
    p = p.mul_(g / total)
    p.scatter_add_(1, target[:, None], -g)
    r["dh"] = (p @ w).to(dt)
    r["dw"] = (p.t() @ h).to(dt)
    return r


# ---------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------
def _own_linear(s):
    from paper_2607_02805_gb300.dense import Linear
    case, op = s["case"], s["kept"].get("op")
    if op is None:
        op = s["kept"]["op"] = Linear(case["rows"], case["d_in"], case["d_out"], act=case["act"],
                                      dtype=TYPES[case["dtype"]], out_dtype=TYPES[case["out"]])
    if case["kind"] == "linear":
        return {"y": op.forward(s["x"], s["w"], s["bias"], s["residual"])}
    y = op.forward(s["x"], s["w"], s["bias"], s["residual"], save_pre=True)
    dx, dw, dbias = op.backward(s["x"], s["w"], s["dy"], bias=s["bias"] is not None)
    r = {"y": y, "dx": dx, "dw": dw}
    if dbias is not None:
        r["dbias"] = dbias
    return r


def _own_loss(s):
    from paper_2607_02805_gb300.dense import LmLoss
    case, op = s["case"], s["kept"].get("op")
    if op is None:
        op = s["kept"]["op"] = LmLoss(case["rows"], case["d_model"], case["vocab"], dtype=TYPES[case["dtype"]],
                                      excluded=case["excluded"])
    loss, lse = op.forward(s["h"], s["w"], s["target"], s["weight"])
    r = {"loss": loss, "lse": lse}
    if case["kind"] == "loss_train":
        r["dh"], r["dw"] = op.backward(s["h"], s["w"], s["target"], s["weight"], s["dloss"])
    return r


def run(state):
    linear = state["case"]["kind"].startswith("linear")
    if own:
        return _own_linear(state) if linear else _own_loss(state)
    return _plain_linear(state) if linear else _plain_loss(state)


# ---------------------------------------------------------------------------
# 64-bit values, from the definitions
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    with torch.enable_grad():
        return _exact_linear(case, s) if case["kind"].startswith("linear") else _exact_loss(case, s)


def _exact_linear(case, s):
    x = s["x"].double().requires_grad_(True)
    w = s["w"].double().requires_grad_(True)
    b = s["bias"].double().requires_grad_(True) if s["bias"] is not None else None
    z = torch.einsum("tk,nk->tn", x, w)
    if b is not None:
        z = z + b[None, :]
    if case["act"] == "silu":
        y = z / (1 + torch.exp(-z))
    elif case["act"] == "gelu":  # 0.5 (1 + tanh u) = 1 / (1 + exp(-2 u))
        y = z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    else:
        y = z
    r = {"y": y.detach() if s["residual"] is None else y.detach() + s["residual"].double()}
    if case["kind"] == "linear":
        return r
    wrt = [x, w] + ([b] if b is not None else [])
    grads = torch.autograd.grad(y, wrt, s["dy"].double())
    r["dx"], r["dw"] = grads[0], grads[1]
    if b is not None:
        r["dbias"] = grads[2]
    return r


def _exact_loss(case, s):
    t = case["rows"]
    w = s["w"].double()
    keep = torch.ones(case["vocab"], dtype=torch.bool, device="cuda")
    if case["excluded"] >= 0:
        keep[case["excluded"]] = False
    rows = torch.nonzero(s["weight"]).squeeze(1)
    loss = torch.zeros(t, dtype=torch.float64, device="cuda")
    lse = torch.zeros_like(loss)
    train = case["kind"] == "loss_train"
    if train:
        dh = torch.zeros(t, case["d_model"], dtype=torch.float64, device="cuda")
        dw = torch.zeros_like(w)
    for part in rows.split(2048):
        h = s["h"][part].double()
        z = torch.einsum("tk,vk->tv", h, w)
        z = torch.where(keep[None, :], z, torch.full_like(z, -math.inf))
        l = torch.logsumexp(z, 1)
        n = torch.arange(part.numel(), device="cuda")
        lse[part] = l
        wt = s["weight"][part].double()
        loss[part] = wt * (l - z[n, s["target"][part]])
        if train:
            dz = torch.exp(z - l[:, None])
            dz[n, s["target"][part]] -= 1
            dz *= (wt * s["dloss"][part].double())[:, None]
            dh[part] = torch.einsum("tv,vk->tk", dz, w)
            dw += torch.einsum("tv,tk->vk", dz, h)
    r = {"loss": loss, "lse": lse}
    if train:
        r["dh"], r["dw"] = dh, dw
    return r
