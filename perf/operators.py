"""Cases of the operators that a client needs for its sensitivity map, the scores that he_select_mask takes.

The map (Algorithm 1, Step 1 of Selective Parameter Encryption) is, for every parameter w, the mean over the client's samples
k of |d/dy_k (d loss / dw)|.  For a language model under cross entropy the derivative by the label's coordinate is, up to its
sign, the gradient of the log probability of the sample's tokens.  A pass over a batch needs

  log_probs        log probabilities of given tokens from logits, with the entropy and the top alternatives of every row,
  log_probs_grad   their gradient back to the logits, from which the backward pass through the model starts,
  norm, norm_grad  layer norm forward and backward; with samples, the weights' gradients are summed within a sample, and their
                   magnitudes over the samples,
  linear           the same for a linear layer: the sum over samples of |dY_k^T X_k| (X_k, dY_k: the sample's rows of the layer's inputs
                   and of its outputs' gradients).

Rows of a sample lie together; `offsets` holds where samples begin and end, and rows behind the last one are padding.
"""
import math

import torch

own = False


# --------------------------------------------------------------------------- cases

def _case(name, op, dtype, **sizes):
    return {"name": name, "op": op, "dtype": dtype, **sizes}


def listed():
    return [
        # One generated token over a large vocabulary, with its 20 best alternatives: latency counts.
        _case("log-probs-one-row", "log_probs", "bf16", rows=1, vocab=131072, top=20, masked=False),
        # A client's few hundred tokens in fp32, a vocabulary of odd size, five alternatives, part of the vocabulary masked.
        _case("log-probs-333-f32", "log_probs", "f32", rows=333, vocab=50257, top=5, masked=True),
        # The largest batch of logits, eight alternatives for each token.
        _case("log-probs-2048", "log_probs", "bf16", rows=2048, vocab=131072, top=8, masked=False),
        # Gradient of log probabilities and entropies, a padded batch, half precision.
        _case("log-probs-grad-777-f16", "log_probs_grad", "f16", rows=777, vocab=30522, masked=True, entropy=True),
        # Where the backward pass of a large batch begins: log probabilities alone.
        _case("log-probs-grad-8192", "log_probs_grad", "bf16", rows=8192, vocab=32768, masked=False, entropy=False),
        # Layer norm of a single token.
        _case("norm-one-row", "norm", "bf16", rows=1, width=4096),
        # Layer norm of a long prompt.
        _case("norm-32768", "norm", "bf16", rows=32768, width=4096),
        # Backward pass of a training batch, gradients of the weights over all rows.
        _case("norm-grad-16384", "norm_grad", "bf16", rows=16384, width=1024, samples=0),
        # The same for the map: ragged samples, odd sizes, fp32.
        _case("norm-map-13333-f32", "norm_grad", "f32", rows=13333, width=1001, samples=97),
        # A small classifier head in fp32, odd sizes: the smallest product there is.
        _case("linear-map-small-f32", "linear", "f32", rows=500, outputs=101, inputs=333, samples=7),
        # A feed-forward layer over a batch of ragged samples.
        _case("linear-map-16384", "linear", "bf16", rows=16384, outputs=1024, inputs=4096, samples=128),
        # Every token a sample of its own.
        _case("linear-map-tokens-f16", "linear", "f16", rows=8192, outputs=2048, inputs=2048, samples=-1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["log_probs", "log_probs_grad", "norm", "norm_grad", "norm_grad", "linear", "linear"])
    dtype = rng.choice(["bf16", "f16", "f32"])
    if op in ("log_probs", "log_probs_grad"):
        vocab = _log_int(rng, 100, 131072)
        rows = _log_int(rng, 1, min(8192, (1 << 27) // vocab))
        c = _case("", op, dtype, rows=rows, vocab=vocab, masked=rng.random() < 0.5)
        if op == "log_probs":
            c["top"] = min(vocab, rng.choice([0, 1, 5, 8, 20, 32]))
        else:
            c["entropy"] = rng.random() < 0.5
    elif op in ("norm", "norm_grad"):
        width = _log_int(rng, 8, 8192)
        rows = _log_int(rng, 1, min(32768, (1 << 24 if op == "norm_grad" else 1 << 26) // width))
        c = _case("", op, dtype, rows=rows, width=width)
        if op == "norm_grad":
            c["samples"] = 0 if rng.random() < 0.4 else _log_int(rng, 1, rows)
    else:
        outputs, inputs = _log_int(rng, 8, 4096), _log_int(rng, 8, 4096)
        most = 1.6e10 if dtype == "f32" else 6.4e10
        rows = _log_int(rng, 1, min(16384, most / (outputs * inputs)))
        c = _case("", op, dtype, rows=rows, outputs=outputs, inputs=inputs)
        c["samples"] = -1 if rng.random() < 0.3 else _log_int(rng, max(1, rows // 2000), min(rows, 256))
    del c["name"]
    return c


# --------------------------------------------------------------------------- inputs

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_EPS = 1e-5


def _cuts(rows, samples, seed):
    """Offsets of `samples` ragged samples in at most `rows` rows: some are empty, and a few rows of padding follow the last."""
    g = torch.Generator()
    g.manual_seed(seed)
    counted = rows - int(torch.randint(0, rows // 50 + 1, (1,), generator=g))
    inner = torch.randint(0, counted + 1, (samples - 1,), generator=g).sort().values
    return [0] + inner.tolist() + [counted]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype, op, rows = _TYPES[case["dtype"]], case["op"], case["rows"]
    s = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if op in ("log_probs", "log_probs_grad"):
        V = case["vocab"]
        # logits of a trained model: a few tokens of every row stand out
        z = normal(rows, V).mul_(2.0)
        lead = torch.randint(0, V, (rows, 4), generator=g, device="cuda")
        z.scatter_add_(1, lead, normal(rows, 4).mul_(2.0).add_(8.0))
        y = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.7, lead[:, 0], torch.randint(0, V, (rows,), generator=g, device="cuda"))
        if case["masked"]:
            # tokens that may not follow, and rows of padding, which have no target
            z.masked_fill_(torch.rand(V, generator=g, device="cuda") < 0.3, -math.inf)
            y = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.1, torch.full_like(y, -100), y)
        s["logits"], s["targets"] = z.to(dtype), y
        if op == "log_probs_grad":
            z = s["logits"].double()
            lse = torch.logsumexp(z, 1)
            logp = z - lse[:, None]
            s["lse"] = lse.float()
            s["entropy"] = -(logp.exp() * logp.masked_fill(logp == -math.inf, 0.0)).sum(1).float()
            del z, logp
            s["dlogp"] = normal(rows).mul_(0.1).add_(1.0)
            s["dentropy"] = normal(rows).mul_(0.1) if case["entropy"] else None
    elif op in ("norm", "norm_grad"):
        D = case["width"]
        # activations: channels of different scale and offset
        x = normal(rows, D).mul_(torch.exp(normal(D).mul_(0.5))).add_(normal(D).mul_(0.3))
        s["x"] = x.to(dtype)
        s["weight"], s["bias"] = normal(D).mul_(0.1).add_(1.0), normal(D).mul_(0.1)
        if op == "norm_grad":
            s["dy"] = normal(rows, D).mul_(torch.exp(normal(rows, 1))).mul_(1e-2).to(dtype)
            x = s["x"].double()
            s["mean"] = x.mean(1).float()
            s["rstd"] = (x.var(1, correction=0) + _EPS).rsqrt().float()
    else:
        s["x"] = normal(rows, case["inputs"]).mul_(torch.exp(normal(case["inputs"]).mul_(0.5))).to(dtype)
        s["dy"] = normal(rows, case["outputs"]).mul_(torch.exp(normal(rows, 1))).mul_(1e-2).to(dtype)
    samples = case.get("samples", 0)
    if samples > 0:
        s["cuts"] = _cuts(rows, samples, seed)
        s["offsets"] = torch.tensor(s["cuts"], dtype=torch.int32, device="cuda")
    return s


# --------------------------------------------------------------------------- plain forms

def _log_probs(s):
    z, y, top = s["logits"].float(), s["targets"], s["case"]["top"]
    V = z.shape[1]
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    t = z - m
    e = torch.exp(t)
    total = e.sum(1)
    lse = m[:, 0] + torch.log(total)
    entropy = torch.log(total) - (e * torch.where(e > 0, t, torch.zeros_like(t))).sum(1) / total
    logp = torch.where(y < 0, torch.zeros_like(lse), z.gather(1, y.clamp(min=0)[:, None])[:, 0] - lse)
    del t, e
    if not top:
        return {"logp": logp, "lse": lse, "entropy": entropy}
    # order: the value, then the lowest index
    bits = torch.where(z == 0, torch.zeros_like(z), z).view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * 2 ** 32 + (V - 1 - torch.arange(V, device=z.device))
    ids = torch.topk(key, top, dim=1).indices
    return {"logp": logp, "lse": lse, "entropy": entropy, "top_logp": z.gather(1, ids) - lse[:, None], "top_ids": ids}


def _log_probs_grad(s):
    z, y = s["logits"].float(), s["targets"]
    lp = z - s["lse"][:, None]
    p = torch.exp(lp)
    g = torch.where(y < 0, torch.zeros_like(s["dlogp"]), s["dlogp"])
    grad = -p * g[:, None]
    if s["dentropy"] is not None:
        lp = torch.where(p > 0, lp, torch.zeros_like(lp))
        grad = grad - s["dentropy"][:, None] * p * (lp + s["entropy"][:, None])
    return {"dlogits": grad.scatter_add(1, y.clamp(min=0)[:, None], g[:, None]).to(s["logits"].dtype)}


def _norm(s):
    x = s["x"].float()
    mean = x.mean(1)
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).mean(1) + _EPS)
    return {"y": (d * rstd[:, None] * s["weight"] + s["bias"]).to(s["x"].dtype), "mean": mean, "rstd": rstd}


def _norm_grad(s):
    x, dy = s["x"].float(), s["dy"].float()
    n = (x - s["mean"][:, None]) * s["rstd"][:, None]
    dn = dy * s["weight"]
    dx = s["rstd"][:, None] * (dn - dn.mean(1, keepdim=True) - n * (dn * n).mean(1, keepdim=True))
    if "cuts" in s:
        row = torch.arange(x.shape[0], device=x.device)
        of = ((row >= s["offsets"][:-1, None]) & (row < s["offsets"][1:, None])).float()     # [samples][rows]
        dw, db = (of @ (dy * n)).abs().sum(0), (of @ dy).abs().sum(0)
    else:
        dw, db = (dy * n).sum(0), dy.sum(0)
    return {"dx": dx.to(s["x"].dtype), "dweight": dw, "dbias": db}


def _linear(s):
    x, dy = s["x"].float(), s["dy"].float()
    if "cuts" not in s:
        return {"weight": dy.abs().T @ x.abs(), "bias": dy.abs().sum(0)}
    w = torch.zeros(dy.shape[1], x.shape[1], device=x.device)
    b = torch.zeros(dy.shape[1], device=x.device)
    for lo, hi in zip(s["cuts"], s["cuts"][1:]):       # samples differ in length: a product for each
        w += (dy[lo:hi].T @ x[lo:hi]).abs()
        b += dy[lo:hi].sum(0).abs()
    return {"weight": w, "bias": b}


# --------------------------------------------------------------------------- the framework's calls

_kept = {}


def _ctx(he):
    """The context that a program makes once (ring of 2^13, three primes)."""
    if "ctx" not in _kept:
        _kept["ctx"] = he.he_ctx_create(8192, [0xfffffffffffc001, 0xfffffdc001, 0xffffffffffe8001], 40)
    return _kept["ctx"]


def _call(s):
    import paper_2303_10837_b200 as he
    ctx, op = _ctx(he), s["case"]["op"]
    if op == "log_probs":
        top = s["case"]["top"]
        logp, lse, entropy, top_logp, top_ids = he.he_token_log_probs(ctx, s["logits"], s["targets"], top=top)
        out = {"logp": logp, "lse": lse, "entropy": entropy}
        return {**out, "top_logp": top_logp, "top_ids": top_ids} if top else out
    if op == "log_probs_grad":
        return {"dlogits": he.he_token_log_probs_backward(ctx, s["logits"], s["targets"], s["lse"], s["dlogp"], entropy=s["entropy"], dentropy=s["dentropy"])}
    if op == "norm":
        y, mean, rstd = he.he_layer_norm(ctx, s["x"], s["weight"], s["bias"], eps=_EPS)
        return {"y": y, "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        dx, dw, db = he.he_layer_norm_backward(ctx, s["dy"], s["x"], s["mean"], s["rstd"], s["weight"], samples=s.get("offsets"))
        return {"dx": dx, "dweight": dw, "dbias": db}
    w, b = he.he_linear_sensitivity(ctx, s["x"], s["dy"], samples=s.get("offsets"))
    return {"weight": w, "bias": b}


def run(state):
    if own:
        return _call(state)
    return {"log_probs": _log_probs, "log_probs_grad": _log_probs_grad, "norm": _norm, "norm_grad": _norm_grad,
            "linear": _linear}[state["case"]["op"]](state)


# --------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    e, rows, op = 4 if case["dtype"] == "f32" else 2, case["rows"], case["op"]
    if op == "log_probs":                   # logits and targets in; three numbers and the alternatives out
        n, top = rows * case["vocab"], case["top"]
        return {"bytes": e * n + rows * (8.0 + 12.0 + 12.0 * top), "flops": 6.0 * n}
    if op == "log_probs_grad":              # logits and the row's numbers in, their gradient out
        n = rows * case["vocab"]
        return {"bytes": 2.0 * e * n + rows * (8.0 + 8.0 + (8.0 if case["entropy"] else 0.0)), "flops": (6.0 if case["entropy"] else 3.0) * n}
    if op == "norm":
        n = rows * case["width"]
        return {"bytes": 2.0 * e * n + 8.0 * case["width"] + 8.0 * rows, "flops": 8.0 * n}
    if op == "norm_grad":
        n = rows * case["width"]
        return {"bytes": 3.0 * e * n + 12.0 * case["width"] + 8.0 * rows, "flops": 14.0 * n}
    o, i = case["outputs"], case["inputs"]
    return {"bytes": e * rows * (o + i) + 4.0 * o * i + 4.0 * o, "flops": 2.0 * rows * o * i}


# --------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "log_probs":
        z, y = s["logits"].double(), s["targets"]
        lp = torch.log_softmax(z, 1)
        lse = torch.logsumexp(z, 1)
        out = {"logp": torch.where(y >= 0, lp.gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0), "lse": lse,
               "entropy": torch.special.entr(lp.exp()).sum(1)}
        if case["top"]:
            got = [torch.sort(r, descending=True, stable=True) for r in lp.split(256)]
            out["top_logp"] = torch.cat([v.values[:, :case["top"]] for v in got])
            out["top_ids"] = torch.cat([v.indices[:, :case["top"]] for v in got])
        return out
    if op == "log_probs_grad":
        z, y = s["logits"].double(), s["targets"]
        p = torch.exp(z - s["lse"].double()[:, None])
        hit = torch.zeros_like(p)
        rows = torch.nonzero(y >= 0)[:, 0]
        hit[rows, y[rows]] = 1.0
        grad = (s["dlogp"].double() * (y >= 0))[:, None] * (hit - p * (y >= 0)[:, None])
        if s["dentropy"] is not None:
            grad += s["dentropy"].double()[:, None] * (torch.special.entr(p) - p * s["entropy"].double()[:, None])
        return {"dlogits": grad}
    if op == "norm":
        x = s["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + _EPS) ** -0.5
        return {"y": torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], s["weight"].double()), "mean": mean, "rstd": rstd}
    if op == "norm_grad":
        x, dy = s["x"].double(), s["dy"].double()
        rstd = s["rstd"].double()[:, None]
        n = (x - s["mean"].double()[:, None]) * rstd
        a = dy * s["weight"].double()
        D = x.shape[1]
        dx = rstd / D * (D * a - a.sum(1, keepdim=True) - n * (a * n).sum(1, keepdim=True))
        cuts = s.get("cuts", None)
        if cuts is None:
            return {"dx": dx, "dweight": torch.einsum("rd,rd->d", dy, n), "dbias": dy.sum(0)}
        pieces = [h - l for l, h in zip(cuts, cuts[1:])]
        pieces.append(x.shape[0] - cuts[-1])
        both = [[v.sum(0).abs() for v in t.split(pieces)[:-1]] for t in (dy * n, dy)]
        return {"dx": dx, "dweight": torch.stack(both[0]).sum(0), "dbias": torch.stack(both[1]).sum(0)}
    x, dy = s["x"].double(), s["dy"].double()
    cuts = s.get("cuts", None)
    if cuts is None:
        return {"weight": torch.einsum("ro,ri->oi", dy.abs(), x.abs()), "bias": dy.abs().sum(0)}
    w = x.new_zeros(dy.shape[1], x.shape[1])
    b = x.new_zeros(dy.shape[1])
    for k in range(len(cuts) - 1):
        part = slice(cuts[k], cuts[k + 1])
        w.add_(torch.mm(dy[part].t(), x[part]).abs_())
        b.add_(dy[part].sum(0).abs_())
    return {"weight": w, "bias": b}
