"""The worker side's training operators as cases for a timing program.

A case names one pass through one entry point of :class:`paper_1709_09393_amd.binding.SlimDP`:

``norm``       layer norm of every worker's rows, with the row statistics that the backward pass reads
``norm_back``  its backward pass, with the sums over rows that are the gradients of weight and bias
``linear``     matrix product with bias, activation and residual in its epilogue
``act_back``   backward pass of that epilogue: gradient before the activation, gradient of the bias
``linear_back``  the two products that are the gradients of the input and of the weight
``distill``    distillation loss from a teacher's top logits with the gradient of the student's logits

``rows`` is written as text, one number a worker ("640,0,77"): the mini-batches of the workers need not be alike.
Vectors of parameters and all gradients of parameters are binary32 (pieces of the flat local model and of the flat
gradient); everything else has the case's type.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
KINDS = ("norm", "norm_back", "linear", "act_back", "linear_back", "distill")
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
EPS = 1e-5
MOST_FLOPS = 2 * 8 * 2048 * 4096 * 4096          # the largest listed product
MOST_ELEMENTS = 8 * 2048 * 4096                  # ... and the most elements of a listed norm
MOST_LOGITS = 4 * 1024 * 128_000


def _case(name, kind, dtype, rows, cols, **more):
    case = {"name": name, "kind": kind, "dtype": dtype, "rows": ",".join(str(r) for r in rows), "cols": int(cols)}
    case.update(more)
    return case


def listed():
    return [
        # one row of one worker, as when a single sample is looked at: latency alone
        _case("norm_one_row", "norm", "f32", [1], 1024),
        # eight workers' mini-batches of 2048 rows through a layer of ordinary width
        _case("norm_batch", "norm", "bf16", [2048] * 8, 4096),
        # workers with mini-batches of different sizes and a width that no vector divides
        _case("norm_back_ragged", "norm_back", "f16", [517, 1000, 3, 640], 1337),
        # the backward pass of norm_batch
        _case("norm_back_batch", "norm_back", "bf16", [2048] * 8, 4096),
        # one row through one layer: the weight's bytes are all there is
        _case("linear_one_row", "linear", "bf16", [1], 4096, out=4096, act="none", residual=False, keep=False),
        # eight workers, the layer of a block that ends in the residual stream, everything the backward pass needs kept
        _case("linear_batch", "linear", "bf16", [2048] * 8, 4096, out=4096, act="gelu", residual=True, keep=True),
        # gradient before the activation, ragged mini-batches
        _case("act_back_ragged", "act_back", "f32", [100, 317, 0, 29], 1001, act="silu"),
        # ... and eight workers' batches
        _case("act_back_batch", "act_back", "bf16", [2048] * 8, 4096, act="gelu"),
        # a classifier's last layer in binary32, small odd mini-batches: the weight's gradient is a product of few rows
        _case("linear_back_odd", "linear_back", "f32", [33, 65, 127], 1001, out=777),
        # the backward products of linear_batch
        _case("linear_back_batch", "linear_back", "bf16", [2048] * 8, 4096, out=4096),
        # few rows, a small odd vocabulary
        _case("distill_small", "distill", "f32", [16, 5], 10_007, top=20, temperature=2.0, padded=True),
        # four workers' 1024 tokens over a large vocabulary, 64 teacher entries each
        _case("distill_batch", "distill", "bf16", [1024] * 4, 128_000, top=64, temperature=1.5, padded=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _ragged(rng, total, workers):
    """Row counts of the workers that add up to about total, a worker without rows among them now and then."""
    if workers == 1 or rng.random() < 0.4:
        return [max(1, total // workers)] * workers
    part = [rng.random() + 0.05 for _ in range(workers)]
    rows = [max(1, int(total * p / sum(part))) for p in part]
    if rng.random() < 0.3:
        rows[rng.randrange(workers)] = 0
    return rows if sum(rows) else [1] * workers


def _width(rng, lo, hi):
    n = _log_int(rng, lo, hi)
    step = rng.choice((1, 1, 8, 64))                # odd, whole vectors, whole tiles
    return max(lo, n // step * step)


def draw(rng):
    kind = rng.choice(KINDS)
    dtype = rng.choice(("f32", "f16", "bf16", "bf16"))
    workers = rng.choice((1, 2, 3, 4, 8))
    if kind in ("norm", "norm_back", "act_back"):
        cols = _width(rng, 16, 16_384)
        rows = _ragged(rng, _log_int(rng, 1, max(1, min(65_536, MOST_ELEMENTS // 2 // cols))), workers)
        more = {"act": rng.choice(ACTS[1:])} if kind == "act_back" else {}
    elif kind in ("linear", "linear_back"):
        cols, out = _width(rng, 16, 8192), _width(rng, 16, 8192)
        most = MOST_FLOPS // (16 if dtype == "f32" else 2) // (4 if kind == "linear_back" else 2) // (cols * out)
        rows = _ragged(rng, _log_int(rng, 1, max(1, min(16_384, most))), workers)
        more = {"out": out}
        if kind == "linear":
            more.update(act=rng.choice(ACTS), residual=rng.random() < 0.5, keep=rng.random() < 0.5)
    else:
        cols = _width(rng, 500, 200_000)
        rows = _ragged(rng, _log_int(rng, 1, max(1, min(8192, MOST_LOGITS // 2 // cols))), workers)
        more = {"top": _log_int(rng, 1, 256), "temperature": rng.choice((1.0, 1.5, 2.0, 4.0)), "padded": rng.random() < 0.5}
    case = _case("", kind, dtype, rows, cols, **more)
    del case["name"]
    return case


# ---------------------------------------------------------------------------------------------------------------
def _rows(case):
    return [int(r) for r in case["rows"].split(",")]


class _Draws:
    """Tensors on the current GPU, drawn one after the other from a seed."""

    def __init__(self, seed):
        self.seed, self.count = int(seed), 0
        self.dev = torch.device("cuda", torch.cuda.current_device())

    def _gen(self):
        self.count += 1
        gen = torch.Generator(device=self.dev)
        gen.manual_seed(1_000_003 * self.seed + self.count)
        return gen

    def normal(self, shape, dtype, sigma=1.0, mean=0.0):
        return torch.empty(shape, dtype=torch.float32, device=self.dev).normal_(mean, sigma, generator=self._gen()).to(dtype)

    def uniform(self, shape):
        return torch.empty(shape, dtype=torch.float32, device=self.dev).uniform_(0.0, 1.0, generator=self._gen())


def _inputs(case, seed):
    """Per worker a dict of what the call reads."""
    d, t, f32, cols = _Draws(seed), TYPES[case["dtype"]], torch.float32, case["cols"]
    kind, out = case["kind"], []
    for rows in _rows(case):
        i = {}
        if kind in ("norm", "norm_back"):
            i["x"] = d.normal((rows, cols), t, 1.5, 0.3)
            i["weight"] = d.normal((cols,), f32, 0.2, 1.0)
            if kind == "norm":
                i["bias"] = d.normal((cols,), f32, 0.2)
            else:
                i["dy"] = d.normal((rows, cols), t, 0.1)
                x = i["x"].double()              # what the forward pass left
                mean = x.mean(1)
                i["mean"] = mean.float()
                i["rstd"] = ((x - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
        elif kind == "linear":
            i["x"] = d.normal((rows, cols), t)
            i["weight"] = d.normal((case["out"], cols), t, cols ** -0.5)
            i["bias"] = d.normal((case["out"],), f32, 0.1)
            if case["residual"]:
                i["residual"] = d.normal((rows, case["out"]), t)
        elif kind == "act_back":
            i["dy"] = d.normal((rows, cols), t, 0.1)
            i["z"] = d.normal((rows, cols), t)
        elif kind == "linear_back":
            i["dz"] = d.normal((rows, case["out"]), t, 0.1)
            i["x"] = d.normal((rows, cols), t)
            i["weight"] = d.normal((case["out"], cols), t, cols ** -0.5)
        else:
            i["logits"] = d.normal((rows, cols), t, 2.0)
            top = min(case["top"], cols)
            # distinct indices in no order: a random start and a step that shares no factor with the vocabulary
            step = next(s for s in (10_007, 7919, 104_729) if math.gcd(s, cols) == 1)
            start = (d.uniform((rows, 1)) * cols).long().clamp_(max=cols - 1)
            i["index"] = ((start + step * torch.arange(top, device=d.dev)) % cols).to(torch.int32)
            i["value"] = d.normal((rows, top), f32, 2.0, 6.0)
            i["row_weight"] = 0.5 + d.uniform((rows,))
            if case["padded"]:
                # shorter lists behind which nothing counts, and tokens that are padding themselves
                keep = (d.uniform((rows, 1)) * (top + 1)).long()
                i["index"] = torch.where(torch.arange(top, device=d.dev) < keep, i["index"], torch.full_like(i["index"], -1))
                i["row_weight"] = torch.where(d.uniform((rows,)) < 0.9, i["row_weight"], torch.zeros_like(i["row_weight"]))
        out.append(i)
    return out


class _State:
    pass


def prepare(case, seed):
    s = _State()
    s.case, s.inputs = case, _inputs(case, seed)
    s.table = {k: [i[k] for i in s.inputs] for k in s.inputs[0]}
    s.sd = None
    if own:
        from paper_1709_09393_amd import binding
        s.sd = binding.SlimDP(4096, len(s.inputs), seed=seed)
        # arrays that a training program allocates once: activations, and gradients as pieces of a flat vector
        t, f32 = TYPES[case["dtype"]], torch.float32
        like = lambda name: [torch.empty_like(x) for x in s.table[name]]
        per_row = lambda: [torch.empty(r, dtype=f32, device="cuda") for r in _rows(case)]
        vec = lambda n: [torch.empty(n, dtype=f32, device="cuda") for _ in s.inputs]
        mat = lambda n: [torch.empty((r, n), dtype=t, device="cuda") for r in _rows(case)]
        kind = case["kind"]
        if kind == "norm":
            s.out = {"y": like("x"), "mean": per_row(), "rstd": per_row()}
        elif kind == "norm_back":
            s.out = {"dx": like("x"), "dweight": vec(case["cols"]), "dbias": vec(case["cols"])}
        elif kind == "linear":
            s.out = {"y": mat(case["out"])}
            if case["keep"]:
                s.out["z"] = mat(case["out"])
        elif kind == "act_back":
            s.out = {"dz": like("dy"), "dbias": vec(case["cols"])}
        elif kind == "linear_back":
            s.out = {"dx": like("x"), "dweight": [v.view(case["out"], case["cols"]) for v in vec(case["out"] * case["cols"])]}
        else:
            s.out = {"loss": per_row(), "lse": per_row(), "dlogits": like("logits")}
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * 0.7071067811865476))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(0.7978845608028654 * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * 0.7071067811865476)) + z * torch.exp(-0.5 * z * z) * 0.3989422804014327
    if act == "gelu_tanh":
        t = torch.tanh(0.7978845608028654 * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * 0.7978845608028654 * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        sig = 1.0 / (1.0 + torch.exp(-z))
        return sig * (1.0 + z * (1.0 - sig))
    return torch.ones_like(z)


def _plain_norm(i, case):
    x = i["x"].float()
    mean = x.sum(1) / case["cols"]
    c = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((c * c).sum(1) / case["cols"] + EPS)
    return {"y": (c * rstd[:, None] * i["weight"] + i["bias"]).to(i["x"].dtype), "mean": mean, "rstd": rstd}


def _plain_norm_back(i, case):
    dy, n = i["dy"].float(), case["cols"]
    xh = (i["x"].float() - i["mean"][:, None]) * i["rstd"][:, None]
    a = dy * i["weight"]
    dx = i["rstd"][:, None] * (a - a.sum(1, keepdim=True) / n - xh * ((a * xh).sum(1, keepdim=True) / n))
    return {"dx": dx.to(i["x"].dtype), "dweight": (dy * xh).sum(0), "dbias": dy.sum(0)}


def _plain_linear(i, case):
    z = i["x"].float() @ i["weight"].float().t() + i["bias"]
    y = _act(z, case["act"])
    if case["residual"]:
        y = y + i["residual"].float()
    out = {"y": y.to(i["x"].dtype)}
    if case["keep"]:
        out["z"] = z.to(i["x"].dtype)
    return out


def _plain_act_back(i, case):
    dz = i["dy"].float() * _act_slope(i["z"].float(), case["act"])
    return {"dz": dz.to(i["dy"].dtype), "dbias": dz.sum(0)}


def _plain_linear_back(i, case):
    dz = i["dz"].float()
    return {"dx": (dz @ i["weight"].float()).to(i["x"].dtype), "dweight": dz.t().contiguous() @ i["x"].float()}


def _plain_distill(i, case):
    tau = case["temperature"]
    s = i["logits"].float() / tau
    top = s.max(1, keepdim=True).values
    e = torch.exp(s - top)
    total = e.sum(1, keepdim=True)
    lse = top + torch.log(total)
    valid = i["index"] >= 0
    at = torch.where(valid, i["index"], torch.zeros_like(i["index"])).long()
    v = torch.where(valid, i["value"] / tau, torch.full_like(i["value"], -math.inf))
    some = valid.any(1, keepdim=True)
    v = v - torch.where(some, v.max(1, keepdim=True).values, torch.zeros_like(lse))
    p = torch.exp(v)
    mass = p.sum(1, keepdim=True)
    p = torch.where(some, p / mass, torch.zeros_like(p))
    logp = torch.where(p > 0, v - torch.log(mass), torch.zeros_like(p))
    logq = torch.gather(s, 1, at) - lse
    w = i["row_weight"]
    loss = w * tau * tau * (p * (logp - logq)).sum(1)
    q = e / total * some.float()
    ds = (w * tau)[:, None] * q.scatter_add(1, at, -p)
    return {"loss": loss, "lse": lse[:, 0], "dlogits": ds.to(i["logits"].dtype)}


def run(state):
    case, kind = state.case, state.case["kind"]
    if not own:
        parts = [globals()["_plain_" + kind](i, case) for i in state.inputs]
        return {k: [p[k] for p in parts] for k in parts[0]}
    sd, t, out = state.sd, state.table, state.out
    if kind == "norm":
        sd.layer_norm(t["x"], t["weight"], t["bias"], EPS, **out)
    elif kind == "norm_back":
        sd.layer_norm_backward(t["dy"], t["x"], t["weight"], t["mean"], t["rstd"], **out)
    elif kind == "linear":
        sd.linear(t["x"], t["weight"], t["bias"], activation=case["act"], residual=t.get("residual"), **out)
    elif kind == "act_back":
        sd.linear_epilogue_backward(t["dy"], t["z"], activation=case["act"], **out)
    elif kind == "linear_back":
        sd.linear_backward(t["dz"], t["x"], t["weight"], **out)
    else:
        sd.distill_loss(t["logits"], t["index"], t["value"], case["temperature"], row_weight=t["row_weight"], **out)
    return out


# ---------------------------------------------------------------------------------------------------------------
def work(case):
    rows, cols, workers = sum(_rows(case)), case["cols"], len(_rows(case))
    e = 4 if case["dtype"] == "f32" else 2
    kind, n = case["kind"], case.get("out", 0)
    if kind == "norm":
        return {"bytes": 2 * e * rows * cols + 8 * workers * cols + 8 * rows, "flops": 8 * rows * cols}
    if kind == "norm_back":
        return {"bytes": 3 * e * rows * cols + 12 * workers * cols + 8 * rows, "flops": 14 * rows * cols}
    if kind == "act_back":
        return {"bytes": 3 * e * rows * cols + 4 * workers * cols, "flops": 20 * rows * cols}
    if kind == "linear":
        outs = 1 + bool(case["residual"]) + bool(case["keep"])
        return {"bytes": e * (rows * cols + workers * n * cols + outs * rows * n) + 4 * workers * n, "flops": 2 * rows * cols * n}
    if kind == "linear_back":
        return {"bytes": e * (rows * n + 2 * rows * cols + workers * n * cols) + 4 * workers * n * cols, "flops": 4 * rows * cols * n}
    top = min(case["top"], cols)
    return {"bytes": 2 * e * rows * cols + 8 * rows * top + 12 * rows, "flops": 8 * rows * cols}


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
def _exact_activation(z, act):
    """Value and slope."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0.0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * torch.sigmoid(-z)
    if act == "gelu":
        phi = 0.5 * torch.erfc(-z / math.sqrt(2.0))
        return z * phi, phi + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    # gelu_tanh: 0.5 (1 + tanh u) is sigmoid(2 u)
    k = math.sqrt(2.0 / math.pi)
    s = torch.sigmoid(2.0 * k * (z + 0.044715 * z ** 3))
    return z * s, s + z * s * (1.0 - s) * 2.0 * k * (1.0 + 0.134145 * z ** 2)


def _exact_one(i, case):
    kind = case["kind"]
    v = {k: (x.double() if x.is_floating_point() else x) for k, x in i.items()}
    if kind == "norm":
        mean = v["x"].mean(1)
        rstd = (v["x"].var(1, unbiased=False) + EPS).pow(-0.5)
        return {"y": torch.addcmul(v["bias"], (v["x"] - mean[:, None]) * rstd[:, None], v["weight"]), "mean": mean, "rstd": rstd}
    if kind == "norm_back":
        xh = (v["x"] - v["mean"][:, None]) * v["rstd"][:, None]
        a = v["dy"] * v["weight"]
        inner = a - a.mean(1, keepdim=True) - xh * (a * xh).mean(1, keepdim=True)
        return {"dx": inner * v["rstd"][:, None], "dweight": torch.sum(v["dy"] * xh, 0), "dbias": torch.sum(v["dy"], 0)}
    if kind == "linear":
        z = torch.mm(v["x"], v["weight"].t().contiguous()) + v["bias"]
        y = _exact_activation(z, case["act"])[0]
        if case["residual"]:
            y += v["residual"]
        return {"y": y, "z": z} if case["keep"] else {"y": y}
    if kind == "act_back":
        dz = v["dy"] * _exact_activation(v["z"], case["act"])[1]
        return {"dz": dz, "dbias": dz.sum(0)}
    if kind == "linear_back":
        return {"dx": torch.mm(v["dz"], v["weight"]), "dweight": torch.mm(v["dz"].t().contiguous(), v["x"])}
    tau, rows = case["temperature"], i["logits"].shape[0]
    loss, lse, grad = [], [], []
    step = max(1, 40_000_000 // case["cols"])
    for a in range(0, rows, step):
        part = slice(a, min(rows, a + step))
        scaled, index = v["logits"][part] / tau, v["index"][part]
        norm = torch.logsumexp(scaled, 1)
        logq = scaled - norm[:, None]
        dense = torch.zeros_like(logq)                       # the teacher's distribution over the whole vocabulary
        keep = index >= 0
        weight = (v["value"][part] / tau).masked_fill(~keep, -math.inf)
        p = torch.softmax(weight, 1).masked_fill(~keep, 0.0)  # a list of nothing gives no NaN
        dense.scatter_add_(1, index.clamp(min=0).long(), p)
        has = keep.any(1).double()
        w = v["row_weight"][part]
        loss.append(w * tau ** 2 * (torch.special.xlogy(dense, dense) - dense * logq).sum(1))
        lse.append(norm)
        grad.append((w * tau)[:, None] * (logq.exp() * has[:, None] - dense))
    join = lambda parts, like: torch.cat(parts) if parts else like
    return {"loss": join(loss, v["row_weight"]), "lse": join(lse, v["row_weight"]), "dlogits": join(grad, v["logits"])}


def exact(case, seed):
    parts = [_exact_one(i, case) for i in _inputs(case, seed)]
    return {k: [p[k] for p in parts] for k in parts[0]}
