"""Cases for the two training operators beside the compressed weight gradient: the classifier's loss with its
gradients (a linear layer over many classes and softmax cross entropy, the logits never kept), and the update of a
weight matrix from its gradient (momentum and orthogonalisation by Newton-Schulz products).

`run` computes a case in plain 32-bit torch operations, or, with `own` true, through this package's entry points.
`exact` computes the same in 64 bits."""
import math

import torch

own = False

#: The quintic polynomial of one Newton-Schulz step: X <- a X + b (X X^T) X + c (X X^T)^2 X.
A, B, C = 3.4445, -4.7750, 2.0315
EPS = 1e-7
IGNORED = -100


def _loss(name, call, tokens, classes, features, bias=False, ignored=0.0, scratch="ample"):
    return {"name": name, "op": "linear_ce", "call": call, "tokens": tokens, "classes": classes, "features": features,
            "bias": bias, "ignored": ignored, "scratch": scratch}


def _update(name, batch, rows, cols, dtype="f32", nesterov=True, steps=5):
    return {"name": name, "op": "muon", "batch": batch, "rows": rows, "cols": cols, "dtype": dtype,
            "nesterov": nesterov, "steps": steps}


def listed():
    return [
        # the classifier of a small residual network at the paper's accounting batch of 32: launch latency
        _loss("head_32x1000x512", "step", 32, 1000, 512, bias=True),
        # ResNet-50's classifier at batch 256, one training step
        _loss("head_256x1000x2048", "step", 256, 1000, 2048, bias=True),
        # evaluation of a language model's head: the loss alone
        _loss("eval_2048x32000x2048", "forward", 2048, 32000, 2048),
        # no size a multiple of eight, a tenth of the tokens padding
        _loss("odd_1537x50021x1021", "step", 1537, 50021, 1021, ignored=0.1),
        # the backward pass alone, from a stored log-sum-exp, in the least scratch memory
        _loss("backward_4096x65536x2048", "backward", 4096, 65536, 2048, ignored=0.05, scratch="least"),
        # a long batch over a large vocabulary, loss and gradients in one call
        _loss("step_8192x131072x4096", "step", 8192, 131072, 4096),
        # one 3x3 convolution of the first stage, as a matrix of 64 x (64 * 9): latency
        _update("update_64x576", 1, 64, 576),
        # the six 3x3 convolutions of ResNet-50's third stage
        _update("update_6x256x2304", 6, 256, 2304),
        # the six expanding 1x1 convolutions of the same stage: more rows than columns
        _update("update_6x1024x256", 6, 1024, 256, nesterov=False),
        # odd sizes, gradients in 16 bits
        _update("update_771x1543_bf16", 1, 771, 1543, "bf16"),
        # a square projection of a wide model, gradients in 16 bits
        _update("update_4096x4096_bf16", 1, 4096, 4096, "bf16"),
        # a wide feed-forward matrix
        _update("update_4096x16384", 1, 4096, 16384),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    if rng.random() < 0.5:
        features = _spread(rng, 128, 4096)
        if rng.random() < 0.7:      # most models' widths are multiples of 8; some are not
            features = max(8, features // 8 * 8)
        case = _loss("", rng.choice(("step", "step", "forward", "backward")), _spread(rng, 1, 8192),
                     _spread(rng, 500, 131072), features, rng.random() < 0.4, rng.choice((0.0, 0.1, 0.5)),
                     rng.choice(("ample", "least")))
    else:
        rows, cols = _spread(rng, 16, 4096), _spread(rng, 16, 16384)
        most = 4096 * 4096 * 16384 // (rows * cols * min(rows, cols))
        case = _update("", max(1, min(rng.randint(1, 8), most)), rows, cols, rng.choice(("f32", "bf16")),
                       rng.random() < 0.7, rng.choice((4, 5, 5, 6)))
    del case["name"]
    return case


def _prepare_loss(case, g):
    t, v, d = case["tokens"], case["classes"], case["features"]
    labels = torch.randint(0, v, (t,), generator=g, device="cuda")
    # rows of unit-variance features, weights that give logits of standard deviation 1.5, and a model that has
    # learnt something: each row leans towards its label's weights
    w = torch.randn((v, d), generator=g, device="cuda", dtype=torch.bfloat16).mul_(1.5 / math.sqrt(d))
    h = torch.randn((t, d), generator=g, device="cuda") + 1.5 * w[labels].float()
    bias = torch.randn((v,), generator=g, device="cuda").mul_(0.1).bfloat16() if case["bias"] else None
    if case["ignored"]:
        labels[torch.rand((t,), generator=g, device="cuda") < case["ignored"]] = IGNORED
    kept = (labels != IGNORED).sum().clamp_(min=1)
    dloss = torch.where(labels != IGNORED, 1.0 / kept, 0.0).float()      # the mean over the tokens that count
    s = {"case": case, "h": h.bfloat16(), "w": w, "bias": bias, "labels": labels, "dloss": dloss, "lse": None}
    if case["call"] == "backward":
        s["lse"] = torch.cat([torch.logsumexp(_logits(x, s), 1) for x in s["h"].split(2048)])
    return s


def _prepare_update(case, g):
    b, m, n = case["batch"], case["rows"], case["cols"]

    def gradient(scale):
        # a few directions carry most of a gradient: singular values that fall off, over noise
        r = max(1, min(m, n) // 4)
        fall = torch.arange(1, r + 1, device="cuda").rsqrt()
        x = torch.randn((b, m, r), generator=g, device="cuda") * fall @ torch.randn((b, r, n), generator=g, device="cuda")
        return scale * (x / math.sqrt(r) + 0.3 * torch.randn((b, m, n), generator=g, device="cuda"))

    grad = gradient(1e-2)
    return {"case": case, "grad": grad.bfloat16() if case["dtype"] == "bf16" else grad, "momentum": gradient(5e-2),
            "beta": 0.95, "scale": math.sqrt(max(1.0, m / n))}


def prepare(case, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    return (_prepare_loss if case["op"] == "linear_ce" else _prepare_update)(case, g)


# -- the plain forms ----------------------------------------------------------


def _logits(h, s):
    x = h.float() @ s["w"].float().T
    return x if s["bias"] is None else x.add_(s["bias"].float())


def _plain_loss(s):
    call, labels, w = s["case"]["call"], s["labels"], s["w"]
    kept = labels != IGNORED
    at = labels.clamp(min=0)[:, None]
    x = _logits(s["h"], s)
    lse, out = s["lse"], {}
    if call != "backward":
        top = x.amax(1)
        lse = top + (x - top[:, None]).exp_().sum(1).log_()
        out["loss"] = torch.where(kept, lse - x.gather(1, at)[:, 0], 0.0)
        out["lse"] = lse
    if call != "forward":
        p = x.sub_(lse[:, None]).exp_()
        p.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
        p.mul_(torch.where(kept, s["dloss"], 0.0)[:, None])
        out["dh"] = (p @ w.float()).to(torch.bfloat16)
        out["dw"] = (p.T @ s["h"].float()).to(torch.bfloat16)
        if s["bias"] is not None:
            out["dbias"] = p.sum(0).to(torch.bfloat16)
    return out


def _plain_update(s):
    case, grad = s["case"], s["grad"].float()
    momentum = s["beta"] * s["momentum"] + grad
    x = grad + s["beta"] * momentum if case["nesterov"] else momentum
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    tall = case["rows"] > case["cols"]
    x = x.mT if tall else x
    for _ in range(case["steps"]):
        g = x @ x.mT
        x = A * x + (B * g + C * (g @ g)) @ x
    x = x.mT if tall else x
    return {"momentum": momentum, "update": (s["scale"] * x).to(torch.bfloat16).contiguous()}


# -- this package's entry points ----------------------------------------------


def _own_loss(s):
    import paper_2409_11902_b200 as ac
    case = s["case"]
    if "desc" not in s:     # what a training loop keeps from step to step: the descriptor, scratch, gradient buffers
        d = ac.LinearCeDesc(case["tokens"], case["classes"], case["features"], bias=case["bias"])
        size = ac.ac_linear_ce_workspace_bytes if case["scratch"] == "ample" else ac.ac_linear_ce_workspace_bytes_min
        s["desc"], s["workspace"] = d, torch.empty(size(d), dtype=torch.uint8, device="cuda")
        rows = lambda: torch.empty(case["tokens"], device="cuda")  # noqa: E731
        s["out"] = {} if case["call"] == "backward" else {"loss": rows(), "lse": rows()}
        if case["call"] != "forward":
            s["out"].update(dh=torch.empty_like(s["h"]), dw=torch.empty_like(s["w"]))
            if case["bias"]:
                s["out"]["dbias"] = torch.empty_like(s["bias"])
    d, o = s["desc"], s["out"]
    if case["call"] == "forward":
        ac.ac_linear_ce_forward(d, s["h"], s["w"], s["bias"], s["labels"], o["loss"], o["lse"], s["workspace"])
    elif case["call"] == "backward":
        ac.ac_linear_ce_backward(d, s["h"], s["w"], s["bias"], s["labels"], s["lse"], s["dloss"], o["dh"], o["dw"],
                                 o.get("dbias"), s["workspace"])
    else:
        ac.ac_linear_ce_step(d, s["h"], s["w"], s["bias"], s["labels"], s["dloss"], o["loss"], o["lse"], o["dh"],
                             o["dw"], o.get("dbias"), s["workspace"])
    return o


def _own_update(s):
    import paper_2409_11902_b200 as ac
    case = s["case"]
    if "desc" not in s:
        d = ac.MuonDesc(case["rows"], case["cols"], batch=case["batch"], dtype=case["dtype"], steps=case["steps"],
                        momentum=s["beta"], nesterov=case["nesterov"], scale=s["scale"], eps=EPS, coefficients=(A, B, C))
        s["desc"], s["workspace"] = d, torch.empty(ac.ac_muon_workspace_bytes(d), dtype=torch.uint8, device="cuda")
        s["out"] = {"momentum": torch.empty_like(s["momentum"]),
                    "update": torch.empty_like(s["momentum"], dtype=torch.bfloat16)}
    o = s["out"]
    ac.ac_muon_update(s["desc"], s["grad"], s["momentum"], o["momentum"], o["update"], s["workspace"])
    return o


def run(state):
    if state["case"]["op"] == "linear_ce":
        return (_own_loss if own else _plain_loss)(state)
    return (_own_update if own else _plain_update)(state)


# -- what a pass cannot do without --------------------------------------------


def work(case):
    if case["op"] == "linear_ce":
        t, v, d = case["tokens"], case["classes"], case["features"]
        read = 2 * (t * d + v * d + (v if case["bias"] else 0)) + 8 * t
        if case["call"] == "forward":
            return {"bytes": read + 8 * t, "flops": 2 * t * v * d}
        # logits, the gradient of the features and the gradient of the weights: a product each
        wrote = 2 * (t * d + v * d + (v if case["bias"] else 0))
        return {"bytes": read + wrote + (8 if case["call"] == "backward" else 12) * t, "flops": 6 * t * v * d}
    b, m, n = case["batch"], case["rows"], case["cols"]
    k, l = min(m, n), max(m, n)
    # the Gram matrix and its square are symmetric: half of each product
    return {"bytes": b * m * n * ((2 if case["dtype"] == "bf16" else 4) + 4 + 4 + 2),
            "flops": b * case["steps"] * (k * k * l + k * k * k + 2 * k * k * l)}


# -- the definitions in 64 bits -----------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "linear_ce":
        return _exact_loss(s)
    g = s["grad"].double()
    v = g + s["beta"] * s["momentum"].double()
    u = torch.add(g, v, alpha=s["beta"]) if case["nesterov"] else v
    u = u / (torch.linalg.matrix_norm(u)[:, None, None] + EPS)
    wide = case["rows"] <= case["cols"]
    eye = torch.eye(min(case["rows"], case["cols"]), device="cuda", dtype=torch.float64)
    for _ in range(case["steps"]):
        q = torch.matmul(u, u.mT) if wide else torch.matmul(u.mT, u)
        q = A * eye + torch.matmul(B * eye + C * q, q)
        u = torch.matmul(q, u) if wide else torch.matmul(u, q)
    return {"momentum": v, "update": s["scale"] * u}


def _exact_loss(s):
    case, w = s["case"], s["w"].double()
    out = {k: [] for k in ("loss", "lse", "dh")}
    dw, dbias = torch.zeros_like(w), torch.zeros(case["classes"], device="cuda", dtype=torch.float64)
    for i in range(0, case["tokens"], 1024):
        h, labels = s["h"][i:i + 1024].double(), s["labels"][i:i + 1024]
        live = labels >= 0
        x = torch.nn.functional.linear(h, w, None if s["bias"] is None else s["bias"].double())
        lse = torch.logsumexp(x, 1)
        rows = torch.arange(len(h), device="cuda")[live]
        loss = torch.zeros_like(lse)
        loss[live] = lse[live] - x[rows, labels[live]]
        out["loss"].append(loss)
        out["lse"].append(lse)
        if case["call"] != "forward":
            stored = lse if s["lse"] is None else s["lse"][i:i + 1024].double()
            p = torch.exp(x - stored[:, None])
            p[rows, labels[live]] -= 1
            p *= (s["dloss"][i:i + 1024].double() * live)[:, None]
            out["dh"].append(p @ w)
            dw.addmm_(p.T, h)
            dbias += p.sum(0)
    out = {k: torch.cat(v) for k, v in out.items() if v}
    if case["call"] != "forward":
        out["dw"] = dw
        if case["bias"]:
            out["dbias"] = dbias
    if case["call"] == "backward":
        del out["loss"], out["lse"]
    return out
