"""Performance cases of the operators around the layer-parallel solver: the opening and closing layers of a residual network
(matrix product with bias, activation and residual, and its backward pass), the cross-entropy loss with its gradient, and
the clipping of all gradients to a global norm.

A case is a dict; its `op` says which operator, the rest its sizes and types:
  forward   z = X W^T + b, Y = R + scale act(z), D = scale act'(z):   M, K, F, x, w, y (types of X; W; R, Y and D), act, bias,
            residual, factor (whether D is kept for a backward pass)
  backward  G = dY D, dX = G W, dW = G^T X, db = sum of G over rows:  M, K, F, x, w, y (types of X and dX; W; dY and D), act
            (identity: no D), need_dx
  loss      per-row cross-entropy, its mean over the counted rows and the gradient by the logits:  B, V, dtype, masked (share of
            the classes at minus infinity), ignored (share of rows that do not count), need_grad
  clip      global norm of many tensors, all of them scaled to at most `max_norm`:  either N, q (the gradients of a stack
            of N dense layers of width q and of its opening and closing layers) or count, least, most, bf16 (that many tensors of
            sizes in between, one behind the other in memory, a share of them bf16), and max_norm
Where `own` is false the operators run in plain torch operations, where it is true through the library.
"""
import math
import random

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SCALE = 0.5                         # of the activation's branch, where there is an activation


def _forward(name, M, K, F, types, act, **kw):
    return dict(dict(name=name, op="forward", M=M, K=K, F=F, x=types[0], w=types[1], y=types[2], act=act, bias=True,
                     residual=False, factor=False), **kw)


def _backward(name, M, K, F, types, act, **kw):
    return dict(dict(name=name, op="backward", M=M, K=K, F=F, x=types[0], w=types[1], y=types[2], act=act, need_dx=True), **kw)


F32, BF16, STATES = ("f32",) * 3, ("bf16",) * 3, ("f32", "bf16", "f32")


def listed():
    return [
        # logits of the wide training stack's head (1024 features, 10 classes, batch 256), float: the smallest call
        _forward("close10_f32_forward", 256, 1024, 10, F32, "identity"),
        # the head of the large image stack (64 channels, 32 x 32, batch 32) backwards: bf16 weights between float states
        _backward("close10_states_backward", 32, 65536, 10, STATES, "identity"),
        # a fully connected layer of flattened images (d = 4096, batch 32) with skip connection, its factors kept: as many
        # rows as a serving batch, so the weights are most of the bytes
        _forward("connected4096_states_forward", 32, 4096, 4096, STATES, "tanh", residual=True, factor=True),
        # one sample's logits over many classes, as answered one at a time
        _forward("single_bf16_forward", 1, 4096, 32768, BF16, "identity", bias=False),
        # an opening layer whose sizes fit no tile, float, backwards with the gradient of its input
        _backward("ragged_f32_backward", 1000, 1031, 517, F32, "tanh"),
        # a wide float layer on many samples
        _forward("wide_f32_forward", 4096, 1024, 4096, F32, "relu", residual=True),
        # the largest: a wide bf16 layer on many samples, with skip connection, both directions
        _forward("wide_bf16_forward", 8192, 4096, 4096, BF16, "tanh", residual=True, factor=True),
        _backward("wide_bf16_backward", 8192, 4096, 4096, BF16, "tanh"),
        # the loss of the wide training stack's head: ten classes
        dict(name="loss10_f32", op="loss", B=256, V=10, dtype="f32", masked=0.0, ignored=0.0, need_grad=True),
        # the loss over many classes, an odd number of them, some masked, padded rows among the samples
        dict(name="loss50021_bf16", op="loss", B=4096, V=50021, dtype="bf16", masked=0.05, ignored=0.1, need_grad=True),
        # several hundred tensors of all sizes, float and bf16, in one allocation
        dict(name="clip_many", op="clip", count=600, least=8, most=500000, bf16=0.3, max_norm=1.0),
        # the gradients of the wide training stack: 1024 layers of width 1024, 4 GB
        dict(name="clip_stack1024", op="clip", N=1024, q=1024, max_norm=1.0),
    ]


# --------------------------------------------------------------------------------------------- drawn cases
def draw(rng: random.Random):
    def logint(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    def size(lo, hi):               # a whole multiple of 64 half the time, else whatever comes
        n = logint(lo, hi)
        return n if n < 128 or rng.random() < 0.5 else n // 64 * 64

    while True:
        op = rng.choice(["forward", "forward", "backward", "backward", "loss", "clip"])
        if op in ("forward", "backward"):
            c = dict(op=op, M=size(1, 8192), K=size(8, 65536), F=size(2, 65536), act=rng.choice(["identity", "tanh", "relu"]))
            c["x"], c["w"], c["y"] = rng.choice([F32, F32, BF16, BF16, STATES, STATES, ("bf16", "bf16", "f32"), ("f32", "f32", "bf16")])
            if op == "forward":
                c.update(bias=rng.random() < 0.8, residual=rng.random() < 0.5, factor=c["act"] == "tanh" and rng.random() < 0.5)
            else:
                c.update(need_dx=rng.random() < 0.8)
            if c["M"] * c["K"] * c["F"] > 8192 * 4096 * 4096 or max(c["M"] * c["K"], c["K"] * c["F"], c["M"] * c["F"]) > 1 << 28:
                continue
            return c
        if op == "loss":
            c = dict(op=op, B=logint(1, 16384), V=logint(2, 131072), dtype=rng.choice(["f32", "bf16"]), masked=rng.choice([0.0, 0.05, 0.5]),
                     ignored=rng.choice([0.0, 0.1, 0.6]), need_grad=rng.random() < 0.8)
            if c["B"] * c["V"] <= 4096 * 50021:
                return c
            continue
        if rng.random() < 0.4:
            c = dict(op=op, N=logint(1, 1024), q=logint(1, 128) * 8, max_norm=rng.choice([1.0, 1.0, 1.0e6]))
        else:
            c = dict(op=op, count=logint(1, 1500), least=1, most=logint(100, 2000000), bf16=rng.choice([0.0, 0.3, 1.0]),
                     max_norm=rng.choice([1.0, 1.0, 1.0e6]))
        return c


# --------------------------------------------------------------------------------------------- counts
def _bytes(t):
    return 4 if t == "f32" else 2


def _clip_shapes(c, seed):
    """Shapes of the tensors in order, and which of them are bf16."""
    if "N" in c:
        N, q = c["N"], c["q"]
        shapes = [(N, q, q), (N, q), (q, 784), (q,), (10, q), (10,)]
        return shapes, [False] * len(shapes)
    r = random.Random(c["count"] * 1000003 + c["most"])           # the sizes belong to the case, the values to the seed
    sizes = [round(math.exp(r.uniform(math.log(c["least"]), math.log(c["most"])))) for _ in range(c["count"])]
    return [(n,) for n in sizes], [r.random() < c["bf16"] for _ in sizes]


def work(case):
    c = case
    if c["op"] in ("forward", "backward"):
        M, K, F = c["M"], c["K"], c["F"]
        xb, wb, yb = _bytes(c["x"]), _bytes(c["w"]), _bytes(c["y"])
        b = xb * M * K + wb * F * K + yb * M * F                  # X, W, Y or dY
        if c["op"] == "forward":
            b += 4 * F * c["bias"] + yb * M * F * (c["residual"] + c["factor"])
            return {"bytes": float(b), "flops": 2.0 * M * K * F}
        b += yb * M * F * (c["act"] != "identity") + 4 * F * K + 4 * F + xb * M * K * c["need_dx"]
        return {"bytes": float(b), "flops": 2.0 * M * K * F * (1 + c["need_dx"])}
    if c["op"] == "loss":
        n = c["B"] * c["V"]
        return {"bytes": float(_bytes(c["dtype"]) * n * (1 + c["need_grad"]) + 12 * c["B"] + 4), "flops": 4.0 * n}
    shapes, half = _clip_shapes(c, 0)
    n = [math.prod(s) for s in shapes]
    return {"bytes": float(2 * sum(k * (2 if h else 4) for k, h in zip(n, half))), "flops": 3.0 * sum(n)}


# --------------------------------------------------------------------------------------------- inputs
def _inputs(c, seed):
    """Inputs of the distributions that training meets: samples and states ~ N(0, 1), weights ~ N(0, 1/K), biases ~ N(0, 0.1),
    gradients of a mean over the rows, logits a few units wide, gradients of a thousandth."""
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(shape, std, dtype="f32"):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std).to(TYPES[dtype])

    x = {}
    if c["op"] in ("forward", "backward"):
        M, K, F = c["M"], c["K"], c["F"]
        x["X"], x["W"] = normal((M, K), 1.0, c["x"]), normal((F, K), K ** -0.5, c["w"])
        if c["op"] == "forward":
            x["b"] = normal((F,), 0.1 ** 0.5) if c["bias"] else None
            x["R"] = normal((M, F), 1.0, c["y"]) if c["residual"] else None
        else:
            x["dY"] = normal((M, F), 1.0 / M, c["y"])
            z = normal((M, F), 1.0)                               # pre-activations, and the factors that a forward pass keeps of them
            x["D"] = None if c["act"] == "identity" else (SCALE * ((z > 0).float() if c["act"] == "relu" else 1.0 - torch.tanh(z) ** 2)).to(TYPES[c["y"]])
    elif c["op"] == "loss":
        B, V = c["B"], c["V"]
        x["labels"] = torch.randint(0, V, (B,), generator=g, device=DEV, dtype=torch.int64)
        x["logits"] = normal((B, V), 2.0, c["dtype"])
        if c["masked"]:
            out = torch.rand((V,), generator=g, device=DEV) < c["masked"]
            out[0] = False                                        # one class is left at least
            x["logits"][:, out] = -math.inf
            x["labels"][out[x["labels"]]] = 0
        if c["ignored"]:
            x["labels"][torch.rand((B,), generator=g, device=DEV) < c["ignored"]] = -1
    else:
        shapes, half = _clip_shapes(c, seed)
        x["flat"], x["src"], x["dst"], x["out"] = {}, [None] * len(shapes), [None] * len(shapes), {}
        for t, is_half in (("f32", False), ("bf16", True)):
            which = [i for i, h in enumerate(half) if h == is_half]
            n = [math.prod(shapes[i]) for i in which]
            if not which:
                continue
            x["flat"][t], x["out"][t] = normal((sum(n),), 1.0e-3, t), torch.empty((sum(n),), device=DEV, dtype=TYPES[t])
            for k in ("src", "dst"):
                for i, v in zip(which, torch.split(x["flat" if k == "src" else "out"][t], n)):
                    x[k][i] = v.view(shapes[i])
    return x


ACTS = {"tanh": 0, "relu": 1, "identity": 2}
ENUM = {"f32": 0, "bf16": 1}


def _handle(c, s):
    """What a program that calls the library keeps: the description of the operator, outputs and the workspace."""
    import paper_2007_07336_amd as mgrit

    def new(shape, t="f32"):
        return torch.empty(shape, device=DEV, dtype=TYPES[t])

    if c["op"] in ("forward", "backward"):
        M, K, F = c["M"], c["K"], c["F"]
        p = mgrit.make_affine(M=M, K=K, F=F, act=ACTS[c["act"]], xtype=ENUM[c["x"]], wtype=ENUM[c["w"]], ytype=ENUM[c["y"]],
                              scale=1.0 if c["act"] == "identity" else SCALE)
        if c["op"] == "forward":
            nbytes = mgrit.mgrit_affine_workspace_bytes(p)
            s.update(Y=new((M, F), c["y"]), D=new((M, F), c["y"]) if c["factor"] else None)
        else:
            nbytes = mgrit.mgrit_affine_backward_workspace_bytes(p)
            s.update(dX=new((M, K), c["x"]) if c["need_dx"] else None, dW=new((F, K)), db=new((F,)))
    elif c["op"] == "loss":
        p = mgrit.make_loss(B=c["B"], V=c["V"], dtype=ENUM[c["dtype"]], reduction=1, scale=1.0)
        nbytes = mgrit.mgrit_cross_entropy_workspace_bytes(p)
        s.update(loss=new((1,)), rows=new((c["B"],)), grad=new((c["B"], c["V"]), c["dtype"]) if c["need_grad"] else None)
    else:
        p = mgrit.make_tensor_list(s["src"], s["dst"])
        nbytes = mgrit.mgrit_clip_workspace_bytes(p)
        s.update(norm=new((1,)))
    s.update(p=p, ws=torch.empty(nbytes, device=DEV, dtype=torch.uint8), mgrit=mgrit)


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    if own:
        _handle(case, s)
    return s


# --------------------------------------------------------------------------------------------- one pass
def _run_own(c, s):
    m = s["mgrit"]
    if c["op"] == "forward":
        m.mgrit_affine_forward(s["p"], s["X"], s["W"], s["b"], s["R"], s["Y"], s["D"], s["ws"])
        return {"Y": s["Y"], "D": s["D"]}
    if c["op"] == "backward":
        m.mgrit_affine_backward(s["p"], s["X"], s["W"], s["D"], s["dY"], s["dX"], s["dW"], s["db"], s["ws"])
        return {"dX": s["dX"], "dW": s["dW"], "db": s["db"]}
    if c["op"] == "loss":
        m.mgrit_cross_entropy(s["p"], s["logits"], s["labels"], s["loss"], s["rows"], s["grad"], s["ws"])
        return {"loss": s["loss"], "rows": s["rows"], "grad": s["grad"]}
    m.mgrit_clip_gradients(s["p"], c["max_norm"], s["norm"], s["ws"])
    return {"norm": s["norm"], "out": s["out"]}


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(c, s)
    if c["op"] == "forward":
        z = s["X"].float() @ s["W"].float().T
        if s["b"] is not None:
            z = z + s["b"]
        if c["act"] == "identity":
            y, d = z, None
        elif c["act"] == "relu":
            y, d = SCALE * torch.clamp(z, min=0.0), None
        else:
            t = torch.tanh(z)
            y, d = SCALE * t, SCALE * (1.0 - t * t) if c["factor"] else None
        if s["R"] is not None:
            y = s["R"].float() + y
        to = TYPES[c["y"]]
        return {"Y": y.to(to), "D": None if d is None else d.to(to)}
    if c["op"] == "backward":
        G = s["dY"].float()
        if s["D"] is not None:
            G = G * s["D"].float()
        dX = (G @ s["W"].float()).to(TYPES[c["x"]]) if c["need_dx"] else None
        return {"dX": dX, "dW": G.T @ s["X"].float(), "db": G.sum(0)}
    if c["op"] == "loss":
        x, y = s["logits"].float(), s["labels"]
        counted = y >= 0
        at = torch.clamp(y, min=0)[:, None]
        top = x.max(dim=1, keepdim=True).values
        e = torch.exp(x - top)
        total = e.sum(dim=1, keepdim=True)
        rows = torch.where(counted, (torch.log(total) + top - x.gather(1, at))[:, 0], 0.0)
        n = torch.clamp(counted.sum(), min=1).float()
        loss = (rows.sum() / n).reshape(1)
        if not c["need_grad"]:
            return {"loss": loss, "rows": rows, "grad": None}
        p = e / total
        p.scatter_add_(1, at, torch.full_like(total, -1.0))
        grad = p * (counted.float() / n)[:, None]
        return {"loss": loss, "rows": rows, "grad": grad.to(TYPES[c["dtype"]])}
    norm = torch.stack([t.float().square().sum() for t in s["src"]]).sum().sqrt().reshape(1)
    f = torch.clamp(c["max_norm"] / norm, max=1.0)
    [d.copy_(t.float() * f) for t, d in zip(s["src"], s["dst"])]
    return {"norm": norm, "out": s["out"]}


# --------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if c["op"] == "forward":
        z = torch.matmul(x["X"].double(), x["W"].double().t())
        if c["bias"]:
            z += x["b"].double()
        s = 1.0 if c["act"] == "identity" else SCALE
        a = {"identity": lambda v: v, "relu": torch.relu, "tanh": torch.tanh}[c["act"]](z)
        Y = s * a + (x["R"].double() if c["residual"] else 0.0)
        return {"Y": Y, "D": s / torch.cosh(z) ** 2 if c["factor"] else None}
    if c["op"] == "backward":
        G = x["dY"].double()
        if c["act"] != "identity":
            G = G * x["D"].double()
        return {"dX": torch.matmul(G, x["W"].double()) if c["need_dx"] else None,
                "dW": torch.matmul(G.t(), x["X"].double()), "db": G.sum(dim=0)}
    if c["op"] == "loss":
        y, V = x["labels"], c["V"]
        rows = torch.zeros((c["B"],), device=DEV, dtype=torch.float64)
        grad = torch.zeros((c["B"], V), device=DEV, dtype=torch.float64) if c["need_grad"] else None
        n = max(1, int((y >= 0).sum()))
        for r in range(0, c["B"], 256):
            v, k = x["logits"][r:r + 256].double(), y[r:r + 256]
            lse = torch.logsumexp(v, dim=1)
            ok = k >= 0
            hot = (torch.arange(V, device=DEV)[None] == k[:, None])
            rows[r:r + 256] = torch.where(ok, lse - torch.where(hot, v, 0.0).sum(dim=1), 0.0)
            if grad is not None:
                grad[r:r + 256] = torch.where(ok[:, None], torch.exp(v - lse[:, None]) - hot.double(), 0.0) / n
        return {"loss": (rows.sum() / n).reshape(1), "rows": rows, "grad": grad}
    ss = sum(float((f.double() ** 2).sum()) for f in x["flat"].values())
    norm = math.sqrt(ss)
    f = c["max_norm"] / norm if norm > c["max_norm"] else 1.0
    return {"norm": torch.tensor([norm], device=DEV, dtype=torch.float64), "out": {k: v.double() * f for k, v in x["flat"].items()}}
