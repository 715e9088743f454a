"""Performance cases of the operators around the layer-parallel solver that keep values in few bits or turn logits into answers: an end
layer with weights in microscaled 4 bits, the backward pass of an end layer from activations that were kept in 8 bits, the norms before and after a block with its gate and residual scale, and the drawing of classes from logits.

Microscaled: rows in blocks of 32 entries, each block with a power of two as its scale, the smallest one for which no entry of the block
exceeds the format's largest value (mx8: 448, sign, 4 exponent and 3 mantissa bits; mx4: 6, sign, 2 and 1); entries are rounded to
nearest, ties to even.

A case is a dict; its `op` says which operator, the rest its sizes and types:
  packed    z = X~ W~^T + b, Y = R + scale act(z), W~ the mx4 values of W, X~ those of X or X rounded to bf16:   M, K, F, x, xf, y (type of X, form of
            X~, type of R and Y), act, bias, residual.  W is packed already, as a server keeps it; X is not.
  kept      X and the activation's factors D are packed to mx8, then G = dY D~, dX = G W, dW = G^T X~, db = sum of G over rows:   M, K, F, x, w, y
            (types of X and dX; W; dY and D), act (identity: no D), need_dx
  norm      n = norm(f) w_post, s = r + scale gate n, y = norm(s) w_pre:   M, q, kind (rms, or layer: less its mean), stream (type of r, s), branch (type of
            f, y and the gate), gate (none, feature: [q], entry: [M][q]), post, pre (whether there is that norm), back: the backward pass, from f, s and
            the gradients by s and y
  sample    one class for each row of logits from a given random number: the classes in falling order (ties: lowest index first), of them the first
            top_k, the fewest that hold top_p of their probability, and those of at least min_p of the largest one; of what is left the first
            class in index order whose running sum of probabilities exceeds u:   B, V, dtype, temperature, top_k, top_p, min_p (whether each
            is given, a value a row), masked (share of the classes at minus infinity)
Where `own` is false the operators run in plain torch operations, where it is true through the library.
"""
import math
import random

import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SCALE = 0.5                         # of a branch: of an activation, or of a block between its norms
EPS = 1.0e-6                        # of the norms
LARGEST = {"mx8": (448.0, -6, 3), "mx4": (6.0, 0, 1)}         # largest value, least exponent, mantissa bits


def _packed(name, M, K, F, x, xf, y, act, **kw):
    return dict(dict(name=name, op="packed", M=M, K=K, F=F, x=x, xf=xf, y=y, act=act, bias=True, residual=False), **kw)


def _kept(name, M, K, F, types, act, **kw):
    return dict(dict(name=name, op="kept", M=M, K=K, F=F, x=types[0], w=types[1], y=types[2], act=act, need_dx=True), **kw)


def _norm(name, M, q, kind, stream, branch, gate, **kw):
    return dict(dict(name=name, op="norm", M=M, q=q, kind=kind, stream=stream, branch=branch, gate=gate, post=True, pre=True, back=False), **kw)


def _sample(name, B, V, dtype, **kw):
    return dict(dict(name=name, op="sample", B=B, V=V, dtype=dtype, temperature=True, top_k=False, top_p=False, min_p=False, masked=0.0), **kw)


F32, BF16, STATES = ("f32",) * 3, ("bf16",) * 3, ("f32", "bf16", "f32")


def listed():
    return [
        # one sample's logits over many classes, as answered one at a time: the weights in 4 bits are most of the bytes
        _packed("single_mx4", 1, 4096, 32768, "bf16", "bf16", "bf16", "identity", bias=False),
        # a fully connected layer of flattened images (d = 4096) with skip connection on a serving batch, float states
        _packed("connected4096_mx4", 48, 4096, 4096, "f32", "bf16", "f32", "tanh", residual=True),
        # an opening layer whose sizes fit no tile and no block
        _packed("ragged_mx4", 1000, 1031, 517, "f32", "mx4", "f32", "relu"),
        # a wide layer on many samples, with skip connection
        _packed("wide_mx4", 8192, 4096, 4096, "bf16", "mx4", "bf16", "tanh", residual=True),
        # the head of the large image stack (64 channels, 32 x 32, batch 32) backwards, its inputs kept in 8 bits
        _kept("close10_states_kept", 32, 65536, 10, STATES, "identity"),
        # the largest: a wide bf16 layer on many samples backwards, inputs and factors kept in 8 bits
        _kept("wide_bf16_kept", 8192, 4096, 4096, BF16, "tanh"),
        # the norms around a block of the wide training stack (1024 features) on a small serving batch: the smallest call
        _norm("norm1024_f32_forward", 32, 1024, "rms", "f32", "f32", "none"),
        # the same of a training batch with odd sizes, backwards, a gate for each feature
        _norm("norm_ragged_backward", 1000, 1031, "layer", "f32", "f32", "feature", back=True),
        # a wide bf16 block between float states, a gate for each entry, backwards
        _norm("norm_wide_backward", 8192, 4096, "rms", "f32", "bf16", "entry", back=True),
        # one answer over many classes with everything that narrows the choice
        _sample("answer50021_bf16", 1, 50021, "bf16", top_k=True, top_p=True),
        # a serving batch's answers, float logits, each row with its own settings
        _sample("answers32768_f32", 256, 32768, "f32", top_k=True, top_p=True, min_p=True, masked=0.05),
        # many rows' answers from all classes that hold a share of the probability
        _sample("answers50021_bf16", 4096, 50021, "bf16", top_p=True),
    ]


# --------------------------------------------------------------------------------------------- drawn cases
def draw(rng: random.Random):
    def logint(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))

    def size(lo, hi):               # a whole multiple of 64 half the time, else whatever comes
        n = logint(lo, hi)
        return n if n < 128 or rng.random() < 0.5 else n // 64 * 64

    while True:
        op = rng.choice(["packed", "packed", "kept", "norm", "norm", "sample"])
        if op in ("packed", "kept"):
            c = dict(op=op, M=size(1, 8192), K=size(8, 65536), F=size(2, 65536), act=rng.choice(["identity", "tanh", "relu"]))
            if c["M"] * c["K"] * c["F"] > 8192 * 4096 * 4096 or max(c["M"] * c["K"], c["K"] * c["F"], c["M"] * c["F"]) > 1 << 27:
                continue
            if op == "packed":
                c.update(x=rng.choice(["f32", "bf16"]), xf=rng.choice(["bf16", "mx4"]), y=rng.choice(["f32", "bf16"]),
                         bias=rng.random() < 0.8, residual=rng.random() < 0.5)
            else:
                c["x"], c["w"], c["y"] = rng.choice([F32, BF16, BF16, STATES, STATES, ("f32", "f32", "bf16")])
                c.update(need_dx=rng.random() < 0.8)
            return c
        if op == "norm":
            c = dict(op=op, M=logint(1, 32768), q=size(8, 16384), kind=rng.choice(["rms", "layer"]), stream=rng.choice(["f32", "f32", "bf16"]),
                     branch=rng.choice(["f32", "bf16"]), gate=rng.choice(["none", "feature", "entry"]), back=rng.random() < 0.6)
            c["post"], c["pre"] = rng.choice([(True, True), (True, True), (False, True), (True, False)])
            if c["M"] * c["q"] <= 1 << 26:
                return c
            continue
        c = dict(op=op, B=logint(1, 8192), V=logint(2, 131072), dtype=rng.choice(["f32", "bf16"]), masked=rng.choice([0.0, 0.05, 0.5]))
        for k in ("temperature", "top_k", "top_p", "min_p"):
            c[k] = rng.random() < 0.6
        if c["B"] * c["V"] <= 4096 * 50021:
            return c


# --------------------------------------------------------------------------------------------- counts
def _bytes(t):
    return {"f32": 4.0, "bf16": 2.0, "mx8": 33.0 / 32.0, "mx4": 17.0 / 32.0}[t]


def work(case):
    c = case
    if c["op"] == "packed":
        M, K, F = c["M"], c["K"], c["F"]
        b = _bytes(c["x"]) * M * K + _bytes("mx4") * F * K + _bytes(c["y"]) * M * F * (1 + c["residual"]) + 4 * F * c["bias"]
        return {"bytes": float(b), "flops": 2.0 * M * K * F}
    if c["op"] == "kept":
        M, K, F = c["M"], c["K"], c["F"]
        b = _bytes(c["x"]) * M * K * (1 + c["need_dx"]) + _bytes(c["w"]) * F * K * c["need_dx"] + _bytes(c["y"]) * M * F * (1 + (c["act"] != "identity"))
        return {"bytes": float(b + 4 * F * K + 4 * F), "flops": 2.0 * M * K * F * (1 + c["need_dx"])}
    if c["op"] == "norm":
        n, s, b = c["M"] * c["q"], _bytes(c["stream"]), _bytes(c["branch"])
        entry, vectors = b * (c["gate"] == "entry"), 4 * c["q"] * (c["post"] + c["pre"] + (c["gate"] == "feature"))
        if not c["back"]:
            return {"bytes": float(n * (2 * s + b * (1 + c["pre"]) + entry) + vectors), "flops": 12.0 * n}
        return {"bytes": float(n * (3 * s + b * (2 + c["pre"]) + 2 * entry) + 2 * vectors), "flops": 25.0 * n}
    n = c["B"] * c["V"]
    return {"bytes": float(_bytes(c["dtype"]) * n + 16 * c["B"]), "flops": 4.0 * n}


# --------------------------------------------------------------------------------------------- inputs
def _inputs(c, seed):
    """Inputs of the distributions that training and serving meet: samples, states and branches ~ N(0, 1), weights ~ N(0, 1/K), biases
    ~ N(0, 0.1), norm weights around one, gates in (0, 1), gradients of a mean over the rows, logits a few units wide."""
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(shape, std, dtype="f32", mean=0.0):
        return (torch.randn(shape, generator=g, device=DEV, dtype=torch.float32) * std + mean).to(TYPES[dtype])

    def uniform(shape, lo=0.0, hi=1.0):
        return torch.rand(shape, generator=g, device=DEV, dtype=torch.float32) * (hi - lo) + lo

    x = {}
    if c["op"] == "packed":
        M, K, F = c["M"], c["K"], c["F"]
        x["X"], x["W"] = normal((M, K), 1.0, c["x"]), normal((F, K), K ** -0.5, "bf16")
        x["b"] = normal((F,), 0.1 ** 0.5) if c["bias"] else None
        x["R"] = normal((M, F), 1.0, c["y"]) if c["residual"] else None
    elif c["op"] == "kept":
        M, K, F = c["M"], c["K"], c["F"]
        x["X"], x["W"] = normal((M, K), 1.0, c["x"]), normal((F, K), K ** -0.5, c["w"])
        x["dY"] = normal((M, F), 1.0 / M, c["y"])
        z = normal((M, F), 1.0)                                   # pre-activations, and the factors that a forward pass makes of them
        x["D"] = None if c["act"] == "identity" else (SCALE * ((z > 0).float() if c["act"] == "relu" else 1.0 - torch.tanh(z) ** 2)).to(TYPES[c["y"]])
    elif c["op"] == "norm":
        M, q = c["M"], c["q"]
        x["f"], x["r"] = normal((M, q), 1.0, c["branch"]), normal((M, q), 1.0, c["stream"])
        x["gate"] = None if c["gate"] == "none" else torch.sigmoid(normal((q,) if c["gate"] == "feature" else (M, q), 1.0))
        if c["gate"] == "entry":
            x["gate"] = x["gate"].to(TYPES[c["branch"]])
        x["post"] = normal((q,), 0.1, mean=1.0) if c["post"] else None
        x["pre"] = normal((q,), 0.1, mean=1.0) if c["pre"] else None
        if c["back"]:                                             # (r is the sum's value here: the backward pass takes s)
            x["dS"], x["dY"] = normal((M, q), 1.0 / M, c["stream"]), normal((M, q), 1.0 / M, c["branch"]) if c["pre"] else None
    else:
        B, V = c["B"], c["V"]
        x["logits"], x["u"] = normal((B, V), 2.0, c["dtype"]), uniform((B,))
        if c["masked"]:
            out = uniform((V,)) < c["masked"]
            out[0] = False                                        # one class is left at least
            x["logits"][:, out] = -math.inf
        x["temperature"] = uniform((B,), 0.5, 1.5) if c["temperature"] else None
        if c["temperature"]:
            x["temperature"][3::8] = 0.0                          # some rows ask for the largest logit
        x["top_k"] = torch.randint(1, 101, (B,), generator=g, device=DEV, dtype=torch.int32) if c["top_k"] else None
        x["top_p"] = uniform((B,), 0.7, 1.0) if c["top_p"] else None
        x["min_p"] = uniform((B,), 0.0, 0.1) if c["min_p"] else None
    return x


ACTS = {"tanh": 0, "relu": 1, "identity": 2}
ENUM = {"f32": 0, "bf16": 1}


def _handle(c, s):
    """What a program that calls the library keeps: the description of the operator, packed weights, outputs and the workspace."""
    import paper_2007_07336_amd as mgrit

    def new(shape, t="f32"):
        return torch.empty(shape, device=DEV, dtype=TYPES[t])

    def room(n):
        return torch.empty(n, device=DEV, dtype=torch.uint8)

    if c["op"] == "packed":
        M, K, F = c["M"], c["K"], c["F"]
        w = mgrit.make_packed(rows=F, cols=K, format=mgrit.MGRIT_MX4, dtype=mgrit.MGRIT_BF16)
        s["packed"] = room(mgrit.mgrit_packed_bytes(w))
        mgrit.mgrit_pack(w, s["W"], s["packed"])
        p = mgrit.make_affine_packed(M=M, K=K, F=F, act=ACTS[c["act"]], xtype=ENUM[c["x"]], xformat={"bf16": mgrit.MGRIT_BF16, "mx4": mgrit.MGRIT_MX4}[c["xf"]],
                                     ytype=ENUM[c["y"]], scale=1.0 if c["act"] == "identity" else SCALE)
        s.update(p=p, Y=new((M, F), c["y"]), ws=room(mgrit.mgrit_affine_packed_workspace_bytes(p)))
    elif c["op"] == "kept":
        M, K, F = c["M"], c["K"], c["F"]
        p = mgrit.make_affine(M=M, K=K, F=F, act=ACTS[c["act"]], xtype=ENUM[c["x"]], wtype=ENUM[c["w"]], ytype=ENUM[c["y"]])
        s.update(p=p, px=mgrit.make_packed(rows=M, cols=K, format=mgrit.MGRIT_MX8, dtype=ENUM[c["x"]]),
                 pd=mgrit.make_packed(rows=M, cols=F, format=mgrit.MGRIT_MX8, dtype=ENUM[c["y"]]))
        s.update(keptX=room(mgrit.mgrit_packed_bytes(s["px"])), keptD=None if s["D"] is None else room(mgrit.mgrit_packed_bytes(s["pd"])),
                 dX=new((M, K), c["x"]) if c["need_dx"] else None, dW=new((F, K)), db=new((F,)), ws=room(mgrit.mgrit_affine_kept_workspace_bytes(p)))
    elif c["op"] == "norm":
        M, q = c["M"], c["q"]
        p = mgrit.make_block_norm(M=M, q=q, kind={"rms": mgrit.MGRIT_NORM_ROOT, "layer": mgrit.MGRIT_NORM_LAYER}[c["kind"]], stype=ENUM[c["stream"]],
                                  ftype=ENUM[c["branch"]], eps=EPS, scale=SCALE, gate={"none": mgrit.MGRIT_GATE_NONE, "feature": mgrit.MGRIT_GATE_FEATURE,
                                                                                       "entry": mgrit.MGRIT_GATE_ENTRY}[c["gate"]])
        s.update(p=p)
        if c["back"]:
            s.update(df=new((M, q), c["branch"]), dr=new((M, q), c["stream"]), dgate=None if s["gate"] is None else torch.empty_like(s["gate"]),
                     dpost=new((q,)) if c["post"] else None, dpre=new((q,)) if c["pre"] else None, ws=room(mgrit.mgrit_block_norm_workspace_bytes(p)))
        else:
            s.update(S=new((M, q), c["stream"]), Y=new((M, q), c["branch"]) if c["pre"] else None)
    else:
        p = mgrit.make_sample(B=c["B"], V=c["V"], dtype=ENUM[c["dtype"]])
        s.update(p=p, index=torch.empty((c["B"],), device=DEV, dtype=torch.int64), logprob=new((c["B"],)),
                 ws=room(mgrit.mgrit_sample_workspace_bytes(p)))
    s["mgrit"] = mgrit


def prepare(case, seed):
    s = dict(_inputs(case, seed), case=dict(case))
    if own:
        _handle(case, s)
    elif case["op"] == "packed":
        s["packed"] = _pack(s["W"], "mx4")                   # the weights' values as a server keeps them
    return s


# --------------------------------------------------------------------------------------------- one pass
def _run_own(c, s):
    m = s["mgrit"]
    if c["op"] == "packed":
        m.mgrit_affine_packed_forward(s["p"], s["X"], s["packed"], s["b"], s["R"], s["Y"], None, s["ws"])
        return {"Y": s["Y"]}
    if c["op"] == "kept":
        m.mgrit_pack(s["px"], s["X"], s["keptX"])
        if s["D"] is not None:
            m.mgrit_pack(s["pd"], s["D"], s["keptD"])
        m.mgrit_affine_kept_backward(s["p"], s["keptX"], s["W"], s["keptD"], s["dY"], s["dX"], s["dW"], s["db"], s["ws"])
        return {"dX": s["dX"], "dW": s["dW"], "db": s["db"]}
    if c["op"] == "norm":
        if c["back"]:
            m.mgrit_block_norm_backward(s["p"], s["f"], s["r"], s["gate"], s["post"], s["pre"], s["dS"], s["dY"], s["df"], s["dr"], s["dgate"], s["dpost"],
                                        s["dpre"], s["ws"])
            return {k: s[k] for k in ("df", "dr", "dgate", "dpost", "dpre")}
        m.mgrit_block_norm_forward(s["p"], s["f"], s["r"], s["gate"], s["post"], s["pre"], s["S"], s["Y"])
        return {"S": s["S"], "Y": s["Y"]}
    m.mgrit_sample(s["p"], s["logits"], s["u"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], s["index"], s["logprob"], s["ws"])
    return {"index": s["index"], "logprob": s["logprob"]}


def _two(e):
    """2^e, to the last bit (torch.ldexp need not be: it takes a power)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _pack(x, form):
    """The microscaled values of the rows of x, in float (every step is exact but the rounding to the format; 64 bits for the powers of two)."""
    largest, least, bits = LARGEST[form]
    rows, n = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -n % 32)).view(rows, -1, 32)
    top = v.abs().amax(2, keepdim=True)
    m, e = torch.frexp(top)
    a, b = math.frexp(largest)
    shift = torch.where(top > 0, e - b + (m > a).int(), -127).clamp(min=-127)          # scale 2^shift
    v = v * _two(-shift)
    step = (torch.frexp(v)[1] - 1).clamp(min=least) - bits
    v = torch.round(v * _two(-step)) * _two(step + shift)
    return v.view(rows, -1)[:, :n].float()


def _norm_of(x, layer):
    """The normalised rows and their reciprocal deviations."""
    if layer:
        x = x - x.mean(1, keepdim=True)
    d = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * d, d


def _norm_back(h, n, d, layer):
    """The gradient by the rows that were normalised, h by the normalised n."""
    return d * (h - n * (h * n).mean(1, keepdim=True) - (h.mean(1, keepdim=True) if layer else 0.0))


def _sample_rows(c, x, u, t, k, p, least):
    """Classes and logarithms of their probabilities of some rows."""
    B, V = x.shape
    x = x.double()
    greedy = torch.zeros((B, 1), device=DEV, dtype=torch.bool) if t is None else (t == 0)[:, None]
    z = x - x.amax(1, keepdim=True)
    if t is not None:
        z = z / torch.where(t == 0, 1.0, t).double()[:, None]
    order, by = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp(order)
    place = torch.arange(V, device=DEV)[None]
    count = torch.where(greedy, 1, torch.full((B, 1), V, device=DEV))                  # how many of the order are left
    if k is not None:
        count = torch.minimum(count, k.long()[:, None])
    if p is not None:
        run_ = torch.cumsum(torch.where(place < count, w, 0.0), 1)
        enough = (run_ < p.double()[:, None] * run_[:, -1:]).sum(1, keepdim=True) + 1
        count = torch.where(p[:, None] < 1, torch.minimum(count, enough), count)
    if least is not None:
        count = torch.minimum(count, (w >= least.double()[:, None]).sum(1, keepdim=True))
    w = torch.zeros_like(w).scatter_(1, by, torch.where(place < count, w, 0.0))        # in index order again
    run_ = torch.cumsum(w, 1)
    total = run_[:, -1:]
    at = (run_ <= u.double()[:, None] * total).sum(1, keepdim=True).clamp(max=V - 1)
    return at[:, 0], (z.gather(1, at) - torch.log(total))[:, 0]


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(c, s)
    if c["op"] == "packed":
        z = (_pack(s["X"], "mx4") if c["xf"] == "mx4" else s["X"].bfloat16().float()) @ s["packed"].T
        if s["b"] is not None:
            z = z + s["b"]
        y = z if c["act"] == "identity" else SCALE * (torch.clamp(z, min=0.0) if c["act"] == "relu" else torch.tanh(z))
        if s["R"] is not None:
            y = s["R"].float() + y
        return {"Y": y.to(TYPES[c["y"]])}
    if c["op"] == "kept":
        X = _pack(s["X"], "mx8")
        G = s["dY"].float()
        if s["D"] is not None:
            G = G * _pack(s["D"], "mx8")
        dX = (G @ s["W"].float()).to(TYPES[c["x"]]) if c["need_dx"] else None
        return {"dX": dX, "dW": G.T @ X, "db": G.sum(0)}
    if c["op"] == "norm":
        layer, to, branch = c["kind"] == "layer", TYPES[c["stream"]], TYPES[c["branch"]]
        f, gate = s["f"].float(), 1.0 if s["gate"] is None else s["gate"].float()
        fn, fd = _norm_of(f, layer) if c["post"] else (f, None)
        n = fn * s["post"] if c["post"] else fn
        if not c["back"]:
            S = s["r"].float() + SCALE * gate * n
            return {"S": S.to(to), "Y": (_norm_of(S, layer)[0] * s["pre"]).to(branch) if c["pre"] else None}
        ds, dpre = s["dS"].float(), None
        if c["pre"]:
            sn, sd = _norm_of(s["r"].float(), layer)
            dy = s["dY"].float()
            ds, dpre = ds + _norm_back(dy * s["pre"], sn, sd, layer), (dy * sn).sum(0)
        t = SCALE * ds
        dgate = None if s["gate"] is None else (t * n).sum(0) if c["gate"] == "feature" else (t * n).to(branch)
        dn, dpost = t * gate, None
        if c["post"]:
            dpost, dn = (dn * fn).sum(0), _norm_back(dn * s["post"], fn, fd, layer)
        return {"df": dn.to(branch), "dr": ds.to(to), "dgate": dgate, "dpost": dpost, "dpre": dpre}
    some = [s[k] for k in ("temperature", "top_k", "top_p", "min_p")]
    parts = [_sample_rows(c, s["logits"][r:r + 1024], s["u"][r:r + 1024], *[None if a is None else a[r:r + 1024] for a in some]) for r in range(0, c["B"], 1024)]
    return {"index": torch.cat([a for a, _ in parts]), "logprob": torch.cat([b for _, b in parts]).float()}


# --------------------------------------------------------------------------------------------- the same in 64 bits
def _exact_values(x, form):
    """The microscaled values of the rows of x in double, from the definition."""
    rows, n = x.shape
    v = torch.zeros((rows, (n + 31) // 32 * 32), device=DEV, dtype=torch.float64)
    v[:, :n] = x.double()
    v = v.reshape(-1, 32)
    top, largest = v.abs().max(dim=1).values, LARGEST[form][0]
    shift = torch.ceil(torch.log2(torch.clamp(top, min=1.0e-300) / largest)).clamp(min=-127.0)
    power = torch.tensor([2.0 ** i for i in range(-130, 131)], device=DEV, dtype=torch.float64)
    shift = shift.long() + 130
    shift = shift + (top > largest * power[shift]).long()                              # (the logarithm may be a rounding off)
    shift = torch.where((shift > 3) & (top <= largest * power[shift - 1]), shift - 1, shift)
    v = v / power[shift][:, None]
    if form == "mx8":
        v = v.float().to(torch.float8_e4m3fn).double()
    else:
        grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV, dtype=torch.float64)
        a = v.abs()
        up = torch.bucketize(a, grid).clamp(max=7)                                     # first grid value >= a
        down = (up - 1).clamp(min=0)
        low, high = grid[down], grid[up]
        take_up = (a - low > high - a) | ((a - low == high - a) & (up % 2 == 0))       # ties to the even code
        v = torch.where(take_up, high, low) * torch.sign(v)
    return (v * power[shift][:, None]).reshape(rows, -1)[:, :n]


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if c["op"] == "packed":
        X = _exact_values(x["X"], "mx4") if c["xf"] == "mx4" else x["X"].to(torch.bfloat16).double()
        z = torch.matmul(X, _exact_values(x["W"], "mx4").t())
        if c["bias"]:
            z += x["b"].double()
        Y = {"identity": lambda v: v, "relu": lambda v: SCALE * torch.relu(v), "tanh": lambda v: SCALE * torch.tanh(v)}[c["act"]](z)
        return {"Y": Y + x["R"].double() if c["residual"] else Y}
    if c["op"] == "kept":
        G = x["dY"].double()
        if c["act"] != "identity":
            G = G * _exact_values(x["D"], "mx8")
        return {"dX": torch.matmul(G, x["W"].double()) if c["need_dx"] else None, "dW": torch.matmul(G.t(), _exact_values(x["X"], "mx8")), "db": G.sum(dim=0)}
    if c["op"] == "norm":
        v = {k: None if t is None else t.double() for k, t in x.items()}

        def normed(a, w):
            if c["kind"] == "layer":
                return w * (a - a.mean(dim=1, keepdim=True)) / torch.sqrt(a.var(dim=1, unbiased=False, keepdim=True) + EPS)
            return w * a / torch.sqrt(a.square().mean(dim=1, keepdim=True) + EPS)

        def block(f, r, gate, post):
            n = normed(f, post) if c["post"] else f
            return r + SCALE * (n if gate is None else gate * n)

        if not c["back"]:
            S = block(v["f"], v["r"], v["gate"], v["post"])
            return {"S": S, "Y": normed(S, v["pre"]) if c["pre"] else None}
        # by automatic differentiation: first of y by s, then, with the whole gradient by s, of s = r + .. by the rest
        ds, dpre = v["dS"], None
        if c["pre"]:
            S, pre = v["r"].requires_grad_(), v["pre"].requires_grad_()
            more, dpre = torch.autograd.grad(normed(S, pre), (S, pre), v["dY"])
            ds = ds + more
        names = [k for k in ("f", "gate", "post") if v[k] is not None]
        leaves = {k: v[k].requires_grad_() for k in names}
        got = dict(zip(names, torch.autograd.grad(block(leaves["f"], torch.zeros_like(ds), leaves.get("gate"), leaves.get("post")), [leaves[k] for k in names], ds)))
        return {"df": got["f"], "dr": ds, "dgate": got.get("gate"), "dpost": got.get("post"), "dpre": dpre}
    B, V = c["B"], c["V"]
    index, logprob = torch.zeros((B,), device=DEV, dtype=torch.int64), torch.zeros((B,), device=DEV, dtype=torch.float64)
    for r in range(0, B, 256):
        part = {k: None if x[k] is None else x[k][r:r + 256] for k in ("logits", "u", "temperature", "top_k", "top_p", "min_p")}
        L = part["logits"].double()
        rows = L.shape[0]
        t = torch.ones((rows,), device=DEV, dtype=torch.float64) if part["temperature"] is None else part["temperature"].double()
        by = torch.argsort(-L, dim=1, stable=True)
        rank = torch.empty_like(by)
        rank.scatter_(1, by, torch.arange(V, device=DEV).expand(rows, V))
        # (a temperature of zero is the limit: all of the probability on the first of the order)
        P = L / torch.where(t > 0, t, 1.0)[:, None]
        P = torch.exp(P - P.max(dim=1, keepdim=True).values)                           # (torch.softmax is 1e-9 off in 64 bits)
        P = P / P.sum(dim=1, keepdim=True)
        keep = torch.where((t > 0)[:, None], rank < V, rank < 1)
        if part["top_k"] is not None:
            keep &= rank < part["top_k"].long()[:, None]
        P1 = P * keep
        if part["top_p"] is not None:
            q = (P1 / P1.sum(dim=1, keepdim=True)).gather(1, by)
            before = torch.cumsum(q, dim=1) - q                                        # what comes before each in the order
            keep &= (before < part["top_p"].double()[:, None]).gather(1, rank)
        if part["min_p"] is not None:
            keep &= P >= part["min_p"].double()[:, None] * P.max(dim=1, keepdim=True).values
        P = P * keep
        P = P / P.sum(dim=1, keepdim=True)
        over = torch.cumsum(P, dim=1) > part["u"].double()[:, None]
        at = torch.argmax(over.int(), dim=1)
        index[r:r + 256], logprob[r:r + 256] = at, torch.log(P.gather(1, at[:, None])[:, 0])
    return {"index": index, "logprob": logprob}
