"""What a training step does around the products and the attention of its blocks, as cases that can be timed and compared: residual
and layer norm, the activation between fc1 and fc2, activations kept in 8 bits for the backward pass, and the loss over the vocabulary.

Kinds of pass, through the public calls of ``paper_2408_11746_amd``:

``norm``        sum of a branch and the residual stream, layer norm of it
``norm_step``   the same and its gradients, from the sum
``norm_kept``   the same with the sum kept in 8 bits: the gradients, and the normed rows again, from what was kept
``gelu_step``   activation and its gradient, from its input
``gelu_kept``   the same from the input kept in 8 bits, and the activation again
``keep``        any activation into 8 bits and back
``loss``        log-sums and losses of tokens over the vocabulary
``loss_step``   the same and the gradients of the hidden states and of the embedding
"""
import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-5
GROUP = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def _rows(name, kind, rows, width, x, y="bf16", dy="f32", dx="f32", erf=False):
    return dict(name=name, kind=kind, rows=rows, width=width, x=x, y=y, dy=dy, dx=dx, erf=erf)


def _loss(name, kind, tokens, width, vocab, dtype, unlabelled=0.0):
    return dict(name=name, kind=kind, tokens=tokens, width=width, vocab=vocab, dtype=dtype, unlabelled=unlabelled)


def listed():
    return [
        # the next token of 32 sequences on a GPT-2-small block: nothing but latency
        _rows("norm_token", "norm", 32, 768, "f32"),
        # the batch of configuration C5 on the GPT-2-large block: what the sparse products write is fp32, so is the residual stream
        _rows("norm_step_batch", "norm_step", 8192, 1280, "f32"),
        # packed sequences of odd length, an odd width, all in fp32
        _rows("norm_step_odd", "norm_step", 3 * 1531, 1001, "f32", "f32"),
        # the batch of configuration C4 on the GPT-2-medium block, a bfloat16 stream kept in 8 bits
        _rows("norm_kept_batch", "norm_kept", 16384, 1024, "bf16", "bf16", "bf16"),
        # between fc1 and fc2 of the GPT-2-large block: fp32 products in and out, bfloat16 activations and gradients for them
        _rows("gelu_step_batch", "gelu_step", 8192, 5120, "f32", "bf16", "f32", "bf16"),
        # the same on the GPT-2-medium block with its input kept in 8 bits
        _rows("gelu_kept_batch", "gelu_kept", 16384, 4096, "f32", "bf16", "f32", "bf16"),
        # the attention's output of a micro-batch of the GPT-2-small block, kept for proj's weight gradient
        _rows("keep_small", "keep", 4096, 768, "bf16"),
        # rows that end inside a group, fp32
        _rows("keep_odd", "keep", 4099, 1601, "f32"),
        # scoring one token of each of eight sequences: reads the embedding once
        _loss("loss_token", "loss", 8, 768, 50257, "bf16"),
        # a micro-batch of the GPT-2-small block, a quarter of it prompts and padding without labels
        _loss("loss_step_small", "loss_step", 1024, 768, 50257, "bf16", 0.25),
        # the batch of configuration C5 on the GPT-2-large width
        _loss("loss_step_batch", "loss_step", 8192, 1280, 50257, "bf16"),
        # odd sizes in fp32
        _loss("loss_step_odd_f32", "loss_step", 1531, 648, 32003, "f32", 0.1),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    kind = rng.choice(["norm", "norm_step", "norm_step", "norm_kept", "gelu_step", "gelu_kept", "keep", "loss", "loss_step", "loss_step"])
    if kind.startswith("loss"):
        width = rng.choice([256, 384, 512, 640, 768, 1024, 1280, 1600, 8 * rng.randint(24, 200)])
        vocab = rng.choice([50257, 50304, 32000, _log_uniform(rng, 500, 60000)])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        most = (0.1e12 if dtype == "f32" else 0.5e12) / (width * vocab)
        tokens = max(1, min(_log_uniform(rng, 1, 16384), int(most)))
        c = _loss("", kind, tokens, width, vocab, dtype, rng.choice([0.0, 0.0, 0.1, 0.5]))
    else:
        most = 40_000_000 if kind.startswith("gelu") else 16_000_000
        width = rng.choice([256, 768, 1024, 1280, 1600, 4096, 5120, _log_uniform(rng, 64, 8192)])
        rows = min(_log_uniform(rng, 1, 32768), max(1, most // width))
        c = _rows("", kind, rows, width, *(rng.choice(["f32", "bf16"]) for _ in range(4)), erf=kind.startswith("gelu") and rng.random() < 0.3)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    st = _prepare_loss(case, gen) if case["kind"].startswith("loss") else _prepare_rows(case, gen)
    if own:
        _handles(st)   # the descriptions and workspaces that a program keeps beside its buffers
    return st


def _empty(*sizes, t):
    return torch.empty(*sizes, dtype=t, device=DEVICE)


def _prepare_rows(case, gen):
    """Rows of a residual stream: components of different sizes, a few of them large, and a branch that adds to them."""
    R, W, kind = case["rows"], case["width"], case["kind"]
    x_type, y_type, dy_type, dx_type = (TYPES[case[n]] for n in ("x", "y", "dy", "dx"))
    n = lambda *s: torch.randn(*s, generator=gen, device=DEVICE)  # noqa: E731
    size = torch.exp(0.4 * n(W)) * torch.where(torch.rand(W, generator=gen, device=DEVICE) < 0.01, 8.0, 1.0)
    st = dict(case=case, x=(n(R, W) * size).to(x_type))
    if kind.startswith("norm"):
        st.update(residual=(n(R, W).add_(0.3).mul_(size)).to(x_type), weight=1 + 0.1 * n(W), bias=0.1 * n(W),
                  total=_empty(R, W, t=x_type), y=_empty(R, W, t=y_type))
        if kind != "norm":
            st.update(dy=n(R, W).to(dy_type), d_total=n(R, W).to(x_type), dx=_empty(R, W, t=x_type),
                      dweight=_empty(W, t=torch.float32), dbias=_empty(W, t=torch.float32))
    elif kind.startswith("gelu"):
        st.update(y=_empty(R, W, t=y_type), dy=n(R, W).to(dy_type), dx=_empty(R, W, t=dx_type))
    else:
        st["again"] = _empty(R, W, t=x_type)
    if kind.endswith("kept"):
        st["again"] = _empty(R, W, t=y_type)
    if kind.endswith("kept") or kind == "keep":
        st.update(codes=_empty(R, W, t=torch.int8), units=_empty(R, -(-W // GROUP), t=torch.float32))
    return st


def _prepare_loss(case, gen):
    """Hidden states as a trained model gives them: a token's state leans towards the embedding of its label; labels are as unequally
    frequent as words are; the loss is a mean over the tokens that have one."""
    T, W, V, dtype = case["tokens"], case["width"], case["vocab"], TYPES[case["dtype"]]
    n = lambda *s: torch.randn(*s, generator=gen, device=DEVICE)  # noqa: E731
    rand = lambda *s: torch.rand(*s, generator=gen, device=DEVICE)  # noqa: E731
    E = n(V, W).mul_(3 / math.sqrt(W)).add_(0.5 / math.sqrt(W) * n(W))
    label = (torch.exp(rand(T).double() * math.log(V)).long() - 1).clamp(0, V - 1)
    h = n(T, W).add_(E[label] * (4 / 3 * rand(T, 1)))
    labelled = rand(T) >= case["unlabelled"]
    st = dict(case=case, h=h.to(dtype), E=E.to(dtype), labels=torch.where(labelled, label, -100).int(),
              loss=_empty(T, t=torch.float32), lse=_empty(T, t=torch.float32))
    if case["kind"] == "loss_step":
        st.update(d_loss=labelled / labelled.sum().clamp(min=1).float(), dh=_empty(T, W, t=dtype), dE=_empty(V, W, t=dtype))
    return st


def _handles(st):
    import paper_2408_11746_amd as mst
    c, types = st["case"], {"f32": mst.MST_F32, "bf16": mst.MST_BF16}
    space = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device=DEVICE)  # noqa: E731
    st["mst"] = mst
    if c["kind"].startswith("loss"):
        st["shape"] = mst.VocabLossShape(c["tokens"], c["width"], c["vocab"], types[c["dtype"]])
        st["ws"] = space(mst.mst_vocab_loss_workspace_bytes(st["shape"], c["kind"] == "loss_step"))
        return
    st["kept"] = mst.Checkpoint8(st["codes"], st["units"]) if "codes" in st else None
    if c["kind"].startswith("norm"):
        st["shape"] = mst.LayerNormShape(c["rows"], c["width"], EPS, types[c["x"]], types[c["y"]], types[c["dy"]])
        st["ws"] = space(mst.mst_layer_norm_workspace_bytes(st["shape"]))
    elif c["kind"].startswith("gelu"):
        st["shape"] = mst.GeluShape(c["rows"], c["width"], c["erf"], types[c["x"]], types[c["y"]], types[c["dy"]], types[c["dx"]])
    else:
        st["type"] = types[c["x"]]


# ---------------------------------------------------------------- one pass

def run(st):
    kind = st["case"]["kind"]
    if kind.startswith("norm"):
        return _own_norm(st) if own else _plain_norm(st)
    if kind.startswith("gelu"):
        return _own_gelu(st) if own else _plain_gelu(st)
    if kind == "keep":
        return _own_keep(st) if own else {"again": _keep(st["x"].float()).to(st["x"].dtype)}
    return _own_loss(st) if own else _plain_loss(st)


def _own_norm(st):
    mst, shape, kind, kept = st["mst"], st["shape"], st["case"]["kind"], st["kept"]
    mst.mst_layer_norm_fwd(shape, st["x"], st["residual"], st["weight"], st["bias"], st["total"], st["y"], kept)
    out = {"total": st["total"], "y": st["y"]}
    if kind == "norm":
        return out
    again = st.get("again")
    mst.mst_layer_norm_bwd(shape, None if kept else st["total"], kept, st["weight"], st["bias"], st["dy"], st["d_total"], st["dx"],
                           st["dweight"], st["dbias"], again, st["ws"])
    out.update(dx=st["dx"], dweight=st["dweight"], dbias=st["dbias"])
    if kept:
        out["again"] = again
    return out


def _own_gelu(st):
    mst, shape, kept = st["mst"], st["shape"], st["kept"]
    mst.mst_gelu_fwd(shape, st["x"], st["y"], kept)
    out = {"y": st["y"], "dx": st["dx"]}
    if kept:
        mst.mst_gelu_bwd(shape, None, kept, st["dy"], st["dx"], st["again"])
        out["again"] = st["again"]
    else:
        mst.mst_gelu_bwd(shape, st["x"], None, st["dy"], st["dx"])
    return out


def _own_keep(st):
    mst, c = st["mst"], st["case"]
    mst.mst_checkpoint_write(c["rows"], c["width"], st["x"], st["type"], st["kept"])
    mst.mst_checkpoint_read(c["rows"], c["width"], st["kept"], st["type"], st["again"])
    return {"again": st["again"]}


def _own_loss(st):
    mst, shape = st["mst"], st["shape"]
    mst.mst_vocab_loss_fwd(shape, st["h"], st["E"], st["labels"], st["loss"], st["lse"], st["ws"])
    out = {"loss": st["loss"], "lse": st["lse"]}
    if st["case"]["kind"] == "loss_step":
        mst.mst_vocab_loss_bwd(shape, st["h"], st["E"], st["labels"], st["lse"], st["d_loss"], st["dh"], st["dE"], st["ws"])
        out.update(dh=st["dh"], dE=st["dE"])
    return out


# ---------------------------------------------------------------- plain forms

def _keep(x):
    """x [rows, width] as 8 bits hold it, in fp32: the unit of a group is a 127th of its largest component, and a component the nearest
    multiple of it, by products with fp32's own 1/127 and 1/unit"""
    R, W = x.shape
    x = torch.nn.functional.pad(x, (0, -W % GROUP)).view(R, -1, GROUP)
    unit = (x.abs().amax(-1, keepdim=True) * torch.tensor(1 / 127, dtype=torch.float32, device=DEVICE)).clamp(min=2.0 ** -126)
    return ((x * unit.reciprocal()).round() * unit).view(R, -1)[:, :W]


def _plain_norm(st):
    c = st["case"]
    w, b = st["weight"], st["bias"]
    # (the sum is an output in the stream's type, and what is normed: the backward pass has nothing else)
    total = (st["x"].float() + st["residual"].float()).to(TYPES[c["x"]])

    def normed(s):
        s = s - s.mean(-1, keepdim=True)
        r = torch.rsqrt(s.square().mean(-1, keepdim=True) + EPS)
        return s * r, r
    y = (normed(total.float())[0] * w + b).to(TYPES[c["y"]])
    out = {"total": total, "y": y}
    if c["kind"] == "norm":
        return out
    n, r = normed(_keep(total.float()) if c["kind"] == "norm_kept" else total.float())
    dy = st["dy"].float()
    g = dy * w
    dx = r * (g - g.mean(-1, keepdim=True) - n * (g * n).mean(-1, keepdim=True)) + st["d_total"].float()
    out.update(dx=dx.to(TYPES[c["x"]]), dweight=(dy * n).sum(0), dbias=dy.sum(0))
    if c["kind"] == "norm_kept":
        out["again"] = (n * w + b).to(TYPES[c["y"]])
    return out


def _gelu(x, erf):
    """(activation, its derivative) at x in fp32"""
    if erf:
        phi = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
        return x * phi, phi + x * torch.exp(-0.5 * x * x) * (1 / math.sqrt(2 * math.pi))
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (x + 0.044715 * x * x * x))
    return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * (k * (1 + 3 * 0.044715 * x * x))


def _plain_gelu(st):
    c = st["case"]
    x = st["x"].float()
    out = {"y": _gelu(x, c["erf"])[0].to(TYPES[c["y"]])}
    again, slope = _gelu(_keep(x) if c["kind"] == "gelu_kept" else x, c["erf"])
    out["dx"] = (st["dy"].float() * slope).to(TYPES[c["dx"]])
    if c["kind"] == "gelu_kept":
        out["again"] = again.to(TYPES[c["y"]])
    return out


def _plain_loss(st):
    c = st["case"]
    h, E, labelled = st["h"].float(), st["E"].float(), st["labels"] >= 0
    at = st["labels"].long().clamp(min=0)[:, None]
    z = h @ E.T
    m = z.amax(-1, keepdim=True)
    mine = z.gather(1, at)
    z.sub_(m).exp_()
    l = z.sum(-1, keepdim=True)
    lse = m + l.log()
    out = {"loss": torch.where(labelled, (lse - mine)[:, 0], 0), "lse": torch.where(labelled, lse[:, 0], 0)}
    if c["kind"] == "loss_step":
        d = torch.where(labelled, st["d_loss"], 0)[:, None]
        z.mul_(d / l)
        z.scatter_add_(1, at, -d)
        out.update(dh=(z @ E).to(st["h"].dtype), dE=(z.T @ h).to(st["h"].dtype))
    return out


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["kind"].startswith("loss"):
        T, W, V, z = case["tokens"], case["width"], case["vocab"], size[case["dtype"]]
        n = round(T * (1 - case["unlabelled"]))
        step = case["kind"] == "loss_step"
        return {"bytes": (1 + step) * z * (T + V) * W + (12 + 4 * step) * T, "flops": (6 if step else 2) * n * V * W}
    n, kind = case["rows"] * case["width"], case["kind"]
    x, y, dy, dx = (size[case[k]] for k in ("x", "y", "dy", "dx"))
    if kind == "keep":
        return {"bytes": 2 * x * n, "flops": 4 * n}
    if kind.startswith("gelu"):
        return {"bytes": n * (x + y + dy + dx + (y if kind == "gelu_kept" else 0)), "flops": 30 * n}
    back = 0 if kind == "norm" else dy + 2 * x + (y if kind == "norm_kept" else 0)
    return {"bytes": n * (3 * x + y + back) + 16 * case["width"], "flops": (8 if kind == "norm" else 24) * n}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    if case["kind"].startswith("loss"):
        return _exact_loss(case, _prepare_loss(case, gen))
    st = _prepare_rows(case, gen)
    if case["kind"] == "keep":
        return {"again": _exact_kept(st["x"])}
    return _exact_norm(case, st) if case["kind"].startswith("norm") else _exact_gelu(case, st)


def _exact_kept(x):
    """group by group; the unit and its reciprocal are fp32 numbers by definition, here rounded from 64 bits, and so is what is rounded to a whole one"""
    parts = []
    for piece in x.double().split(GROUP, dim=1):
        unit = (piece.abs().max(dim=1, keepdim=True).values * float(torch.tensor(1 / 127))).float().double()
        unit = torch.where(unit < 2.0 ** -126, 2.0 ** -126, unit)
        code = torch.round((piece * (1 / unit).float().double()).float()).double()
        parts.append(code * unit)
    return torch.cat(parts, 1)


def _exact_norm(case, st):
    """torch's differentiation of the definition"""
    W = case["width"]
    w, b = st["weight"].double(), st["bias"].double()
    total = (st["x"].double() + st["residual"].double()).to(TYPES[case["x"]]).double()

    def forward(s, w, b):
        mean = s.sum(-1, keepdim=True) / W
        variance = ((s - mean) ** 2).sum(-1, keepdim=True) / W
        return (s - mean) / torch.sqrt(variance + EPS) * w + b
    out = {"total": total, "y": forward(total, w, b)}
    if case["kind"] == "norm":
        return out
    s = _exact_kept(total) if case["kind"] == "norm_kept" else total
    s, w, b = (t.requires_grad_() for t in (s, w, b))
    y = forward(s, w, b)
    dx, dweight, dbias = torch.autograd.grad(y, (s, w, b), st["dy"].double())
    out.update(dx=dx + st["d_total"].double(), dweight=dweight, dbias=dbias)
    if case["kind"] == "norm_kept":
        out["again"] = y.detach()
    return out


def _exact_gelu(case, st):
    def forward(x):
        if case["erf"]:
            return x / 2 * torch.special.erfc(-x / math.sqrt(2))
        return x * torch.sigmoid(math.sqrt(8 / math.pi) * (x + 0.044715 * x ** 3))
    x = st["x"].double()
    out = {"y": forward(x)}
    x = (_exact_kept(st["x"]) if case["kind"] == "gelu_kept" else x).requires_grad_()
    again = forward(x)
    out["dx"], = torch.autograd.grad(again, x, st["dy"].double())
    if case["kind"] == "gelu_kept":
        out["again"] = again.detach()
    return out


def _exact_loss(case, st):
    """some tokens at a time"""
    T, V, W = case["tokens"], case["vocab"], case["width"]
    step, E = case["kind"] == "loss_step", st["E"].double()
    new = lambda *s: torch.zeros(*s, dtype=torch.float64, device=DEVICE)  # noqa: E731
    loss, lse = new(T), new(T)
    dh, dE = (new(T, W), new(V, W)) if step else (None, None)
    for some in torch.nonzero(st["labels"] >= 0)[:, 0].split(1024):
        h, label = st["h"][some].double(), st["labels"][some].long()
        z = h @ E.T
        lse[some] = torch.logsumexp(z, 1)
        loss[some] = lse[some] - z[torch.arange(len(some), device=DEVICE), label]
        if step:
            d = st["d_loss"][some].double()[:, None]
            dz = torch.softmax(z, 1) - torch.nn.functional.one_hot(label, V)
            dz *= d
            dh[some] = dz @ E
            dE += dz.T @ h
    out = {"loss": loss, "lse": lse}
    if step:
        out.update(dh=dh, dE=dE)
    return out
