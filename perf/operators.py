"""The attention half of a block as cases that can be timed and compared: norms and rotation of queries and keys, and
attention over blocks of keys that an 8-bit score selects for each query.

Kinds of pass, through the public calls of ``paper_2408_11746_amd``:

``rotate``       norm of every query and key head and the rotation by its position, from the rows of a fused qkv product
``rotate_back``  the gradients of that: of both inputs, inside the gradient of such a row, and of both weights
``attend``       summaries of all key blocks, selection, plan and attention forward
``train``        the same and the gradients of queries, keys and values
``token``        one new token per sequence over a cache: summary of a block that it completes, selection, attention
"""
import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def _rotate(name, kind, batch, tokens, heads, kv_heads, dim, rotated, interleaved, x, y):
    return dict(name=name, kind=kind, batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, rotated=rotated,
                interleaved=interleaved, x=x, y=y)


def _attend(name, kind, batch, tokens, heads, kv_heads, dim, block, select, dtype, ragged=False):
    return dict(name=name, kind=kind, batch=batch, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, block=block,
                select=select, dtype=dtype, ragged=ragged)


def listed():
    return [
        # the next token of 32 sequences on a GPT-2-small block: nothing but latency
        _rotate("rotate_token", "rotate", 32, 1, 12, 12, 64, 64, False, "bf16", "bf16"),
        # the batch of configuration C5 on the GPT-2-large block: fp32 rows as the sparse product writes them, bfloat16 heads
        # for the attention
        _rotate("rotate_batch", "rotate", 8, 1024, 20, 20, 64, 64, False, "f32", "bf16"),
        # packed sequences of odd length, shared key heads, neighbouring pairs, part of the head rotated, all in fp32
        _rotate("rotate_back_odd", "rotate_back", 3, 1531, 16, 4, 128, 96, True, "f32", "f32"),
        # the batch of configuration C4 on the GPT-2-medium block, bfloat16 rows
        _rotate("rotate_back_batch", "rotate_back", 16, 1024, 16, 16, 64, 64, False, "bf16", "bf16"),
        # evaluation on GPT-2's own sequence length: few blocks, a third of them read
        _attend("attend_short", "attend", 16, 1024, 12, 12, 64, 64, 6, "bf16"),
        # fp32 heads of an unusual width, an odd length, short blocks, two query heads to a key head
        _attend("attend_odd_f32", "attend", 2, 2999, 10, 5, 80, 32, 8, "f32", ragged=True),
        # a long prompt with shared key heads
        _attend("attend_long", "attend", 1, 32768, 32, 8, 128, 128, 16, "bf16"),
        # a micro-batch of the GPT-2-small block
        _attend("train_small", "train", 4, 1024, 12, 12, 64, 64, 4, "bf16"),
        # the batch of configuration C5 as one long sequence on the GPT-2-large block
        _attend("train_large", "train", 1, 8192, 20, 20, 64, 64, 8, "bf16"),
        # left-padded sequences of odd length, three query heads to a key head
        _attend("train_odd", "train", 2, 4099, 24, 8, 128, 64, 8, "bf16", ragged=True),
        # answering in a small service: eight sequences of up to 1024 tokens
        _attend("token_small", "token", 8, 1024, 12, 12, 64, 64, 4, "bf16", ragged=True),
        # answering in a large one: 64 sequences of up to 16384 tokens, shared key heads
        _attend("token_large", "token", 64, 16384, 32, 8, 128, 64, 16, "bf16", ragged=True),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate_back", "attend", "attend", "train", "train", "token", "token"])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 12])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8])
    dim = rng.choice([64, 64, 128, 128, 32, 40, 80, 96])
    if kind.startswith("rotate"):
        batch = rng.choice([1, 2, 3, 8, 16])
        tokens = min(_log_uniform(rng, 1, 16384), max(1, 40_000_000 // (batch * (heads + kv_heads) * dim)))
        rotated = rng.choice([dim, dim, dim // 2, 0])
        c = _rotate("", kind, batch, tokens, heads, kv_heads, dim, rotated, rng.random() < 0.4, rng.choice(["f32", "bf16"]),
                    rng.choice(["f32", "bf16", "bf16"]))
    else:
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        block, select = rng.choice([32, 64, 64, 128]), rng.choice([2, 4, 8, 8, 12, 16])
        if kind == "token":
            batch = _log_uniform(rng, 1, 64)
            tokens = min(_log_uniform(rng, 16, 32768), 2_000_000_000 // (batch * kv_heads * dim * 4))
        else:
            batch = rng.choice([1, 1, 2, 4])
            # (row, key) pairs times width of the plain form: below the largest listed case's, a third of it with gradients
            most = (4.0e12 if kind == "attend" else 0.5e12) / (batch * heads * dim)
            tokens = min(_log_uniform(rng, 16, 16384), int(math.sqrt(most)))
        c = _attend("", kind, batch, tokens, heads, kv_heads, dim, block, select, dtype, rng.random() < 0.5)
    del c["name"]
    return c


# ---------------------------------------------------------------- inputs

def _lengths(case):
    """tokens of each sequence: all of them, or from about half to all"""
    B, T = case["batch"], case["tokens"]
    return [T - (b * (T // 2)) // B - (b % 3 if T > 8 else 0) for b in range(B)] if case["ragged"] else [T] * B


def _unit(x):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)


def _table(rows, rotated):
    """[rows, rotated]: cosines, then sines, of the angles of a position"""
    half = rotated // 2
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    return torch.cat([angle.cos(), angle.sin()], 1).float().to(DEVICE)


def _prepare_rotate(case, gen):
    B, T, H, G, D = case["batch"], case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    n = lambda *s: torch.randn(*s, generator=gen, device=DEVICE)  # noqa: E731
    rows = (n(B, T, (H + 2 * G) * D) * torch.exp(0.5 * n((H + 2 * G) * D))).to(TYPES[case["x"]])
    st = dict(case=case, rows=rows, wq=1 + 0.1 * n(D), wk=1 + 0.1 * n(D), table=_table(16384 + 64, case["rotated"]),
              positions=(torch.arange(T, device=DEVICE)[None] + torch.randint(0, 64, (B, 1), generator=gen, device=DEVICE)).int().contiguous(),
              out=torch.empty(B, T, H + G, D, dtype=TYPES[case["y"]], device=DEVICE))
    if case["kind"] == "rotate_back":
        st["dy"] = n(B, T, H + G, D).to(TYPES[case["y"]])
        st["drows"] = torch.zeros_like(rows)
        st["dwq"], st["dwk"] = torch.empty(D, device=DEVICE), torch.empty(D, device=DEVICE)
    return st


def _prepare_attend(case, gen):
    """Heads as a trained model gives them: a token has one of 48 topics, kept for some 150 tokens; the keys of a topic point one way,
    the queries ask for it, and the rest is each token's own."""
    B, S, H, G, D = case["batch"], case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    token, dtype = case["kind"] == "token", TYPES[case["dtype"]]
    T = 1 if token else S
    n = lambda *s: torch.randn(*s, generator=gen, device=DEVICE)  # noqa: E731
    part = (torch.rand(B, S, generator=gen, device=DEVICE) < 1 / 150).cumsum(1)
    topic = torch.randint(0, 48, (B, S + 1), generator=gen, device=DEVICE).gather(1, part)
    heading = n(G, 48, D)
    # (in bfloat16 from the start: a large cache in fp32 would be made longer than it is read)
    k = heading.to(dtype).permute(1, 0, 2)[topic]
    k = _unit_rows(k.add_(torch.randn(B, S, G, D, generator=gen, device=DEVICE, dtype=dtype)))
    v = torch.randn(B, S, G, D, generator=gen, device=DEVICE, dtype=dtype)
    asked = heading.permute(1, 0, 2)[topic[:, S - T:]].repeat_interleave(H // G, 2)
    q = _unit(asked + n(B, T, H, D)).to(dtype)
    blocks = -(-S // case["block"])
    zeros = lambda *s, t=dtype: torch.zeros(*s, dtype=t, device=DEVICE)  # noqa: E731
    st = dict(case=case, q=q, k=k, v=v, o=torch.empty_like(q), lse=zeros(B, H, T, t=torch.float32),
              sums=zeros(B, G, blocks, D, t=torch.int8), scales=zeros(B, G, blocks, t=torch.float32),
              blocks=zeros(B, G, T, case["select"], t=torch.int32), scale=1 / math.sqrt(D),
              lengths=torch.tensor(_lengths(case), dtype=torch.int32, device=DEVICE))
    if case["kind"] == "train":
        st["do"] = n(B, T, H, D).to(dtype)
        st["dq"], st["dk"], st["dv"] = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    if token:  # the summaries of the cache before the new token; it completes a block at most
        done = (st["lengths"].long() - 1) // case["block"]
        sums, scales = _summaries(k, case["block"])
        kept = (torch.arange(sums.shape[2], device=DEVICE) < done[:, None])[:, None]
        st["sums"][:, :, :sums.shape[2]] = torch.where(kept[..., None], sums, 0)
        st["scales"][:, :, :sums.shape[2]] = torch.where(kept, scales, 0)
    return st


def _unit_rows(k):
    """k / rms(k), in place"""
    return k.mul_(torch.rsqrt(torch.linalg.vector_norm(k, dim=-1, keepdim=True, dtype=torch.float32).square() / k.shape[-1] + EPS))


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    st = (_prepare_rotate if case["kind"].startswith("rotate") else _prepare_attend)(case, gen)
    if own:
        _handles(st)   # the descriptions and workspaces that a program keeps beside its buffers
    return st


def _handles(st):
    import paper_2408_11746_amd as mst
    c, types = st["case"], {"f32": mst.MST_F32, "bf16": mst.MST_BF16}
    space = lambda n: torch.empty(max(n, 16), dtype=torch.uint8, device=DEVICE)  # noqa: E731
    st["mst"] = mst
    if c["kind"].startswith("rotate"):
        st["shape"] = mst.QKNormShape(c["batch"], c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["rotated"], c["interleaved"],
                                      st["table"].shape[0], EPS, types[c["x"]], types[c["y"]])
        st["ws"] = space(mst.mst_qk_norm_rotate_workspace_bytes(st["shape"]))
        return
    st["shape"] = mst.BlockAttentionShape(c["batch"], st["q"].shape[1], c["tokens"], c["heads"], c["kv_heads"], c["dim"], c["block"],
                                          c["select"], st["scale"], types[c["dtype"]], st["lengths"])
    if c["kind"] != "token":
        st["plan"] = space(mst.mst_block_plan_bytes(st["shape"]))
        st["ws"] = space(mst.mst_block_attention_workspace_bytes(st["shape"], c["kind"] == "train"))


# ---------------------------------------------------------------- one pass

def run(st):
    kind = st["case"]["kind"]
    if kind.startswith("rotate"):
        return _own_rotate(st) if own else _plain_rotate(st)
    return _own_attend(st) if own else _plain_attend(st)


def _own_rotate(st):
    mst, c, shape = st["mst"], st["case"], st["shape"]
    H, G, D = c["heads"], c["kv_heads"], c["dim"]
    x = st["rows"].view(c["batch"], c["tokens"], H + 2 * G, D)
    q, k = x[:, :, :H], x[:, :, H:H + G]
    if c["kind"] == "rotate":
        y = st["out"]
        mst.mst_qk_norm_rotate(shape, q, k, st["wq"], st["wk"], st["table"], st["positions"], y[:, :, :H], y[:, :, H:])
        return {"q": y[:, :, :H], "k": y[:, :, H:]}
    dx, dy = st["drows"].view(x.shape), st["dy"]
    mst.mst_qk_norm_rotate_bwd(shape, q, k, st["wq"], st["wk"], st["table"], st["positions"], dy[:, :, :H], dy[:, :, H:],
                               dx[:, :, :H], dx[:, :, H:H + G], st["dwq"], st["dwk"], st["ws"])
    return {"dq": dx[:, :, :H], "dk": dx[:, :, H:H + G], "dwq": st["dwq"], "dwk": st["dwk"]}


def _own_attend(st):
    mst, c, shape = st["mst"], st["case"], st["shape"]
    q, k, v, o, lse, blocks = st["q"], st["k"], st["v"], st["o"], st["lse"], st["blocks"]
    mst.mst_key_summary(shape, k, st["sums"], st["scales"], q.shape[1])
    mst.mst_block_select(shape, q, st["sums"], st["scales"], blocks)
    out = {"sums": st["sums"], "scales": st["scales"], "blocks": blocks, "o": o, "lse": lse}
    if c["kind"] == "token":
        mst.mst_block_attention_decode(shape, q, k, v, blocks, o, lse)
        return out
    mst.mst_block_plan(shape, blocks, st["plan"])
    mst.mst_block_attention_fwd(shape, q, k, v, st["plan"], o, lse, st["ws"])
    if c["kind"] == "train":
        mst.mst_block_attention_bwd(shape, q, k, v, st["plan"], o, lse, st["do"], st["dq"], st["dk"], st["dv"], st["ws"])
        out.update(dq=st["dq"], dk=st["dk"], dv=st["dv"])
    return out


# ---------------------------------------------------------------- plain form of norm and rotation

def _turn(x, table, rotated, interleaved, back=False):
    """pairs of the leading `rotated` components by their angles; table [B, T, 1, rotated]"""
    half = rotated // 2
    cos, sin = table[..., :half], -table[..., half:] if back else table[..., half:]
    a, b = (x[..., 0:rotated:2], x[..., 1:rotated:2]) if interleaved else (x[..., :half], x[..., half:rotated])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rotated:]], -1)


def _plain_rotate(st):
    c = st["case"]
    H, G, D = c["heads"], c["kv_heads"], c["dim"]
    x = st["rows"].view(c["batch"], c["tokens"], H + 2 * G, D)[:, :, :H + G].float()
    table = st["table"][st["positions"].long()].unsqueeze(2)
    w = torch.cat([st["wq"].expand(H, D), st["wk"].expand(G, D)])
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    if c["kind"] == "rotate":
        y = _turn(x * r * w, table, c["rotated"], c["interleaved"]).to(TYPES[c["y"]])
        return {"q": y[:, :, :H], "k": y[:, :, H:]}
    dn = _turn(st["dy"].float(), table, c["rotated"], c["interleaved"], back=True)
    g = dn * w
    dx = (r * (g - x * r.square() * (g * x).mean(-1, keepdim=True))).to(TYPES[c["x"]])
    dw = (dn * x * r).sum((0, 1))
    return {"dq": dx[:, :, :H], "dk": dx[:, :, H:], "dwq": dw[:H].sum(0), "dwk": dw[H:].sum(0)}


# ---------------------------------------------------------------- plain form of selection and attention

def _power(e):
    """2^e as fp32, from its bits"""
    return ((e + 127).int() << 23).view(torch.float32)


def _exponent(x):
    """floor(log2 x) of x >= 0; far below all others for 0"""
    return torch.where(x > 0, torch.frexp(x)[1] - 1, -1000)


def _to_8_bits(x, dims, over):
    """(8-bit values of the sum of x over `over`, exponent of their unit); the largest component of `dims` sets the first unit"""
    x = torch.where(torch.isfinite(x), x, 0)
    e = _exponent(x.abs().amax(dims, keepdim=True)).clamp(-100, 100)
    s = (x * _power(6 - e)).round().clamp(-127, 127).sum(over, keepdim=True)
    r = (_exponent(s.abs().amax(-1, keepdim=True)) - 6).clamp(min=0)
    return (s * _power(-r)).round().clamp(-127, 127).squeeze(over), (e.amax(over, keepdim=True) - 6 + r).squeeze(over)


def _summaries(k, block):
    """[B, G, complete blocks, D] 8-bit sums of the keys of a block, [B, G, complete blocks] their units"""
    B, S, G, D = k.shape
    n = S // block
    x = k[:, :n * block].view(B, n, block, G, D).float()
    s, e = _to_8_bits(x, (2, 4), 2)
    return s.permute(0, 2, 1, 3).to(torch.int8), _power(e.squeeze(-1)).permute(0, 2, 1)


def _place(c, st, T):
    """[B, T] position of each query"""
    return st["lengths"].long()[:, None] - T + torch.arange(T, device=DEVICE)


def _choose(c, st, q, sums, scales):
    """[B, G, T, select] blocks, ascending, -1 behind; the float scores are exact"""
    B, T, H, D = q.shape
    G, n, place = c["kv_heads"], sums.shape[2], _place(c, st, T)
    q8, _ = _to_8_bits(q.view(B, T, G, H // G, D).float(), (3, 4), 3)
    score = (q8.permute(0, 2, 1, 3) @ sums.float().transpose(2, 3)) * scales[:, :, None]
    at = torch.arange(n, device=DEVICE)
    mine = torch.div(place, c["block"], rounding_mode="floor")[:, None, :, None]
    score = torch.where(at < mine, score, torch.where((at == mine) & (mine >= 0), math.inf, -math.inf))
    order = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :c["select"]]
    order = torch.where(score.gather(-1, order) > -math.inf, order, n).sort(-1).values
    order = torch.where(order < n, order, -1).int()
    return torch.nn.functional.pad(order, (0, c["select"] - order.shape[-1]), value=-1)


def _plain_attend(st):
    c = st["case"]
    B, T, H, D = st["q"].shape
    S, G, block = c["tokens"], c["kv_heads"], c["block"]
    sums, scales = st["sums"].clone(), st["scales"].clone()
    if c["kind"] == "token":  # the block that the new token may complete
        last = (st["lengths"].long() - 1) // block
        whole = st["lengths"] % block == 0
        keys = (last[:, None] * block + torch.arange(block, device=DEVICE)).clamp(max=S - 1)
        each = torch.arange(B, device=DEVICE)
        s1, e1 = _summaries(st["k"][each[:, None], keys], block)
        sums[each, :, last] = torch.where(whole[:, None, None], s1[:, :, 0], sums[each, :, last])
        scales[each, :, last] = torch.where(whole[:, None], e1[:, :, 0], scales[each, :, last])
    else:
        s1, e1 = _summaries(st["k"], block)
        done = (torch.arange(s1.shape[2], device=DEVICE) < (st["lengths"] // block)[:, None])[:, None]
        sums[:, :, :s1.shape[2]] = torch.where(done[..., None], s1, 0)
        scales[:, :, :s1.shape[2]] = torch.where(done, e1, 0)
    blocks = _choose(c, st, st["q"], sums, scales)
    out = {"sums": sums, "scales": scales, "blocks": blocks}
    out.update(_plain_token(c, st, blocks) if c["kind"] == "token" else _plain_sequences(c, st, blocks))
    return out


def _plain_token(c, st, blocks):
    B, T, H, D = st["q"].shape
    S, G, block = c["tokens"], c["kv_heads"], c["block"]
    keys = (blocks[:, :, 0, :, None].long() * block + torch.arange(block, device=DEVICE)).flatten(2)   # [B, G, n]
    seen = (keys >= 0) & (keys < st["lengths"][:, None, None])
    keys = keys.clamp(0, S - 1)
    b, g = torch.arange(B, device=DEVICE)[:, None, None], torch.arange(G, device=DEVICE)[None, :, None]
    k, v = st["k"][b, keys, g].float(), st["v"][b, keys, g].float()
    s = torch.where(seen[:, :, None], (st["q"].view(B, G, H // G, D).float() @ k.transpose(2, 3)) * st["scale"], -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    return {"o": ((p / l) @ v).view(B, T, H, D).to(st["q"].dtype), "lse": (m + l.log()).view(B, H, T)}


def _plain_sequences(c, st, blocks):
    """dense products under the mask of the selection, as many key heads at a time as 24 GB hold"""
    B, T, H, D = st["q"].shape
    S, G, block, train = c["tokens"], c["kv_heads"], c["block"], c["kind"] == "train"
    R = H // G
    rows = lambda x: x.view(B, T, G, R, D).permute(0, 2, 3, 1, 4).reshape(B * G, R * T, D).float()  # noqa: E731
    flat = lambda x: x.permute(0, 2, 1, 3).reshape(B * G, S, D).float()  # noqa: E731
    q, k, v = rows(st["q"]), flat(st["k"]), flat(st["v"])
    do = rows(st["do"]) if train else None
    place = _place(c, st, T).repeat_interleave(G, 0)
    blocks = blocks.view(B * G, T, -1).long()
    n = -(-S // block)
    got, at_once = [], max(1, int(24e9 // (R * T * S * 4 * (4 if train else 3))))
    for i in range(0, B * G, at_once):
        j = slice(i, i + at_once)
        chosen = torch.zeros(blocks[j].shape[0], T, n + 1, dtype=torch.bool, device=DEVICE)
        chosen.scatter_(2, torch.where(blocks[j] < 0, n, blocks[j]), True)
        seen = chosen[..., :n].repeat_interleave(block, 2)[..., :S] & (torch.arange(S, device=DEVICE) <= place[j, :, None])
        s = ((q[j] * st["scale"]) @ k[j].transpose(1, 2)).view(-1, R, T, S)
        s.masked_fill_(~seen[:, None], -math.inf)
        m = s.amax(-1, keepdim=True)
        p = torch.exp(s.sub_(torch.where(m > -math.inf, m, 0)))
        l = p.sum(-1, keepdim=True)
        p = p.div_(torch.where(l > 0, l, 1)).view(-1, R * T, S)
        o = p @ v[j]
        one = [o, (m + l.log()).view(-1, R * T)]
        if train:
            ds = do[j] @ v[j].transpose(1, 2)
            ds = ds.sub_((do[j] * o).sum(-1, keepdim=True)).mul_(p)
            one += [ds @ k[j] * st["scale"], ds.transpose(1, 2) @ q[j] * st["scale"], p.transpose(1, 2) @ do[j]]
        got.append(one)
    o, lse, *grads = [torch.cat(x) for x in zip(*got)]
    back = lambda x: x.view(B, G, R, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, H, D).to(st["q"].dtype)  # noqa: E731
    keys = lambda x: x.view(B, G, S, D).permute(0, 2, 1, 3).to(st["q"].dtype)  # noqa: E731
    out = {"o": back(o), "lse": lse.view(B, H, T)}
    if train:
        out.update(dq=back(grads[0]), dk=keys(grads[1]), dv=keys(grads[2]))
    return out


# ---------------------------------------------------------------- what a pass cannot do without

def _pairs(case):
    """(selected (query, key) pairs of one key head over all sequences, (query, candidate block) pairs)"""
    n = pairs = scored = 0
    for length in _lengths(case):
        for p in range(length - 1 if case["kind"] == "token" else 0, length):
            mine = p // case["block"]
            pairs += min(case["select"] - 1, mine) * case["block"] + p % case["block"] + 1
            scored += mine
    return pairs, scored


def work(case):
    B, T, H, G, D = case["batch"], case["tokens"], case["heads"], case["kv_heads"], case["dim"]
    size = {"f32": 4, "bf16": 2}
    if case["kind"].startswith("rotate"):
        n = B * T * (H + G) * D
        angles = B * T * 4 + min(B * T, 16448) * case["rotated"] * 4
        if case["kind"] == "rotate":
            return {"bytes": n * (size[case["x"]] + size[case["y"]]) + angles + 8 * D, "flops": 8 * n}
        return {"bytes": n * (2 * size[case["x"]] + size[case["y"]]) + angles + 16 * D, "flops": 18 * n}
    z = size[case["dtype"]]
    pairs, scored = _pairs(case)
    flops = 4 * D * H * pairs + 2 * D * G * scored
    if case["kind"] == "token":
        rows = B * H * D * 2 * z + B * H * 4 + B * G * case["select"] * 4
        return {"bytes": rows + pairs * G * D * 2 * z + scored * G * (D + 4), "flops": flops}
    total = sum(_lengths(case))
    blocks = sum(n // case["block"] for n in _lengths(case)) * G
    moved = total * (2 * H + 2 * G) * D * z + total * H * 4 + total * G * case["select"] * 4 + blocks * (D + 4)
    if case["kind"] == "train":
        moved += total * (2 * H + 2 * G) * D * z
        flops += 10 * D * H * pairs
    return {"bytes": moved, "flops": flops}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(case, seed):
    st = _prepare_rotate(case, torch.Generator(device=DEVICE).manual_seed(seed)) if case["kind"].startswith("rotate") else \
        _prepare_attend(case, torch.Generator(device=DEVICE).manual_seed(seed))
    return _exact_rotate(case, st) if case["kind"].startswith("rotate") else _exact_attend(case, st)


def _exact_rotate(case, st):
    """as a product with complex numbers; the gradients from torch's differentiation of it"""
    H, G, D, R = case["heads"], case["kv_heads"], case["dim"], case["rotated"]
    x = st["rows"].view(case["batch"], case["tokens"], H + 2 * G, D)[:, :, :H + G].double()
    angle = torch.complex(st["table"][:, :R // 2].double(), st["table"][:, R // 2:].double())[st["positions"].long()][:, :, None]

    def forward(x, wq, wk):
        w = torch.cat([wq.expand(H, D), wk.expand(G, D)])
        y = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / D + EPS) * w
        if case["interleaved"]:
            z = torch.complex(y[..., 0:R:2], y[..., 1:R:2]) * angle
            turned = torch.view_as_real(z).flatten(-2)
        else:
            z = torch.complex(y[..., :R // 2], y[..., R // 2:R]) * angle
            turned = torch.cat([z.real, z.imag], -1)
        return torch.cat([turned, y[..., R:]], -1)

    wq, wk = st["wq"].double(), st["wk"].double()
    if case["kind"] == "rotate":
        y = forward(x, wq, wk)
        return {"q": y[:, :, :H], "k": y[:, :, H:]}
    x, wq, wk = (t.requires_grad_() for t in (x, wq, wk))
    dx, dwq, dwk = torch.autograd.grad(forward(x, wq, wk), (x, wq, wk), st["dy"].double())
    return {"dq": dx[:, :, :H], "dk": dx[:, :, H:], "dwq": dwq, "dwk": dwk}


def _two_to(e):
    """2^e in 64 bits, looked up (a power that a device computes may be one off in its last bit)"""
    return torch.tensor([2.0 ** i for i in range(-300, 301)], dtype=torch.float64, device=DEVICE)[e.long() + 300]


def _exact_eight(x, members):
    """x [..., members * D] integers or numbers in 64 bits -> 8-bit sums over the members and the exponent of their unit"""
    x = torch.where(torch.isfinite(x), x, 0.0)
    top = x.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.frexp(top)[1] - 1, -100).clamp(-100, 100)
    s = torch.round(x * _two_to(6 - e)).clamp(-127, 127).unflatten(-1, (members, -1)).sum(-2)
    r = (torch.frexp(s.abs().amax(-1, keepdim=True))[1] - 7).clamp(min=0)
    return torch.round(s * _two_to(-r)).clamp(-127, 127), (e - 6 + r)[..., 0]


def _exact_attend(case, st):
    """query by query over gathered keys, a slice of queries at a time"""
    q, k, v = st["q"], st["k"], st["v"]
    B, T, H, D = q.shape
    S, G, block, select = case["tokens"], case["kv_heads"], case["block"], case["select"]
    R, n, lengths = H // G, S // block, _lengths(case)
    sums, units = torch.zeros_like(st["sums"]), torch.zeros_like(st["scales"])
    if n:
        s8, e8 = _exact_eight(k[:, :n * block].double().unflatten(1, (n, block)).permute(0, 3, 1, 2, 4).flatten(-2), block)
        for b in range(B):
            whole = lengths[b] // block
            sums[b, :, :whole] = s8[b, :, :whole].to(torch.int8)
            units[b, :, :whole] = _two_to(e8[b, :, :whole]).float()
    train = case["kind"] == "train"
    o, lse = torch.zeros(B, T, H, D, dtype=torch.float64, device=DEVICE), torch.full((B, H, T), -math.inf, dtype=torch.float64, device=DEVICE)
    grads = [torch.zeros(x.shape, dtype=torch.float64, device=DEVICE) for x in (q, k, v)] if train else []
    blocks = torch.full((B, G, T, select), -1, dtype=torch.int32, device=DEVICE)
    slice_of = max(1, int(2e8 // (select * block * D)))
    for b in range(B):
        for g in range(G):
            heads = slice(g * R, (g + 1) * R)
            kb, vb = k[b, :, g].double(), v[b, :, g].double()
            for t in range(max(0, T - lengths[b]), T, slice_of):
                u = min(t + slice_of, T)
                p = torch.arange(t, u, device=DEVICE) + (lengths[b] - T)
                mine = p // block
                qb = q[b, t:u, heads].double()                                      # [t, R, D]
                q8, _ = _exact_eight(qb.flatten(1), R)
                # integers below 2^53 and powers of two: the order of the sum changes nothing
                at = torch.arange(sums.shape[2], device=DEVICE)
                score = (q8 @ sums[b, g].double().T) * units[b, g].double()
                score = torch.where(at < mine[:, None], score, torch.where(at == mine[:, None], math.inf, -math.inf))
                _, first = torch.sort(-score, dim=1, stable=True)
                first = first[:, :select]
                taken = score.gather(1, first) > -math.inf
                first = torch.where(taken, first, 1 << 20).sort(1).values
                blocks[b, g, t:u, :first.shape[1]] = torch.where(first < 1 << 20, first, -1).int()
                keys = (first[:, :, None] * block + torch.arange(block, device=DEVICE)).flatten(1)
                seen = keys <= p[:, None]
                keys = torch.where(seen, keys, 0)
                kk, vv = kb[keys], vb[keys]                                         # [t, n, D]
                s = torch.where(seen[:, None], qb @ kk.transpose(1, 2) * st["scale"], -math.inf)
                z = torch.logsumexp(s, 2)
                w = torch.exp(s - z[..., None])
                o[b, t:u, heads], lse[b, heads, t:u] = w @ vv, z.T
                if train:
                    d = st["do"][b, t:u, heads].double()
                    dw = d @ vv.transpose(1, 2)
                    ds = w * (dw - (w * dw).sum(-1, keepdim=True)) * st["scale"]
                    grads[0][b, t:u, heads] = ds @ kk
                    grads[1][b, :, g].index_add_(0, keys.flatten(), (ds.transpose(1, 2) @ qb).flatten(0, 1))
                    grads[2][b, :, g].index_add_(0, keys.flatten(), (w.transpose(1, 2) @ d).flatten(0, 1))
    out = {"sums": sums, "scales": units, "blocks": blocks, "o": o, "lse": lse}
    if train:
        out.update(dq=grads[0], dk=grads[1], dv=grads[2])
    return out
