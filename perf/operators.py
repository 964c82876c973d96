"""Operators around a compressed training step: per-head norms of queries and
keys with the position rotation (and their gradients from a compressed context),
the global gradient norm over many tensors, and clipping.

A case is a dict of plain values.  ``prepare`` makes what a program has in hand
before the call, ``run`` is one pass through an operator: the package's calls
where ``own`` is true, else the same formulas in elementary torch operations.
``exact`` computes a case's outputs in 64 bits.

Formulas.  x is [batch, tokens, heads, D]; per head
    r = 1 / sqrt(mean x^2 + eps),   n = x r w,
    y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin
for the R / 2 pairs (a, b) of its first R elements: (i, i + R/2) or (2i, 2i + 1);
y = n behind them.  The context that a training step keeps of x is x cut into
groups of G consecutive elements and rounded stochastically to `bits` bits
(the quantizer of arXiv 2206.11357, App. A.4, per group): with mn, mx a group's
minimum and maximum, t = (x - mn) (2^bits - 1) / (mx - mn), q = floor(t) or one
more if a noise value in (0, 1) is below t - floor(t), and x^ = q step + mn.
Backward, dn = dy rotated back, x^ in place of x (r stays the forward pass's):
    dx = r (dn w - x^ r^2 mean(dn w x^)),   dw = sum over heads and tokens of dn x^ r.
Gradients: norm = sqrt(sum g^2) or max |g| over all tensors,
    out = g min(1, max_norm / (norm + 1e-6)).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-6
RANKS = 2.0                             # a norm over several ranks, beside this one's
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
LARGEST = 2 * 16 * 2048 * 40 * 128      # bytes of queries and keys together


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # the gradients of a graph network of three layers, 256 wide: the smallest list, where the launches count
        dict(name="clip_gcn_f32", op="clip", set="gcn", dtype="f32", kind=2, share=0.5, place="out"),
        # a CNN late in training: the norm stays below its bound and nothing has to be scaled
        dict(name="clip_resnet50_f32_below", op="clip", set="resnet50", dtype="f32", kind=2, share=2.0, place="in"),
        # the norm alone, watched or summed over ranks: an 8-layer encoder, hidden 1024, bf16
        dict(name="norm_encoder8_bf16", op="norm", set="encoder", layers=8, hidden=1024, dtype="bf16", kind=2),
        # the largest gradient element of a vision transformer whose gradients lie in one flat buffer at odd offsets
        dict(name="norm_inf_vit_large_bf16", op="norm", set="vit_large", dtype="bf16", kind=0, flat=True),
        # clipping by a norm that all ranks have agreed on
        dict(name="clip_by_encoder8_bf16", op="clip_by", set="encoder", layers=8, hidden=1024, dtype="bf16", kind=2, share=0.25,
             place="out"),
        # the largest list: BERT-large, fp32, the norm above its bound
        dict(name="clip_bert_large_f32", op="clip", set="encoder", layers=24, hidden=1024, dtype="f32", kind=2, share=0.5,
             place="out"),
        # generation: one token of each of 8 sequences, far into the tables; launch and latency
        dict(name="rotate_one_token_bf16", op="rotate", batch=8, tokens=1, heads_q=16, heads_k=4, dim=64, rot=64, dtype="bf16",
             weights="bf16", pairs="halves", fused=True, layout="bshd", positions=4096),
        # a prompt: queries and keys out of one projection's output, written head by head for the attention behind
        dict(name="rotate_prompt_bf16", op="rotate", batch=1, tokens=8192, heads_q=32, heads_k=8, dim=128, rot=128, dtype="bf16",
             weights="bf16", pairs="halves", fused=True, layout="bhsd", positions=8192),
        # a training step of an encoder layer, hidden 1024, 16 x 512 tokens, 4 bits, groups of four heads
        dict(name="train_encoder_bf16", op="train", batch=16, tokens=512, heads_q=16, heads_k=16, dim=64, rot=64, dtype="bf16",
             weights="f32", pairs="halves", fused=False, layout="bhsd", positions=512, bits=4, group=256),
        # a vision transformer's 197 tokens in fp32, 2 bits, neighbouring elements as pairs, groups of half a head
        dict(name="train_vit_f32", op="train", batch=64, tokens=197, heads_q=16, heads_k=16, dim=64, rot=64, dtype="f32",
             weights="f32", pairs="neighbours", fused=False, layout="bshd", positions=197, bits=2, group=32),
        # heads of 80 of which 32 elements are rotated, one key head, nothing compressed: the backward pass reads q and k
        dict(name="train_dim80_bf16", op="train", batch=3, tokens=1021, heads_q=12, heads_k=1, dim=80, rot=32, dtype="bf16",
             weights="bf16", pairs="halves", fused=True, layout="bshd", positions=2048, bits=32, group=0),
        # the largest step: 16 x 2048 tokens, 32 query and 8 key heads of 128, 4 bits, a group a head
        dict(name="train_long_bf16", op="train", batch=16, tokens=2048, heads_q=32, heads_k=8, dim=128, rot=128, dtype="bf16",
             weights="bf16", pairs="halves", fused=True, layout="bshd", positions=4096, bits=4, group=128),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _lanes(dim):
    return 1 << max(0, (dim // 8 - 1).bit_length())


def _groups(dim, *heads):
    """Group sizes a context of such heads can have: a power of two that divides a head, or 1, 2, 4, ... whole heads;
    whole ones in a token."""
    sizes = [g for g in (32, 64, 128, 256, 512) if dim % g == 0]
    sizes += [dim << j for j in range(6) if (dim << j) % 32 == 0 and _lanes(dim) << j <= 64]
    return sorted({g for g in sizes if all(h * dim % g == 0 for h in heads)})


def draw(rng):
    dtype = rng.choice(("f32", "bf16"))
    if rng.random() < 0.45:
        case = dict(op=rng.choice(("norm", "clip", "clip", "clip_by")), dtype=dtype, kind=rng.choice((2, 2, 0)),
                    flat=rng.random() < 0.3)
        if rng.random() < 0.5:
            case.update(set="encoder", layers=rng.randint(1, 24), hidden=8 * _log_uniform(rng, 16, 120))
        else:                           # from one tensor to hundreds, of all sizes, odd ones too
            case.update(set="any", tensors=_log_uniform(rng, 1, 700), largest=_log_uniform(rng, 1000, 4_000_000),
                        sizes=rng.randrange(1 << 30))
        if case["op"] != "norm":
            case.update(share=math.exp(rng.uniform(-3, 1)), place=rng.choice(("in", "out")))
            if case["place"] == "in":   # below the bound, so that repeated passes see the same gradients
                case["share"] += 2.5
        return case
    while True:
        dim = rng.choice((64, 128, 64, 128, 256, 8 * rng.randint(2, 32), 512))
        kv = rng.choice((1, 2, 4, 8, 16, rng.randint(1, 12)))
        q = kv * rng.choice((1, 1, 2, 4, 8))
        tokens = _log_uniform(rng, 1, 8192)
        batch = _log_uniform(rng, 1, 256)
        if batch * tokens * (q + kv) * dim * SIZE[dtype] <= LARGEST:
            break
    rot = rng.choice((dim // 16 * 16, dim // 16 * 16, 16 * rng.randint(0, dim // 16)))
    case = dict(op=rng.choice(("rotate", "train", "train")), batch=batch, tokens=tokens, heads_q=q, heads_k=kv, dim=dim, rot=rot,
                dtype=dtype, weights=rng.choice(("f32", dtype, "none")), pairs=rng.choice(("halves", "neighbours")),
                fused=rng.random() < 0.5, layout=rng.choice(("bshd", "bhsd")), positions=tokens + rng.choice((0, 1, 777)))
    if case["op"] == "train":
        fit = _groups(dim, q, kv)
        case.update(bits=rng.choice((1, 2, 4, 8, 32)) if fit else 32)
        case.update(group=rng.choice(fit) if case["bits"] != 32 else 0)
    return case


# --------------------------------------------------------------- gradient lists
def _resnet50():
    sizes, cin = [64 * 3 * 49, 64, 64], 64
    for w, blocks in ((64, 3), (128, 4), (256, 6), (512, 3)):
        for b in range(blocks):
            sizes += [cin * w, w, w, w * w * 9, w, w, w * 4 * w, 4 * w, 4 * w]
            if b == 0:
                sizes += [cin * 4 * w, 4 * w, 4 * w]
            cin = 4 * w
    return sizes + [cin * 1000, 1000]


def _encoder(layers, h):
    layer = [h * h, h] * 4 + [4 * h * h, 4 * h, 4 * h * h, h] + [h] * 4
    return layer * layers


def _sizes(case):
    if case["set"] == "gcn":
        return [128 * 256, 256, 256 * 256, 256, 256 * 40, 40]
    if case["set"] == "resnet50":
        return _resnet50()
    if case["set"] == "vit_large":
        return [768 * 1024, 1024, 197 * 1024, 1024] + _encoder(24, 1024) + [1024, 1024, 1000 * 1024, 1000]
    if case["set"] == "encoder":
        return _encoder(case["layers"], case["hidden"])
    rng = np.random.default_rng(case["sizes"])
    sizes = np.exp(rng.uniform(0, math.log(case["largest"]), case["tensors"])).astype(np.int64)
    return [int(n) for n in np.minimum(sizes, 250_000_000 // case["tensors"])]


def _gradients(case, seed):
    """Gradients whose scale varies from tensor to tensor, and their norm."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 11)
    scales = np.exp(np.random.default_rng(seed).normal(-6.0, 1.0, len(_sizes(case))))
    out = [torch.randn(n, device=DEV, generator=g).mul_(float(s)).to(DTYPES[case["dtype"]]) for n, s in zip(_sizes(case), scales)]
    if case["kind"] == 2:
        return out, torch.stack([(t.double() ** 2).sum() for t in out]).sum().sqrt().item()
    return out, torch.stack([t.abs().max() for t in out]).max().item()


def _buffer(case):
    """A zeroed buffer for all of a list's tensors, and the slices: on 256 bytes each, or one element apart."""
    sizes = _sizes(case)
    step = 1 if case.get("flat") else 256 // SIZE[case["dtype"]]
    starts, at = [], step
    for n in sizes:
        starts.append(at)
        at = (at + n) // step * step + step
    buf = torch.zeros(at, dtype=DTYPES[case["dtype"]], device=DEV)
    return buf, [buf[o:o + n] for o, n in zip(starts, sizes)]


def _prepare_gradients(case, seed):
    values, norm_of = _gradients(case, seed)
    whole, g = _buffer(case)
    for t, v in zip(g, values):
        t.copy_(v)
    s = dict(op=case["op"], kind=case["kind"], g=g, outs=None, whole=whole)
    if case["op"] != "norm":
        s["max_norm"] = case["share"] * norm_of
        if case["place"] == "out":
            s["whole"], s["outs"] = _buffer(case)
    if case["op"] == "clip_by":
        s["norm"] = torch.full((1,), RANKS * norm_of, dtype=torch.float64, device=DEV)
    if own:
        import paper_2206_11357_amd as gact
        s["bufs"] = gact.make_grad_bufs(g, s["outs"])
        s["ws"] = torch.empty(gact.gact_grad_norm_workspace_bytes(len(g)), dtype=torch.uint8, device=DEV)
    return s


def _run_gradients(s):
    if own:
        import paper_2206_11357_amd as gact
        kind = 2.0 if s["kind"] == 2 else math.inf
        if s["op"] == "norm":
            return gact.gact_grad_norm(s["g"], kind, workspace=s["ws"], bufs=s["bufs"])
        if s["op"] == "clip_by":
            gact.gact_grad_clip_by(s["g"], s["max_norm"], s["norm"], s["outs"], workspace=s["ws"], bufs=s["bufs"])
            return s["whole"]
        return gact.gact_grad_clip(s["g"], s["max_norm"], kind, s["outs"], workspace=s["ws"], bufs=s["bufs"]), s["whole"]
    norm = s.get("norm")
    if norm is None and s["kind"] == 2:     # a sum over up to hundreds of millions of elements
        norm = torch.stack([t.double().square_().sum() for t in s["g"]]).sum().sqrt().reshape(1)
    elif norm is None:
        norm = torch.stack([t.abs().max() for t in s["g"]]).max().double().reshape(1)
    if s["op"] == "norm":
        return norm
    c = (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
    if s["outs"] is None:
        for t in s["g"]:
            t.copy_(t.float() * c)
    else:
        for t, o in zip(s["g"], s["outs"]):
            o.copy_(t.float() * c)
    return s["whole"] if s["op"] == "clip_by" else (norm, s["whole"])


def _exact_gradients(case, seed):
    g, norm_of = _gradients(case, seed)
    if case["op"] == "clip_by":
        norm = torch.full((1,), RANKS * norm_of, dtype=torch.float64, device=DEV)
    elif case["kind"] == 2:
        norm = torch.sqrt(sum((t.double() ** 2).sum() for t in g)).reshape(1)
    else:
        norm = torch.tensor([max(float(t.double().abs().max()) for t in g)], dtype=torch.float64, device=DEV)
    if case["op"] == "norm":
        return norm
    c = min(1.0, case["share"] * norm_of / (float(norm) + 1e-6))
    whole, parts = _buffer(case)
    whole = whole.double()
    for t, part in zip(g, parts):
        whole[part.storage_offset():part.storage_offset() + t.numel()] = t.double() * c
    return whole if case["op"] == "clip_by" else (norm, whole)


# ------------------------------------------------------------- queries and keys
def _heads(case, seed):
    B, S, Hq, Hk, D, R = (case[k] for k in ("batch", "tokens", "heads_q", "heads_k", "dim", "rot"))
    dt = DTYPES[case["dtype"]]
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 6007 + 5)

    def normal(*shape):
        return torch.randn(*shape, device=DEV, generator=gen)
    if case["fused"]:                   # one projection's output holds queries, keys and values of a token side by side
        x = normal(B, S, Hq + 2 * Hk, D)
        x *= torch.exp(normal(D) * 0.5)
        x = x.to(dt)
        q, k = x[:, :, :Hq], x[:, :, Hq:Hq + Hk]
    else:
        q, k = (normal(B, S, H, D).mul_(1.5).to(dt) for H in (Hq, Hk))
    w = [None, None]
    if case["weights"] != "none":
        w = [normal(D).mul_(0.3).add_(1.0).to(DTYPES[case["weights"]]) for _ in range(2)]
    angle = torch.arange(case["positions"], device=DEV, dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(0, R, 2, device=DEV, dtype=torch.float64) / max(R, 1))
    first = torch.randint(0, case["positions"] - S + 1, (B, 1), device=DEV, generator=gen)
    s = dict(q=q, k=k, wq=w[0], wk=w[1], cos=angle.cos().float(), sin=angle.sin().float(),
             positions=(first + torch.arange(S, device=DEV)).reshape(-1), halves=case["pairs"] == "halves", rot=R,
             layout=case["layout"])
    if case["op"] == "train":
        s.update(bits=case["bits"], group=case["group"], seeds=(2 * seed + 1, 2 * seed + 2))
        s["dy"] = []
        for H in (Hq, Hk):              # as the attention's backward pass leaves it
            d = normal(B, H, S, D).transpose(1, 2) if case["layout"] == "bhsd" else normal(B, S, H, D)
            s["dy"].append(d.mul_(0.1).to(dt))
    return s


def _empty_like_layout(x, layout):
    B, S, H, D = x.shape
    if layout == "bhsd":
        return torch.empty(B, H, S, D, dtype=x.dtype, device=x.device).transpose(1, 2)
    return torch.empty(B, S, H, D, dtype=x.dtype, device=x.device)


def _prepare_heads(case, seed):
    s = _heads(case, seed)
    s["op"] = case["op"]
    if own and case["op"] == "rotate" and case["tokens"] == 1:      # a generating loop keeps its buffers and its call
        import paper_2206_11357_amd as gact
        s["out"] = tuple(_empty_like_layout(x, s["layout"]) for x in (s["q"], s["k"]))
        s["call"] = gact.prepare_head_norm_rotate(s["q"], s["k"], s["cos"], s["sin"], s["wq"], s["wk"], s["positions"], EPS,
                                                  not s["halves"], out=s["out"])
    return s


def _run_heads(s):
    if not own:
        return _plain_heads(s)
    import paper_2206_11357_amd as gact
    if "call" in s:
        s["call"](torch.cuda.current_stream().cuda_stream)
        return s["out"]
    out = tuple(_empty_like_layout(x, s["layout"]) for x in (s["q"], s["k"]))
    args = (s["cos"], s["sin"], s["wq"], s["wk"], s["positions"])
    if s["op"] == "rotate":
        return gact.gact_head_norm_rotate(s["q"], s["k"], *args, eps=EPS, interleaved=not s["halves"], out=out)
    context = tuple(gact.make_head_context(x, s["bits"], s["group"], seed) for x, seed in zip((s["q"], s["k"]), s["seeds"]))
    gact.gact_head_norm_rotate(s["q"], s["k"], *args, eps=EPS, interleaved=not s["halves"], out=out, context=context)
    x = (s["q"], s["k"]) if s["bits"] == 32 else None
    grads = gact.gact_head_norm_rotate_backward(*s["dy"], *args, context=context, x=x, interleaved=not s["halves"])
    return list(out) + [t for t in grads if t is not None]


def _plain_rotate(n, cos, sin, rot, halves, back=False):
    """Pairs of the first `rot` elements turned by the angle (or back)."""
    if rot == 0:
        return n
    c, s = cos[:, None], (-sin if back else sin)[:, None]
    if halves:
        a, b = n[..., :rot // 2], n[..., rot // 2:rot]
        turned = torch.cat((a * c - b * s, b * c + a * s), -1)
    else:
        a, b = n[..., 0:rot:2], n[..., 1:rot:2]
        turned = torch.stack((a * c - b * s, b * c + a * s), -1).flatten(-2)
    return torch.cat((turned, n[..., rot:]), -1)


def _plain_noise(blocks, seed):
    """Philox4x32-10 of counters 0 .. blocks - 1, eight 16-bit values each, as numbers in (0, 1)."""
    c = [torch.arange(blocks, device=DEV, dtype=torch.int64)] + [torch.zeros(blocks, device=DEV, dtype=torch.int64) for _ in range(3)]
    k0, k1, low = seed & 0xFFFFFFFF, seed >> 32, 0xFFFFFFFF
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57        # modulo 2^64
        c = [((p1 >> 32) & low) ^ c[1] ^ k0, p1 & low, ((p0 >> 32) & low) ^ c[3] ^ k1, p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    slots = torch.stack([h for w in c for h in (w & 0xFFFF, w >> 16)], -1)
    return (slots.reshape(-1).float() + 0.5) / 65536.0


def _plain_context(x, group, bits, seed):
    """x after the quantizer and back, in 32 bits."""
    v = x.reshape(-1, group)
    mn = v.amin(1, keepdim=True) + 0.0
    rng = v.amax(1, keepdim=True) - mn
    flat = rng < 2.0 ** -100
    top = torch.full_like(rng, 2 ** bits - 1)       # a tensor: by a plain number torch divides with its reciprocal
    inv, step = (top / rng).masked_fill(flat, 0.0), (rng / top).masked_fill(flat, 0.0)
    t = (v - mn) * inv
    f = t.floor()
    u = _plain_noise(x.numel() // 8, seed).view_as(v)
    q = (f + (u < t - f)).clamp_(max=2.0 ** bits - 1)
    return (q * step + mn).view_as(x)


def _plain_heads(s):
    outs, grads, weights = [], [], []
    for j, (x, w) in enumerate(((s["q"], s["wq"]), (s["k"], s["wk"]))):
        B, S, H, D = x.shape
        xf = x.reshape(B * S, H, D).float()
        cos, sin = s["cos"][s["positions"]], s["sin"][s["positions"]]
        r = 1.0 / torch.sqrt((xf * xf).mean(-1, keepdim=True) + EPS)
        n = xf * r
        if w is not None:
            n = n * w.float()
        y = _empty_like_layout(x, s["layout"])
        y.copy_(_plain_rotate(n, cos, sin, s["rot"], s["halves"]).view(B, S, H, D))
        outs.append(y)
        if s["op"] == "rotate":
            continue
        if s["bits"] != 32:
            xf = _plain_context(xf, s["group"], s["bits"], s["seeds"][j])
        dn = _plain_rotate(s["dy"][j].reshape(B * S, H, D).float(), cos, sin, s["rot"], s["halves"], back=True)
        xr = xf * r
        if w is not None:
            weights.append((dn * xr).sum((0, 1)).to(w.dtype))
            dn = dn * w.float()
        grads.append((r * (dn - xr * (dn * xr).mean(-1, keepdim=True))).to(x.dtype).view(B, S, H, D))
    return outs + grads + weights


def _exact_noise(blocks, seed):
    c = np.zeros((4, blocks), dtype=np.uint64)
    c[0] = np.arange(blocks, dtype=np.uint64)
    key = [np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = np.stack(((b >> half) ^ c[1] ^ key[0], b & low, (a >> half) ^ c[3] ^ key[1], a & low))
        key = [(key[0] + np.uint64(0x9E3779B9)) & low, (key[1] + np.uint64(0xBB67AE85)) & low]
    words = np.ascontiguousarray(c.T.astype("<u4")).view("<u2")
    return words.reshape(-1)


def _exact_context(x, group, bits, seed):
    """Codes by the quantizer's own arithmetic, each step rounded to 32 bits; the values they stand for in 64."""
    v = x.astype(np.float32).reshape(-1, group)
    top = np.float32(2 ** bits - 1)
    mn = v.min(1, keepdims=True) + np.float32(0)
    rng = v.max(1, keepdims=True) - mn
    with np.errstate(divide="ignore"):
        inv, step = top / rng, rng / top
    small = rng < np.float32(2.0 ** -100)
    inv[small], step[small] = 0, 0
    t = (v - mn) * inv
    f = np.floor(t)
    u = (_exact_noise(x.size // 8, seed).astype(np.float32) + np.float32(0.5)) / np.float32(65536)
    q = np.minimum(f + (u.reshape(v.shape) < t - f), top)
    return (q.astype(np.float64) * step.astype(np.float64) + mn.astype(np.float64)).reshape(x.shape)


def _exact_heads(case, seed):
    if case["batch"] * case["tokens"] * (case["heads_q"] + case["heads_k"]) * case["dim"] > 60_000_000:
        return None
    s = _heads(case, seed)
    R, D = case["rot"], case["dim"]
    i = torch.arange(R // 2, device=DEV)
    a, b = (i, i + R // 2) if s["halves"] else (2 * i, 2 * i + 1)
    outs, grads, weights = [], [], []
    for j, (x, w) in enumerate(((s["q"], s["wq"]), (s["k"], s["wk"]))):
        B, S, H, _ = x.shape
        p = s["positions"].view(B, S)
        c, sn = s["cos"].double()[p][:, :, None], s["sin"].double()[p][:, :, None]
        v = x.double()
        r = ((v ** 2).sum(-1, keepdim=True) / D + EPS) ** -0.5
        wd = torch.ones(D, dtype=torch.float64, device=DEV) if w is None else w.double()
        y = v * r * wd
        na, nb = y[..., a], y[..., b]
        y[..., a], y[..., b] = na * c - nb * sn, nb * c + na * sn
        outs.append(y)
        if case["op"] == "rotate":
            continue
        if case["bits"] != 32:
            flat = x.reshape(-1).float().cpu().numpy()
            v = torch.from_numpy(_exact_context(flat, case["group"], case["bits"], s["seeds"][j])).to(DEV).view(B, S, H, D)
        dn = s["dy"][j].double()
        da, db = dn[..., a], dn[..., b]
        dn[..., a], dn[..., b] = da * c + db * sn, db * c - da * sn
        if w is not None:
            weights.append((dn * v * r).sum((0, 1, 2)))
        gr = dn * wd
        grads.append(r * gr - v * r ** 3 * ((gr * v).sum(-1, keepdim=True) / D))
    return outs + grads + weights


# ---------------------------------------------------------------------- the file
def prepare(case, seed):
    return (_prepare_heads if case["op"] in ("rotate", "train") else _prepare_gradients)(case, seed)


def run(state):
    return (_run_heads if state["op"] in ("rotate", "train") else _run_gradients)(state)


def exact(case, seed):
    return (_exact_heads if case["op"] in ("rotate", "train") else _exact_gradients)(case, seed)


def work(case):
    if case["op"] not in ("rotate", "train"):
        n, s = sum(_sizes(case)), SIZE[case["dtype"]]
        scaled = case["op"] != "norm" and (case["place"] == "out" or case["share"] < 1.0)
        if case["op"] == "clip_by" and case["place"] == "in":
            scaled = case["share"] < RANKS
            return {"bytes": n * s * 2 * int(scaled) + 8, "flops": n * int(scaled) + 1}
        return {"bytes": n * s * (1 + int(scaled)) + 8, "flops": n * (2 if case["op"] == "norm" else 3)}
    T = case["batch"] * case["tokens"]
    n, s = T * (case["heads_q"] + case["heads_k"]) * case["dim"], SIZE[case["dtype"]]
    tables = min(T, case["positions"]) * case["rot"] * 4 + 8 * T
    w = 0 if case["weights"] == "none" else 2 * case["dim"] * SIZE[case["weights"]]
    if case["op"] == "rotate":
        return {"bytes": 2 * n * s + tables + w, "flops": 7 * n}
    return {"bytes": 4 * n * s + tables + 2 * w, "flops": 20 * n}
