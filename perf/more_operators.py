"""Layers whose context is kept compressed and read as codes: the weight gradient
of a linear layer, and group normalisation with an activation, channels last.

A case is a dict of plain values.  ``prepare`` makes what a program has in hand
before the call, ``run`` is one pass through an operator: the package's calls
where ``own`` is true, else the same formulas in elementary torch operations.
``exact`` computes a case's outputs in 64 bits.

Formulas.  A context is x, flattened, in groups of G consecutive elements that
are rounded stochastically to `bits` bits (the quantizer of arXiv 2206.11357,
App. A.4, per group; every step in binary32): with mn, mx a group's minimum and
maximum, t = (x - mn) (2^bits - 1) / (mx - mn), q = floor(t) or one more if a
noise value in (0, 1) is below t - floor(t); x^ = q step + mn, rounded to x's
type.

Linear layer, y = x W^T + b, x [T, K], dy [T, N]:
    dW[n, k] = sum over t of dy[t, n] x^[t, k],   db[n] = sum over t of dy[t, n].

Group norm, x [B, P, C] with the C channels of a pixel consecutive, in H groups
of C / H channels; over a group's M = P C / H elements of a sample
    m = mean x,  r = 1 / sqrt(mean (x - m)^2 + eps),
    z = (x - m) r w + b,   y = act(z),   act(z) = z or z / (1 + exp(-z)).
Backward, n = (x^ - m) r with the forward pass's m and r and x^ in binary32, and
z from it:
    dz = dy act'(z),   g = dz w,   dx = r (g - mean g - n mean(g n)),
    dw = sum of dz n,   db = sum of dz   over samples and pixels.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
MOST_FLOPS = {"f32": 2 * 169343 * 256 * 256, "bf16": 2 * 32768 * 1024 * 4096}    # of a weight gradient
MOST_BYTES = 205_520_896                                                       # of one tensor of a norm


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # a classifier's head on a small last batch: one short product, where the launches count
        dict(name="weight_head_64_f32", op="weight", tokens=64, n=1000, k=1024, dtype="f32", weights="f32", bias=True, bits=4,
             group=256, spread=False),
        # a graph network's layer: few weights, 169,343 nodes to add over, 2 bits
        dict(name="weight_gcn_f32", op="weight", tokens=169343, n=256, k=256, dtype="f32", weights="f32", bias=True, bits=2,
             group=256, spread=False),
        # odd sizes throughout: three sequences of 1021 tokens, 47 classes, 200 features in groups that pass from row to row
        dict(name="weight_odd_bf16", op="weight", tokens=3 * 1021, n=47, k=200, dtype="bf16", weights="f32", bias=False, bits=1,
             group=96, spread=True),
        # a vision transformer's projection, 64 x 197 tokens, 8 bits, the gradient half of a wider one's columns
        dict(name="weight_vit_bf16", op="weight", tokens=64 * 197, n=1024, k=1024, dtype="bf16", weights="f32", bias=True, bits=8,
             group=128, spread=True),
        # the first layer of an encoder's feed-forward block, hidden 1024, 16 x 512 tokens, 4 bits
        dict(name="weight_ffn_bf16", op="weight", tokens=16 * 512, n=4096, k=1024, dtype="bf16", weights="bf16", bias=True, bits=4,
             group=256, spread=False),
        # the largest product: the second layer at 16 x 2048 tokens
        dict(name="weight_long_bf16", op="weight", tokens=16 * 2048, n=1024, k=4096, dtype="bf16", weights="bf16", bias=True, bits=4,
             group=256, spread=False),
        # inference on one small feature map: three short passes at most, the launches count
        dict(name="norm_small_bf16", op="norm", batch=1, pixels=64, channels=512, heads=32, act="silu", dtype="bf16", weights="bf16",
             wide=0),
        # inference on one large image: few channels, a group's sum over a million elements
        dict(name="norm_image_bf16", op="norm", batch=1, pixels=512 * 512, channels=128, heads=32, act="silu", dtype="bf16",
             weights="f32", wide=0),
        # a training step at 32 x 32 pixels, 4 bits
        dict(name="step_silu_bf16", op="step", batch=32, pixels=1024, channels=512, heads=32, act="silu", dtype="bf16", weights="f32",
             wide=0, bits=4, group=256),
        # a CNN's largest map, 64 x 56 x 56 x 256, norm alone, 2 bits
        dict(name="step_cnn_f32", op="step", batch=64, pixels=3136, channels=256, heads=32, act="none", dtype="f32", weights="f32",
             wide=0, bits=2, group=256),
        # odd sizes: 13 x 17 pixels, 104 channels, groups of 8 channels, context groups that end inside a pixel and a sample
        dict(name="step_odd_f32", op="step", batch=3, pixels=13 * 17, channels=104, heads=13, act="silu", dtype="f32", weights="f32",
             wide=0, bits=8, group=64),
        # part of a concatenated map's channels, nothing compressed: the backward pass reads x
        dict(name="step_slice_bf16", op="step", batch=16, pixels=2304, channels=320, heads=32, act="silu", dtype="bf16",
             weights="bf16", wide=320, bits=32, group=0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(("f32", "bf16", "bf16"))
    weights = rng.choice(("f32", dtype))
    bits = rng.choice((1, 2, 4, 8))
    if rng.random() < 0.5:
        while True:
            T, n = _log_uniform(rng, 1, 170_000), _log_uniform(rng, 1, 8192)
            k = rng.choice((8, 1)) * _log_uniform(rng, 1, 1024)
            if 2 * T * n * k <= MOST_FLOPS[dtype] and T * max(n, k) <= 1 << 28:
                break
        return dict(op="weight", tokens=T, n=n, k=k, dtype=dtype, weights=weights, bias=rng.random() < 0.5, bits=bits,
                    group=rng.choice((32, 64, 128, 256, 256, 512, 1024, 32 * rng.randint(1, 32))), spread=rng.random() < 0.3)
    while True:
        channels = 8 * _log_uniform(rng, 1, 256)
        heads = rng.choice([h for h in (1, 2, 4, 8, 16, 32, channels // 8, channels) if channels % h == 0])
        batch, pixels = _log_uniform(rng, 1, 256), _log_uniform(rng, 1, 270_000)
        # a group of one element has no spread; a handful has one that is all rounding now and then
        if batch * pixels * channels * SIZE[dtype] <= MOST_BYTES and pixels * channels // heads >= 16:
            break
    case = dict(op=rng.choice(("norm", "step", "step")), batch=batch, pixels=pixels, channels=channels, heads=heads,
                act=rng.choice(("none", "silu", "silu")), dtype=dtype, weights=rng.choice((weights, weights, "none")),
                wide=rng.choice((0, 0, 8 * rng.randint(1, 40))))
    if case["op"] == "step":
        case.update(bits=rng.choice((bits, bits, 32)), group=rng.choice((32, 64, 128, 256, 512)))
    return case


# ------------------------------------------------------- weights' gradients
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 9176 + 23)
    return g


def _weight_inputs(case, seed):
    T, N, K, G, bits = (case[f] for f in ("tokens", "n", "k", "group", "bits"))
    dt, gen = DTYPES[case["dtype"]], _generator(seed)

    def normal(*shape):
        return torch.randn(*shape, device=DEV, generator=gen)
    # the layer's input: channels of different sizes, a few values far out; compressed in the forward pass
    x = (normal(T, K) * torch.exp(0.5 * normal(K)) + 0.3 * normal(K)).to(dt).float().reshape(-1)
    ends = -x.numel() % G
    v = torch.cat((x, x[-1:].expand(ends))).view(-1, G)
    mn, top = v.amin(1, keepdim=True), 2 ** bits - 1
    step = (v.amax(1, keepdim=True) - mn) / torch.full_like(mn, top)
    q = ((v - mn) / step.clamp(min=1e-30) + torch.rand(v.shape, device=DEV, generator=gen)).floor().clamp(0, top)
    q = q.to(torch.uint8).view(-1)
    q[x.numel():] = 0
    per = 8 // bits
    q = torch.cat((q, q.new_zeros(-q.numel() % (16 * per)))).view(-1, per)
    packed = torch.zeros(q.shape[0], dtype=torch.uint8, device=DEV)
    for j in range(per):
        packed |= q[:, j] << (j * bits)
    packed = packed[:(T * K * bits + 127) // 128 * 16].contiguous()
    columns = 2 * N if case["spread"] else N
    dy = (normal(T, columns) * 0.02).to(dt)
    return dict(op="weight", dy=dy[:, columns - N:], packed=packed, gmin=mn.view(-1), gscale=step.view(-1), T=T, N=N, K=K, G=G,
                bits=bits, w=DTYPES[case["weights"]], bias=case["bias"])


def _run_weight(s):
    if own:
        import paper_2206_11357_amd as gact
        dw, db = gact.gact_linear_weight_grad(s["dy"], s["packed"], s["gmin"], s["gscale"], s["K"], s["G"], s["bits"],
                                              w_dtype=s["w"], bias=s["bias"])
        return (dw, db) if s["bias"] else dw
    n, bits, dy = s["T"] * s["K"], s["bits"], s["dy"]
    shifts = torch.arange(0, 8, bits, device=DEV, dtype=torch.uint8)
    q = ((s["packed"][:, None] >> shifts) & (2 ** bits - 1)).view(-1)[:n].float()
    ends = -n % s["G"]
    q = torch.cat((q, q.new_zeros(ends))).view(-1, s["G"])
    x = (q * s["gscale"][:, None] + s["gmin"][:, None]).view(-1)[:n].view(s["T"], s["K"]).to(dy.dtype).float()
    dw = (dy.float().t() @ x).to(s["w"])
    return (dw, dy.float().sum(0).to(s["w"])) if s["bias"] else dw


def _exact_weight(case, seed):
    s = _weight_inputs(case, seed)
    T, N, K, bits = s["T"], s["N"], s["K"], s["bits"]
    dw = torch.zeros(N, K, dtype=torch.float64, device=DEV)
    # rows at a time; an element's code by its place in the bit string; products and sums of two binary32 numbers, rounded from 64
    # bits to 32, are what 32 bits give
    rows = max(1, (1 << 24) // K)
    for t in range(0, T, rows):
        m = min(rows, T - t)
        i = torch.arange(t * K, (t + m) * K, device=DEV)
        q = (s["packed"][i * bits // 8].long() >> (i * bits % 8)) % (1 << bits)
        g = i // s["G"]
        x = ((q.double() * s["gscale"][g].double()).float().double() + s["gmin"][g].double()).float().to(s["dy"].dtype)
        dw += s["dy"][t:t + m].double().t() @ x.double().view(m, K)
    return (dw, s["dy"].double().sum(0)) if case["bias"] else dw


# ------------------------------------------------------------------ group norms
def _norm_inputs(case, seed):
    B, P, C = case["batch"], case["pixels"], case["channels"]
    dt, gen = DTYPES[case["dtype"]], _generator(seed)

    def normal(*shape):
        return torch.randn(*shape, device=DEV, generator=gen)

    def map_of(scale, shift):           # possibly the first channels of a wider one
        v = normal(B, P, C + case["wide"])
        v[..., :C].mul_(scale).add_(shift)
        return v.to(dt)[..., :C]
    x = map_of(torch.exp(0.3 * normal(C)), 0.5 * normal(C))
    w, b = (None, None) if case["weights"] == "none" else ((1.0 + 0.2 * normal(C)).to(DTYPES[case["weights"]]),
                                                           (0.2 * normal(C)).to(DTYPES[case["weights"]]))
    s = dict(op=case["op"], x=x, w=w, b=b, H=case["heads"], act=case["act"])
    if case["op"] == "step":
        s.update(dy=map_of(torch.full((C,), 0.1, device=DEV), 0.0), bits=case["bits"], group=case["group"], seed=seed * 3 + 1)
    return s


def _prepare_norm(case, seed):
    s = _norm_inputs(case, seed)
    if own and case["op"] == "norm" and case["batch"] * case["pixels"] <= 4096:     # a serving loop keeps its buffers and its call
        import paper_2206_11357_amd as gact
        s["out"] = torch.empty(s["x"].shape, dtype=s["x"].dtype, device=DEV)
        s["call"] = gact.prepare_group_norm(s["x"], s["H"], s["w"], s["b"], EPS, s["act"], out=s["out"])
    return s


def _run_norm(s):
    if not own:
        return _plain_norm(s)
    import paper_2206_11357_amd as gact
    if "call" in s:
        s["call"](torch.cuda.current_stream().cuda_stream)
        return s["out"]
    if s["op"] == "norm":
        return gact.gact_group_norm(s["x"], s["H"], s["w"], s["b"], EPS, s["act"])
    context = gact.make_group_norm_context(s["x"], s["H"], s["bits"], s["group"], s["seed"])
    y = gact.gact_group_norm(s["x"], s["H"], s["w"], s["b"], EPS, s["act"], context=context)
    dx, dw, db = gact.gact_group_norm_backward(s["dy"], s["H"], s["w"], s["b"], s["act"], context=context,
                                               x=s["x"] if s["bits"] == 32 else None)
    return (y, dx) if dw is None else (y, dx, dw, db)


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
    """x after the quantizer and back, in 32 bits; the last group may be short."""
    n, ends = x.numel(), -x.numel() % group
    v = torch.cat((x.reshape(-1), x.reshape(-1)[-1:].expand(ends))).view(-1, group)
    mn = v.amin(1, keepdim=True) + 0.0
    rng = v.amax(1, keepdim=True) - mn
    flat = rng < 2.0 ** -100
    top = torch.full_like(rng, 2 ** bits - 1)       # a tensor: by a plain number torch divides with its reciprocal
    inv, step = (top / rng).masked_fill(flat, 0.0), (rng / top).masked_fill(flat, 0.0)
    t = (v - mn) * inv
    f = t.floor()
    q = (f + (_plain_noise(v.numel() // 8, seed).view_as(v) < t - f)).clamp_(max=2.0 ** bits - 1)
    return (q * step + mn).view(-1)[:n].view_as(x)


def _plain_norm(s):
    x, w, b, H = s["x"], s["w"], s["b"], s["H"]
    B, P, C = x.shape
    shape, channels = (B, P, H, C // H), (1, 1, H, C // H)
    xf = x.float().reshape(shape)
    w = 1.0 if w is None else w.float().view(channels)
    b = 0.0 if b is None else b.float().view(channels)
    # sums over up to a million elements: 64 bits
    m = xf.double().mean((1, 3), keepdim=True).float()
    r = (1.0 / torch.sqrt((xf - m).square().double().mean((1, 3), keepdim=True) + EPS)).float()
    z = (xf - m) * r * w + b
    y = (z / (1.0 + torch.exp(-z)) if s["act"] == "silu" else z).to(x.dtype).view(B, P, C)
    if s["op"] == "norm":
        return y
    if s["bits"] != 32:
        xf = _plain_context(xf, s["group"], s["bits"], s["seed"])
    n = (xf - m) * r
    dz = s["dy"].float().reshape(shape)
    if s["act"] == "silu":
        z = n * w + b
        p = 1.0 / (1.0 + torch.exp(-z))
        dz = dz * (p * (1.0 + z * (1.0 - p)))
    g = dz * w
    m1 = g.double().mean((1, 3), keepdim=True).float()
    m2 = (g * n).double().mean((1, 3), keepdim=True).float()
    dx = (r * (g - m1 - n * m2)).to(x.dtype).view(B, P, C)
    if s["w"] is None:
        return y, dx
    dw, db = ((t.double().sum((0, 1)).view(C)).to(s["w"].dtype) for t in (dz * n, dz))
    return y, dx, dw, db


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
    n = x.size
    v = np.full((n + group - 1) // group * group, x[-1], dtype=np.float32)
    v[:n] = x
    v = v.reshape(-1, group)
    top = np.float32(2 ** bits - 1)
    mn = v.min(1, keepdims=True) + np.float32(0)
    rng = v.max(1, keepdims=True) - mn
    with np.errstate(divide="ignore"):
        inv, step = top / rng, rng / top
    small = rng < np.float32(2.0 ** -100)
    inv[small], step[small] = 0, 0
    t = (v - mn) * inv
    f = np.floor(t)
    u = (_exact_noise(v.size // 8, seed).astype(np.float32) + np.float32(0.5)) / np.float32(65536)
    q = np.minimum(f + (u.reshape(v.shape) < t - f), top)
    return (q.astype(np.float64) * step.astype(np.float64) + mn.astype(np.float64)).reshape(-1)[:n]


def _exact_norm(case, seed):
    B, P, C, H = (case[f] for f in ("batch", "pixels", "channels", "heads"))
    if case["op"] == "step" and case["bits"] != 32 and B * P * C > 60_000_000:
        return None
    s = _norm_inputs(case, seed)
    one = torch.ones(C, dtype=torch.float64, device=DEV)
    w, b = (one, 0 * one) if s["w"] is None else (s["w"].double(), s["b"].double())
    of = torch.arange(C, device=DEV) // (C // H)            # a channel's group
    x = s["x"].double()
    M = P * (C // H)

    def mean(v):                        # over a group's elements, for each channel
        sums = torch.zeros(B, H, dtype=torch.float64, device=DEV).index_add_(1, of, v.sum(1))
        return (sums / M)[:, None, of]
    m = mean(x)
    r = (mean((x - m) ** 2) + EPS) ** -0.5
    z = (x - m) * r * w + b
    y = z * torch.sigmoid(z) if s["act"] == "silu" else z
    if case["op"] == "norm":
        return y
    if case["bits"] != 32:
        flat = s["x"].float().cpu().numpy().reshape(-1)
        x = torch.from_numpy(_exact_context(flat, case["group"], case["bits"], s["seed"])).to(DEV).view(B, P, C)
    n = (x - m) * r
    dz = s["dy"].double()
    if s["act"] == "silu":
        z = n * w + b
        sg = torch.sigmoid(z)
        dz = dz * (sg + z * sg * torch.sigmoid(-z))
    dx = r * (dz * w - mean(dz * w) - n * mean(dz * w * n))
    return (y, dx) if s["w"] is None else (y, dx, (dz * n).sum((0, 1)), dz.sum((0, 1)))


# ---------------------------------------------------------------------- the file
def prepare(case, seed):
    return _weight_inputs(case, seed) if case["op"] == "weight" else _prepare_norm(case, seed)


def run(state):
    return _run_weight(state) if state["op"] == "weight" else _run_norm(state)


def exact(case, seed):
    return _exact_weight(case, seed) if case["op"] == "weight" else _exact_norm(case, seed)


def work(case):
    s = SIZE[case["dtype"]]
    if case["op"] == "weight":
        T, N, K, G, bits = (case[f] for f in ("tokens", "n", "k", "group", "bits"))
        weights = (N * K + N * int(case["bias"])) * SIZE[case["weights"]]
        return {"bytes": T * N * s + T * K * bits // 8 + (T * K + G - 1) // G * 8 + weights, "flops": 2 * T * N * K}
    n, C = case["batch"] * case["pixels"] * case["channels"], case["channels"]
    w = 0 if case["weights"] == "none" else 2 * C * SIZE[case["weights"]]
    if case["op"] == "norm":
        return {"bytes": 2 * n * s + w, "flops": 10 * n}
    return {"bytes": 4 * n * s + 2 * w, "flops": 30 * n}
