"""The 8-bit projections of a transformer that runs beside the decode, as measurable cases.

The streaming loop decodes latents that a generator makes in every tick.  Its layers are, with the decode, all that the GPU
does: a root-mean-square norm with the residual's addition, products with fixed weights, a gate, products again, and at the
end a product whose output is the latent that the decode reads.  These are their operators with operands in e4m3 and one fp32 scale
for each block of 128 along the channels (weights: for each 128 x 128 block):

  kind "norm"      h = x + residual;  y = h / sqrt(mean(h^2) + eps) * weight;  y in 8 bits with its scales, and h
  kind "quantize"  y = x, or with `gated` y = silu(gate) * up of rows [gate | up];  y in 8 bits with its scales
  kind "weights"   a weight matrix in 8 bits with a scale for each 128 x 128 block
  kind "matmul"    out[m][n] = bias[n] + sum over blocks b of a_scale[b][m] w_scale[n / 128][b] sum over k in b of a[m][k] w[n][k];
                   rows of n values, or with `n_frames` the latent [clip, n, frame] of rows m = clip * n_frames + frame

Scales of rows are [blocks, rows], scales of weights [blocks of rows, blocks of columns].  A block's scale is max(|y|, 2^-100) / 448, its
values are e4m3(y / scale).

The other keys of a case: rows, channels (of the norm and the rows that are quantised), n and k (of weights and products; the product's
rows are `rows`), dtype (of the input; the product's: of the output), residual, gated, bias, n_frames, and `tight` (rows of 8-bit operands
follow each other without a gap; else each starts at a multiple of 16 bytes, as the quantising operators leave them).
"""
import math

import torch

own = False

DEV = "cuda:0"
BLOCK = 128
LARGEST = 448.0          # the largest e4m3 value
FLOOR = 2.0 ** -100      # a block of zeros has the scale of this
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
MOST_PRODUCT = 12000 * 11264 * 2048
MOST_ELEMENTS = 12000 * 8192


def listed():
    return [
        # one new row, where only latency counts: a norm before a layer's product
        dict(name="norm_1", kind="norm", rows=1, channels=2048, dtype="bf16", residual=True),
        # a 60 s clip's 1500 rows with an odd number of channels, in 32 bits, nothing to add (a first layer)
        dict(name="norm_1500_odd_f32", kind="norm", rows=1500, channels=1111, dtype="f32", residual=False),
        # a ring of eight 60 s clips: the layer's whole batch
        dict(name="norm_12000", kind="norm", rows=12000, channels=2048, dtype="bf16", residual=True),
        # the gate of a feed-forward layer for a 3 s window of one clip, for a ring of eight clips of 60 s, and an attention's output
        dict(name="gate_75", kind="quantize", rows=75, channels=5632, dtype="bf16", gated=True),
        dict(name="gate_12000", kind="quantize", rows=12000, channels=5632, dtype="bf16", gated=True),
        # weights laid out at load or after an update: a layer's gate and up, and an odd matrix
        dict(name="weights_11264x2048", kind="weights", n=11264, k=2048, dtype="bf16"),
        dict(name="weights_517x1111_f32", kind="weights", n=517, k=1111, dtype="f32"),
        # one row, and one row for each of eight slots: the weights are read once and little is computed
        dict(name="matmul_1", kind="matmul", rows=1, n=2048, k=2048, dtype="bf16", bias=False, n_frames=0, tight=False),
        dict(name="matmul_8", kind="matmul", rows=8, n=11264, k=2048, dtype="bf16", bias=False, n_frames=0, tight=False),
        # the product that ends in the latent of four 15 s windows: 64 channels, frames fastest, with an odd number of channels before it
        dict(name="matmul_latent", kind="matmul", rows=1500, n=64, k=1111, dtype="f32", bias=True, n_frames=375, tight=True),
        # a 60 s clip through a feed-forward layer's second product
        dict(name="matmul_1500", kind="matmul", rows=1500, n=2048, k=5632, dtype="bf16", bias=True, n_frames=0, tight=False),
        # eight of them through its first
        dict(name="matmul_12000", kind="matmul", rows=12000, n=11264, k=2048, dtype="bf16", bias=False, n_frames=0, tight=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A number of channels: mostly a multiple of 64, else any."""
    v = _log_int(rng, lo, hi)
    return max(64, v // 64 * 64) if rng.random() < 0.6 else v


def draw(rng):
    kind = rng.choice(["norm", "norm", "quantize", "quantize", "weights", "matmul", "matmul", "matmul", "matmul"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "weights":
        return dict(kind=kind, n=_width(rng, 64, 12000), k=_width(rng, 64, 2048), dtype=dtype)
    if kind == "matmul":
        n, k = _width(rng, 64, 11264), _width(rng, 64, 8192)
        rows = _log_int(rng, 1, max(1, min(12000, MOST_PRODUCT // (n * k))))
        n_frames = 0
        if rng.random() < 0.2:
            clips = rng.choice([1, 2, 4])
            n_frames = max(1, rows // clips)
            rows = clips * n_frames
        return dict(kind=kind, rows=rows, n=n, k=k, dtype=dtype, bias=rng.random() < 0.5, n_frames=n_frames, tight=rng.random() < 0.3)
    channels = _width(rng, 64, 8192)
    rows = _log_int(rng, 1, min(12000, MOST_ELEMENTS // channels // (2 if dtype == "f32" else 1)))
    if kind == "norm":
        return dict(kind=kind, rows=rows, channels=channels, dtype=dtype, residual=rng.random() < 0.7)
    return dict(kind=kind, rows=rows, channels=channels, dtype=dtype, gated=rng.random() < 0.6)


def _blocks(n):
    return -(-n // BLOCK)


def _by_block(y):
    """[rows, channels] as [rows, blocks, 128], zeros behind the last channel."""
    pad = _blocks(y.shape[1]) * BLOCK - y.shape[1]
    return torch.nn.functional.pad(y, (0, pad)).view(y.shape[0], -1, BLOCK)


def _scaled_rows(y):
    """(y / scale [rows, channels], scale [blocks, rows]) of each row's blocks."""
    b = _by_block(y)
    scale = b.abs().amax(2).clamp_min(FLOOR) / LARGEST
    return (b / scale[:, :, None]).reshape(y.shape[0], -1)[:, :y.shape[1]], scale.t().contiguous()


def _scaled_weights(w):
    """(w / scale [n, k], scale [blocks of n, blocks of k]) of each 128 x 128 block."""
    n, k = w.shape
    b = torch.nn.functional.pad(w, (0, _blocks(k) * BLOCK - k, 0, _blocks(n) * BLOCK - n)).view(_blocks(n), BLOCK, _blocks(k), BLOCK)
    scale = b.abs().amax((1, 3)).clamp_min(FLOOR) / LARGEST
    return (b / scale[:, None, :, None]).reshape(_blocks(n) * BLOCK, -1)[:n, :k], scale


def _stored(q, tight):
    """An 8-bit operand as a user holds it: rows without a gap, or each at a multiple of 16 bytes."""
    q = q.to(torch.float8_e4m3fn)
    if tight:
        return q.contiguous()
    out = torch.zeros((q.shape[0], -(-q.shape[1] // 16) * 16), dtype=torch.uint8, device=q.device)
    out[:, :q.shape[1]] = q.view(torch.uint8)
    return out.view(torch.float8_e4m3fn)[:, :q.shape[1]]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)

    kind, dtype = case["kind"], DTYPES[case["dtype"]]
    s = dict(case=case, dtype=dtype)
    if kind == "norm":
        c = case["channels"]
        # a residual stream has a few channels that are much larger than the others
        loud = 1 + 20 * (torch.rand(c, generator=g, device=DEV) < 0.005).float()
        s["x"] = normal(case["rows"], c).mul_(0.5).to(dtype)
        s["residual"] = (normal(case["rows"], c) * loud).to(dtype) if case["residual"] else None
        s["weight"] = 1 + 0.2 * normal(c)
    elif kind == "quantize":
        s["x"] = normal(case["rows"], case["channels"] * (2 if case["gated"] else 1)).mul_(1.5).to(dtype)
    elif kind == "weights":
        s["w"] = (normal(case["n"], case["k"]) * case["k"] ** -0.5).to(dtype)
    else:
        q, scale = _scaled_rows(normal(case["rows"], case["k"]))
        s["a"], s["a_scale"] = _stored(q, case["tight"]), scale
        q, scale = _scaled_weights(normal(case["n"], case["k"]) * case["k"] ** -0.5)
        s["w"], s["w_scale"] = _stored(q, case["tight"]), scale
        s["bias"] = normal(case["n"]) if case["bias"] else None
    return s


def _product(s, to):
    """The product of the operands' values in the type `to`."""
    a, w = s["a"].to(to), s["w"].to(to)
    a *= s["a_scale"].t().to(to).repeat_interleave(BLOCK, 1)[:, :a.shape[1]]
    w *= s["w_scale"].to(to).repeat_interleave(BLOCK, 0)[:w.shape[0]].repeat_interleave(BLOCK, 1)[:, :w.shape[1]]
    out = a @ w.t()
    if s["bias"] is not None:
        out += s["bias"].to(to)
    frames = s["case"]["n_frames"]
    if frames:
        out = out.view(-1, frames, out.shape[1]).transpose(1, 2).contiguous()
    return out


def run(s):
    case, kind = s["case"], s["case"]["kind"]
    if own:
        import paper_2605_28657_amd as pa
        if kind == "norm":
            return pa.rms_norm_fp8(s["x"], s["weight"], EPS, residual=s["residual"])
        if kind == "quantize":
            return pa.quantize_fp8(s["x"], gated=case["gated"])
        if kind == "weights":
            return pa.quantize_weights_fp8(s["w"])
        return pa.matmul_fp8(s["a"], s["a_scale"], s["w"], s["w_scale"], bias=s["bias"], dtype=s["dtype"], n_frames=case["n_frames"])
    if kind == "norm":
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["weight"]
        q, scale = _scaled_rows(y)
        return q.to(torch.float8_e4m3fn), scale, h.to(s["dtype"]) if s["residual"] is not None else None
    if kind == "quantize":
        x = s["x"].float()
        if case["gated"]:
            gate, up = x.chunk(2, 1)
            x = gate / (1 + torch.exp(-gate)) * up
        q, scale = _scaled_rows(x)
        return q.to(torch.float8_e4m3fn), scale
    if kind == "weights":
        q, scale = _scaled_weights(s["w"].float())
        return q.to(torch.float8_e4m3fn), scale
    return _product(s, torch.float32).to(s["dtype"])


def exact(case, seed):
    """The 8-bit outputs as y / scale before it is rounded, everything from sums and quotients in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]

    def in_blocks(y, size):
        """Largest magnitude of each block of `size` rows by 128 columns, at every element and by block."""
        rows, cols = y.shape
        top = torch.zeros((-(-rows // size), _blocks(cols)), dtype=torch.float64, device=DEV)
        for b in range(top.shape[1]):
            part = y[:, b * BLOCK:(b + 1) * BLOCK].abs().amax(1)
            full = torch.zeros(top.shape[0] * size, dtype=torch.float64, device=DEV)
            full[:rows] = part
            top[:, b] = full.view(-1, size).amax(1)
        scale = torch.maximum(top, torch.tensor(FLOOR, dtype=torch.float64, device=DEV)) / LARGEST
        r = torch.arange(rows, device=DEV) // size
        c = torch.arange(cols, device=DEV) // BLOCK
        return y / scale[r][:, c], scale

    if kind == "norm":
        h = s["x"].double()
        if case["residual"]:
            h = h + s["residual"].double()
        y = h / torch.sqrt((h * h).sum(1) / case["channels"] + EPS)[:, None] * s["weight"].double()
        q, scale = in_blocks(y, 1)
        return q, scale.t().contiguous(), h if case["residual"] else None
    if kind == "quantize":
        x = s["x"].double()
        if case["gated"]:
            c = case["channels"]
            x = x[:, :c] * torch.sigmoid(x[:, :c]) * x[:, c:]
        q, scale = in_blocks(x, 1)
        return q, scale.t().contiguous()
    if kind == "weights":
        return in_blocks(s["w"].double(), BLOCK)
    out = torch.zeros((case["rows"], case["n"]), dtype=torch.float64, device=DEV)
    where = torch.arange(case["n"], device=DEV) // BLOCK
    for b in range(_blocks(case["k"])):
        k = slice(b * BLOCK, (b + 1) * BLOCK)
        part = s["a"][:, k].double() @ s["w"][:, k].double().t().contiguous()
        part *= s["a_scale"][b].double()[:, None]
        part *= s["w_scale"][where, b].double()
        out += part
    if case["bias"]:
        out += s["bias"].double()
    if case["n_frames"]:
        out = out.view(-1, case["n_frames"], case["n"]).permute(0, 2, 1).contiguous()
    return out


def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "matmul":
        m, n, k = case["rows"], case["n"], case["k"]
        read = m * k + n * k + 4 * (_blocks(k) * m + _blocks(n) * _blocks(k) + (n if case["bias"] else 0))
        return {"bytes": read + m * n * size, "flops": 2 * m * n * k}
    if case["kind"] == "weights":
        n, k = case["n"], case["k"]
        return {"bytes": n * k * (size + 1) + 4 * _blocks(n) * _blocks(k), "flops": 2 * n * k}
    m, c = case["rows"], case["channels"]
    wrote = m * c + 4 * _blocks(c) * m
    if case["kind"] == "norm":
        return {"bytes": m * c * size * (3 if case["residual"] else 1) + 4 * c + wrote, "flops": 6 * m * c}
    return {"bytes": m * c * size * (2 if case["gated"] else 1) + wrote, "flops": (8 if case["gated"] else 2) * m * c}
