"""Definitions of the 8-bit operators in 64 bits, on the CPU, and what their results may be off by."""
import torch

BLOCK = 128
FLOOR = 2.0 ** -100
E4M3 = torch.float8_e4m3fn
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # of a rounding, relative to the value


def blocks(n):
    return -(-n // BLOCK)


def e4m3(v):
    """The nearest e4m3 values (ties to even) of 64-bit values, as 64-bit values."""
    return v.float().to(E4M3).double()


def row_scales(y):
    """[blocks, rows], 64 bits."""
    pad = torch.nn.functional.pad(y, (0, blocks(y.shape[1]) * BLOCK - y.shape[1]))
    return (pad.view(y.shape[0], -1, BLOCK).abs().amax(2).clamp_min(FLOOR) / 448).t()


def at_rows(scale, channels):
    """Scales [blocks, rows] at every element."""
    return scale.t().repeat_interleave(BLOCK, 1)[:, :channels]


def at_weights(scale, n, k):
    return scale.repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]


def check_quantized(q, scale_at, want_scale_at, y, rel):
    """q [rows, channels] (e4m3) of 64-bit y: the nearest value to y / scale, or its neighbour where the border between the two is nearer than
    `rel`, the relative error that the fp32 arithmetic before the rounding may have; the scales within `rel`."""
    assert bool((scale_at - want_scale_at).abs().le(rel * want_scale_at).all()), float(((scale_at - want_scale_at).abs() / want_scale_at).max())
    v, got = y / want_scale_at, q.double()
    a, b = e4m3(v * (1 - rel)), e4m3(v * (1 + rel))
    ok = (got >= torch.minimum(a, b)) & (got <= torch.maximum(a, b))
    assert bool(ok.all()), (got[~ok][:4], v[~ok][:4])


def product(a, a_scale, w, w_scale, bias):
    """(result, sum of the terms' magnitudes, sum over the blocks of a bound on their largest product) in 64 bits; the operands on any device."""
    a, w, sa, sw = (t.cpu().double() for t in (a, w, a_scale, w_scale))
    k = a.shape[1]
    x, z = a * at_rows(sa, k), w * at_weights(sw, *w.shape)
    out, mag = x @ z.t(), x.abs() @ z.abs().t()
    pad = (0, blocks(k) * BLOCK - k)
    largest = [torch.nn.functional.pad(t.abs(), pad).view(t.shape[0], -1, BLOCK).amax(2) for t in (x, z)]
    if bias is not None:
        out, mag = out + bias.cpu().double(), mag + bias.cpu().double().abs()
    return out, mag, largest[0] @ largest[1].t()


def check_product(got, want, mag, largest, k, dtype):
    """Products of e4m3 values are exact in fp32.  The 128 additions of a block may each be off by a step of fp32 (2^-23, not half of it: how
    the matrix unit rounds is not assumed) of the magnitudes summed so far, an addition of a block and the two roundings of its scales
    by half a step each, and so may the additions of up to 16 parts of K and of the bias.  For bf16 outputs the unit keeps 13 bits below the largest
    product of those it adds at once: 128 errors of up to 2^-14 of it either way, which is 128^(1/2) 2^-14 / 3^(1/2) = 2^-11.3 of it in the mean square; six
    of these cover every output of a test, less than 2^-8.7 of the block's largest product."""
    rel = 128 * 2.0 ** -23 + (3 * blocks(k) + 16 + 1) * 2.0 ** -24
    off = (got.cpu().double() - want).abs()
    sums = rel * mag + (2.0 ** -8.7 * largest if dtype == torch.bfloat16 else 0)
    most = sums * (1 + HALF_STEP[dtype]) + HALF_STEP[dtype] * want.abs()
    assert bool((off <= most).all()), (float((off - most).max()), float((off / mag.clamp_min(1e-300)).max()))


def random_e4m3(shape, seed, device="cuda:0", spread=1.5):
    """Values over all of e4m3's range: normals times powers of two."""
    g = torch.Generator().manual_seed(seed)
    v = torch.randn(shape, generator=g) * torch.exp2(spread * torch.randn(shape, generator=g))
    return v.clamp(-448, 448).to(E4M3).to(device)


def laid_out(q, stride=None, before=0, fill=0x7f):
    """q [rows, channels] as a view with the given row stride, `before` bytes after an aligned address; every byte that is not q's is NaN."""
    rows, channels = q.shape
    stride = stride or channels
    store = torch.full((before + rows * stride + 64,), fill, dtype=torch.uint8, device=q.device)
    view = torch.as_strided(store, (rows, channels), (stride, 1), before)
    view.copy_(q.view(torch.uint8))
    return view.view(E4M3)
