"""Sums of the 8-bit product over operands of very different magnitudes: what bf16 outputs lose in the 8-bit matrix instructions, and that fp32 sums do not."""
import pytest
import torch

import paper_2605_28657_amd as pa
from fp8_util import E4M3, at_rows, at_weights, blocks, laid_out, product, random_e4m3

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# without LDS, tiles with K in two groups of waves, with ragged edges, and the largest tiles
SIZES = [(1, 2048, 640), (3, 40, 600), (16, 8200, 272), (300, 600, 640), (420, 1104, 1291), (2300, 2100, 272), (4100, 4090, 384)]


def _loud(rows, n, k, kind, seed):
    """Of every 8 values of K one, at a place of its own, is 256 in both operands, and the products of the others lie just below 2^-13 and 2^-14 of that one's:
    all of one sign ("same"), of random signs ("mixed"), or small products of one sign beside large ones that cancel in pairs ("cancel")."""
    g = torch.Generator().manual_seed(seed + rows + 31 * n + 57 * k)
    groups = -(-k // 8)
    at = (torch.arange(groups) * 8 + torch.randint(0, 8, (groups,), generator=g)).clamp_max(k - 1)
    if kind == "cancel":
        a, w = torch.ones(rows, k), torch.ones(n, k)
        a[:, at], w[:, at] = 256.0, 256.0
        w[:, at[1::2]] = -256.0
    else:
        a = 1.875 * torch.exp2(torch.randint(-1, 1, (rows, k), generator=g).float())
        w = torch.full((n, k), 3.75)
        a[:, at], w[:, at] = 256.0, 256.0
        if kind == "mixed":
            a *= torch.randint(0, 2, (rows, k), generator=g) * 2 - 1
            w *= torch.randint(0, 2, (n, k), generator=g) * 2 - 1
    power = lambda *shape: torch.ones(shape) if kind == "cancel" else torch.exp2(torch.randint(-2, 3, shape, generator=g).float())      # noqa: E731
    return a.to(E4M3).to(DEV), power(blocks(k), rows).to(DEV), w.to(E4M3).to(DEV), power(blocks(n), blocks(k)).to(DEV)


def _fp32_error(k, mag):
    """128 additions of a block by a step of 2^-23 each, of the magnitudes summed so far; the scales' two roundings, an addition of a block, those of up to 16 parts of
    K and of the bias by half a step of 2^-24."""
    return (128 * 2.0 ** -23 + (3 * blocks(k) + 17) * 2.0 ** -24) * mag


def _cut(a, a_scale, w, w_scale):
    """What the 8-bit instructions may cut off: less than 2^-13 of the largest product's power of two for 7 of every 8 products.  The largest product is at most the product of
    the operands' largest magnitudes, subnormal ones (below 2^-6) counted as 2^-6."""
    def largest(t, scale):
        t = t.cpu().float().abs().clamp_min(2.0 ** -6).double() * scale
        pad = torch.nn.functional.pad(t, (0, -t.shape[1] % 8))
        return pad.view(t.shape[0], -1, 8).amax(2)
    k = a.shape[1]
    return 7 * 2.0 ** -13 * (largest(a, at_rows(a_scale.cpu().double(), k)) @ largest(w, at_weights(w_scale.cpu().double(), *w.shape)).t())


def _layouts(rows, n, k):
    aligned = -(-k // 16) * 16
    return ((aligned, 0),) if rows * n > 1 << 22 else ((aligned, 0), (k + 5, 3))


@pytest.mark.parametrize("kind", ["same", "mixed", "cancel"])
@pytest.mark.parametrize("rows,n,k", SIZES)
def test_fp32_sums_of_a_bf16_output_lose_nothing_beside_a_large_product(rows, n, k, kind):
    a, sa, w, sw = _loud(rows, n, k, kind, 1)
    want, mag, _ = product(a, sa, w, sw, None)
    most = _fp32_error(k, mag)
    for stride, before in _layouts(rows, n, k):
        got = pa.matmul_fp8(laid_out(a, stride, before), sa, laid_out(w, stride, before), sw, fp32_sums=True).cpu().double()
        assert bool(((got - want).abs() <= most * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()).all())
        if kind == "cancel":                                # whole numbers below 2^24: fp32 has all sums exactly
            assert float(mag.max()) < 2 ** 24 and torch.equal(got, want.float().bfloat16().double())


@pytest.mark.parametrize("kind", ["same", "mixed", "cancel", "normal"])
@pytest.mark.parametrize("rows,n,k", SIZES)
def test_sums_of_a_bf16_output_lose_no_more_than_is_stated(rows, n, k, kind):
    if kind == "normal":                                    # over all of e4m3's range, subnormal values too
        g = torch.Generator().manual_seed(rows + n + k)
        a, w = random_e4m3((rows, k), 11, spread=4.0), random_e4m3((n, k), 12, spread=4.0)
        sa, sw = (torch.exp2(torch.randn(shape, generator=g)).to(DEV) for shape in ((blocks(k), rows), (blocks(n), blocks(k))))
    else:
        a, sa, w, sw = _loud(rows, n, k, kind, 2)
    want, mag, _ = product(a, sa, w, sw, None)
    most = (_cut(a, sa, w, sw) + _fp32_error(k, mag)) * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
    for stride, before in _layouts(rows, n, k):
        got = pa.matmul_fp8(laid_out(a, stride, before), sa, laid_out(w, stride, before), sw).cpu().double()
        assert bool(((got - want).abs() <= most).all())
        if kind == "same":                                  # no product cancels: the loss is less than a quarter of the output's rounding
            assert bool(((got - want).abs() <= (1.25 * 2.0 ** -8 + 2.0 ** -13) * want).all())


@pytest.mark.parametrize("bias,n_frames", [(False, 0), (True, 0), (True, 5), (False, 1)])
@pytest.mark.parametrize("rows,n,k", [(5, 1, 1), (5, 64, 128), (15, 4103, 300), (65, 64, 15), (130, 257, 384), (300, 600, 400), (420, 1104, 1291), (1500, 64, 1111), (1460, 2000, 1152), (2300, 2100, 272)])
def test_a_bf16_output_of_fp32_sums_is_the_fp32_output_rounded(rows, n, k, bias, n_frames):
    g = torch.Generator().manual_seed(rows + n + k)
    a, w = random_e4m3((rows, k), 1, spread=3.0), random_e4m3((n, k), 2, spread=3.0)
    sa, sw = (torch.exp2(torch.randn(shape, generator=g)).to(DEV) for shape in ((blocks(k), rows), (blocks(n), blocks(k))))
    b = torch.randn(n, generator=g).to(DEV) if bias else None
    aligned = -(-k // 16) * 16
    for stride, before in ((aligned, 0), (k, 1)):
        av, wv = laid_out(a, stride, before), laid_out(w, stride, before)
        want = pa.matmul_fp8(av, sa, wv, sw, bias=b, n_frames=n_frames, dtype=torch.float32)
        assert torch.equal(pa.matmul_fp8(av, sa, wv, sw, bias=b, n_frames=n_frames, fp32_sums=True), want.bfloat16())
        assert torch.equal(pa.matmul_fp8(av, sa, wv, sw, bias=b, n_frames=n_frames, dtype=torch.float32, fp32_sums=True), want)
    if not n_frames:                                        # rows of a wider output, and nothing beside them
        store = torch.full((rows + 2, n + 3), -7.0, dtype=torch.bfloat16, device=DEV)
        pa.matmul_fp8(av, sa, wv, sw, bias=b, fp32_sums=True, out=store[1:1 + rows, 2:2 + n])
        assert torch.equal(store[1:1 + rows, 2:2 + n], want.bfloat16())
        assert bool((store[0] == -7).all()) and bool((store[1 + rows:] == -7).all()) and bool((store[:, :2] == -7).all()) and bool((store[:, 2 + n:] == -7).all())


def test_fp32_sums_in_a_captured_call():
    a, sa, w, sw = _loud(300, 600, 640, "mixed", 5)
    x = a.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = pa.matmul_fp8(x, sa, w, sw, fp32_sums=True)
    for i in range(4):
        fresh = _loud(300, 600, 640, "mixed", 20 + i)[0]
        x.copy_(fresh)
        want = pa.matmul_fp8(fresh, sa, w, sw, fp32_sums=True)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, want)
