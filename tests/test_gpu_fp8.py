"""The 8-bit operators against their definitions in 64 bits (fp8_util), at the sizes, strides and values where they can go wrong."""
import pytest
import torch

import demon_inputs as di
import paper_2605_28657_amd as pa
from fp8_util import (E4M3, HALF_STEP, TORCH, at_rows, at_weights, blocks, check_product, check_quantized, e4m3, laid_out, product, random_e4m3,
                      row_scales)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# What the fp32 arithmetic before the rounding to 8 bits may be off by, relative (steps of 2^-24): the reciprocal and the product with it 3,
# the scale's quotient 1; the gate's exponential 16 (its argument is rounded at up to 23 = log2 of the magnitudes that count), its quotient and products 4;
# the norm's sum of squares (32 in a thread, 6 + 16 joined, the additions of positive terms: 55, halved by the root), its root 2, products 3.
REL_PLAIN, REL_GATE, REL_NORM = 4 * 2.0 ** -24, 32 * 2.0 ** -24, 48 * 2.0 ** -24


def _normal(shape, seed, dtype, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * torch.exp2(spread * torch.randn(shape, generator=g))).to(TORCH[dtype]).to(DEV)


def _wide(t, extra, before=0):
    """The same rows as a view into wider ones that hold NaN elsewhere."""
    store = torch.full((t.shape[0] + 1, t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    view = store[:t.shape[0], before:before + t.shape[1]]
    view.copy_(t)
    return view


# ---------------------------------------------------------------------------------- rows
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,channels", [(1, 1), (1, 128), (2, 7), (3, 129), (5, 1111), (16, 2048), (17, 640), (75, 5632), (130, 1000), (1, 20000), (2000, 72)])
def test_rows(rows, channels, dtype, gated):
    x = _normal((rows, channels * (2 if gated else 1)), rows * channels, dtype)
    q, scale = pa.quantize_fp8(x, gated=gated)
    y = x.cpu().double()
    if gated:
        y = y[:, :channels] * torch.sigmoid(y[:, :channels]) * y[:, channels:]
    check_quantized(q.cpu(), at_rows(scale.cpu().double(), channels), at_rows(row_scales(y), channels), y, REL_GATE if gated else REL_PLAIN)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gated", [False, True])
def test_rows_of_any_stride_and_alignment_write_nothing_else(dtype, gated):
    rows, channels = 37, 333
    x = _normal((rows, channels * (2 if gated else 1)), 5, dtype)
    want_q, want_s = pa.quantize_fp8(x, gated=gated)
    for before in (1, 3, 8):
        xv = _wide(x, 11, before)
        q = torch.full((rows + 2, channels + 5), 0x55, dtype=torch.uint8, device=DEV)
        s = torch.full((blocks(channels) + 1, rows + 3), -1.0, device=DEV)
        qv, sv = q[:rows, before % 4:before % 4 + channels].view(E4M3), s[:-1, 2:2 + rows]
        pa.quantize_fp8(xv, gated=gated, out=(qv, sv))
        assert torch.equal(qv.view(torch.uint8), want_q.view(torch.uint8)) and torch.equal(sv, want_s)
        assert int((q == 0x55).sum()) == q.numel() - rows * channels + int((want_q.view(torch.uint8) == 0x55).sum())
        assert int((s == -1).sum()) == s.numel() - sv.numel()


def test_rows_of_special_values():
    x = torch.zeros((8, 300), device=DEV)
    x[1] = 2.0 ** -120                                    # below the smallest scale: zeros
    x[2] = torch.linspace(-1, 1, 300, device=DEV) * 2.0 ** 120
    x[3, 5], x[3, 140:] = float("inf"), 1.0               # an infinity in the first block only
    x[4, 200] = float("nan")                              # a NaN in the second
    x[4, :128] = 1.0
    x[5, 299] = -float("inf")
    x[6] = torch.finfo(torch.float32).max
    x[7] = -0.0
    q, s = pa.quantize_fp8(x)
    v, s = q.float().cpu(), s.cpu()
    floor = 2.0 ** -100 / 448
    assert bool((v[0] == 0).all()) and bool((v[1] == 0).all()) and bool((v[7] == 0).all())
    assert torch.allclose(s[:, [0, 1, 7]], torch.full((3, 3), floor), rtol=2.0 ** -23)
    assert bool(torch.isfinite(v[2]).all()) and float(v[2, 0]) == -448 and float(v[2, 299]) == 448
    assert torch.isinf(s[0, 3]) and bool(torch.isnan(v[3, 5])) and bool((v[3, :5] == 0).all()) and bool((v[3, 140:] == 448).all())
    assert bool((v[4, :128] == 448).all()) and bool(torch.isnan(v[4, 128:256]).all()) and bool(torch.isnan(s[1, 4])) and bool((v[4, 256:] == 0).all())
    assert bool(torch.isnan(v[5, 299])) and bool((v[5, :299] == 0).all())
    assert bool((v[6] == 448).all())
    # every e4m3 value comes back as itself under the scale of one
    every = torch.arange(256, dtype=torch.uint8).view(E4M3).float()
    every = torch.where(torch.isnan(every), torch.full_like(every, 448), every).view(2, 128)
    q, s = pa.quantize_fp8(every.to(DEV))
    assert bool((s == 1).all()) and torch.equal(q.float().cpu(), every)


def test_gate_of_large_magnitudes():
    gate = torch.tensor([[-1e4, -200.0, -88.0, 0.0, 88.0, 200.0, 1e4, float("inf"), -float("inf")]], device=DEV)
    x = torch.cat([gate[:, :7], torch.ones(1, 7, device=DEV)], 1)
    q, s = pa.quantize_fp8(x, gated=True)
    got = q.float() * s[0, 0]
    assert float(got[0, 6]) == pytest.approx(1e4, rel=2e-7) and bool((got[0, :4] == 0).all()) and float(got[0, 5]) == pytest.approx(200, rel=2 ** -4)
    q, s = pa.quantize_fp8(torch.cat([gate, torch.ones(1, 9, device=DEV)], 1), gated=True)      # -inf * 0 is NaN, as by the formula
    assert bool(torch.isnan(s).all())


# ---------------------------------------------------------------------------------- norm
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,channels", [(1, 1), (3, 8), (1, 2048), (5, 512), (6, 513), (9, 1024), (7, 1111), (130, 2048), (33, 2049), (4, 4096), (3, 5000),
                                           (2, 8192), (2, 8200), (1, 16384), (2, 16385), (3, 32768), (1000, 64)])
def test_norm(rows, channels, dtype, residual):
    x = _normal((rows, channels), rows + channels, dtype)
    r = _normal((rows, channels), rows + channels + 1, dtype, 2.0) if residual else None
    w = _normal((channels,), 3, "f32", 0.3)
    q, scale, h = pa.rms_norm_fp8(x, w, 1e-6, residual=r)
    want = x.cpu().double() + (r.cpu().double() if residual else 0)
    assert (h is None) == (not residual)
    if residual:
        # the fp32 addition and the rounding to the type
        assert bool(((h.cpu().double() - want).abs() <= (HALF_STEP[TORCH[dtype]] + 2.0 ** -24) * want.abs() * (1 + 2.0 ** -8)).all())
    y = want / torch.sqrt((want * want).mean(1, keepdim=True) + 1e-6) * w.cpu().double()
    # a sum of two terms that nearly cancel is off by 2^-24 of itself, like any other
    check_quantized(q.cpu(), at_rows(scale.cpu().double(), channels), at_rows(row_scales(y), channels), y, REL_NORM)


def test_norm_in_place_and_strided():
    rows, channels = 21, 1111
    for dtype in ("bf16", "f32"):
        x, r = _normal((rows, channels), 1, dtype), _normal((rows, channels), 2, dtype)
        w = _normal((channels,), 3, "f32", 0.3)
        q, s, h = pa.rms_norm_fp8(x, w, residual=r)
        for where in ("x", "residual", "wide"):
            xv, rv = _wide(x, 5, 3), _wide(r, 9, 1)
            out = {"x": xv, "residual": rv, "wide": _wide(torch.zeros_like(x), 3, 2)}[where]
            q2, s2, h2 = pa.rms_norm_fp8(xv, w, residual=rv, sum_out=out)
            assert h2 is out and torch.equal(out, h) and torch.equal(s2, s) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8)), where
            base = out._base
            assert int(torch.isnan(base).sum()) == base.numel() - rows * channels
        # h without a residual is x
        copy = torch.zeros_like(x)
        assert torch.equal(pa.rms_norm_fp8(x, w, sum_out=copy)[2], x)
        # one row for all
        one = pa.rms_norm_fp8(x[:1].expand(rows, channels), w, residual=r)
        assert torch.equal(one[2], pa.rms_norm_fp8(x[:1].repeat(rows, 1), w, residual=r)[2])


def test_norm_of_special_rows():
    c = 400
    x = torch.ones((6, c), device=DEV)
    x[0] = 0
    x[1, 7] = float("nan")
    x[2, 7] = float("inf")
    x[3] = 1e25                      # the squares overflow: inv = 0, y = 0
    w = torch.ones(c, device=DEV)
    q, s, _ = pa.rms_norm_fp8(x, w, 1e-6)
    v = q.float()
    assert bool((v[0] == 0).all()) and bool(torch.isnan(v[1]).all())
    assert bool(torch.isnan(v[2, :128]).all()) and bool((v[2, 128:] == 0).all())
    assert bool((v[3] == 0).all()) and bool((v[4] == 448).all())
    q, s, _ = pa.rms_norm_fp8(x, w, 0.0)
    assert bool(torch.isnan(q.float()[0]).all()) and bool((q.float()[5] == 448).all())


# ---------------------------------------------------------------------------------- weights
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,k", [(1, 1), (128, 128), (129, 127), (64, 1111), (517, 300), (1000, 2048)])
def test_weights(n, k, dtype):
    w = _normal((n, k), n + k, dtype)
    q, scale = pa.quantize_weights_fp8(w)
    y = w.cpu().double()
    want = torch.stack([torch.stack([y[i:i + 128, j:j + 128].abs().max() for j in range(0, k, 128)]) for i in range(0, n, 128)]) / 448
    check_quantized(q.cpu(), at_weights(scale.cpu().double(), n, k), at_weights(want, n, k), y, REL_PLAIN)
    view = _wide(w, 3, 1)
    store = torch.full((n + 1, k + 3), 0x55, dtype=torch.uint8, device=DEV)
    q2, s2 = pa.quantize_weights_fp8(view, out=(store[:n, 1:1 + k].view(E4M3), torch.empty_like(scale)))
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, scale)
    assert bool((store[n] == 0x55).all()) and bool((store[:, 0] == 0x55).all()) and bool((store[:, k + 1:] == 0x55).all())


def test_weights_of_special_values():
    w = torch.zeros((256, 256), device=DEV)
    w[3, 200], w[200, 5], w[130:140, 130:140] = float("nan"), float("inf"), 3.0
    q, s = pa.quantize_weights_fp8(w)
    v, s = q.float().cpu(), s.cpu()
    assert bool((v[:128, :128] == 0).all()) and float(s[0, 0]) == pytest.approx(2.0 ** -100 / 448, rel=2 ** -22)
    assert bool(torch.isnan(v[:128, 128:]).all()) and bool(torch.isnan(s[0, 1]))
    assert bool(torch.isnan(v[200, 5])) and int(torch.isnan(v[128:, :128]).sum()) == 1 and bool(torch.isinf(s[1, 0]))
    assert bool((v[130:140, 130:140] == 448).all()) and int((v[128:, 128:] != 0).sum()) == 100


# ---------------------------------------------------------------------------------- matrix product
SIZES = [(1, 1, 1), (1, 64, 128), (2, 17, 16), (7, 65, 129), (16, 128, 256), (17, 130, 1111), (1, 2048, 2048), (8, 1000, 640), (33, 96, 4096),
         (64, 64, 127), (65, 64, 15), (75, 192, 320), (128, 128, 128), (129, 257, 384), (300, 520, 1040), (513, 300, 2000), (700, 1030, 528), (2100, 260, 136),
         (1500, 64, 1111), (260, 2100, 96), (2300, 2100, 272)]


def _operands(rows, n, k, seed=0):
    g = torch.Generator().manual_seed(seed + rows + 31 * n + 57 * k)
    a, w = random_e4m3((rows, k), seed + 1), random_e4m3((n, k), seed + 2)
    sa = torch.exp2(torch.randn((blocks(k), rows), generator=g)).to(DEV)
    sw = torch.exp2(torch.randn((blocks(n), blocks(k)), generator=g)).to(DEV)
    return a, sa, w, sw, torch.randn(n, generator=g).mul(8).to(DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n,k", SIZES)
def test_product(rows, n, k, dtype):
    a, sa, w, sw, bias = _operands(rows, n, k)
    aligned = -(-k // 16) * 16
    for b in (None, bias):
        want = product(a, sa, w, sw, b)
        for stride_a, stride_w, before in ((aligned, aligned, 0), (k, k, 0), (k + 37, aligned + 16, 5)):
            got = pa.matmul_fp8(laid_out(a, stride_a, before), sa, laid_out(w, stride_w, 0), sw, bias=b, dtype=TORCH[dtype])
            check_product(got, *want, k, TORCH[dtype])


@pytest.mark.parametrize("rows,n,k", SIZES)
def test_product_of_whole_numbers_is_exact(rows, n, k):
    g = torch.Generator().manual_seed(rows + n + k)
    a = torch.randint(-4, 5, (rows, k), generator=g).float().to(E4M3).to(DEV)
    w = torch.randint(-4, 5, (n, k), generator=g).float().to(E4M3).to(DEV)
    sa = torch.exp2(torch.randint(-1, 2, (blocks(k), rows), generator=g).float()).to(DEV)
    sw = torch.exp2(torch.randint(-1, 2, (blocks(n), blocks(k)), generator=g).float()).to(DEV)
    bias = torch.randint(-9, 10, (n,), generator=g).float().to(DEV)
    want, mag, _ = product(a, sa, w, sw, bias)
    assert float(mag.max()) < 2 ** 22                       # in quarters: all sums are whole numbers below 2^24
    aligned = -(-k // 16) * 16
    for stride, before in ((aligned, 0), (aligned, 16), (k, 1)):
        got = pa.matmul_fp8(laid_out(a, stride, before), sa, laid_out(w, stride, before), sw, bias=bias, dtype=torch.float32)
        assert torch.equal(got.cpu().double(), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("clips,frames,n,k", [(1, 1, 64, 128), (3, 7, 64, 200), (2, 75, 16, 256), (4, 375, 64, 1111), (1, 700, 300, 272), (8, 33, 65, 512)])
def test_product_as_a_latent(clips, frames, n, k, dtype):
    a, sa, w, sw, bias = _operands(clips * frames, n, k, 9)
    rows = pa.matmul_fp8(a, sa, w, sw, bias=bias, dtype=TORCH[dtype])
    store = torch.full((clips * n * frames + 2,), -7.0, dtype=TORCH[dtype], device=DEV)
    out = store[1:-1].view(clips, n, frames)
    assert pa.matmul_fp8(a, sa, w, sw, bias=bias, n_frames=frames, out=out) is out
    assert torch.equal(out, rows.view(clips, frames, n).transpose(1, 2)) and float(store[0]) == -7 and float(store[-1]) == -7


@pytest.mark.parametrize("rows,n,k", [(1, 70, 144), (20, 100, 300), (150, 200, 272), (600, 300, 640)])
def test_product_leaves_what_is_behind_its_rows(rows, n, k):
    a, sa, w, sw, _ = _operands(rows, n, k, 4)
    for dtype in ("bf16", "f32"):
        want = pa.matmul_fp8(a, sa, w, sw, dtype=TORCH[dtype])
        for extra in (0, 3, 8):
            store = torch.full((rows + 3, n + extra), -7.0, dtype=TORCH[dtype], device=DEV)
            pa.matmul_fp8(a, sa, w, sw, out=store[1:1 + rows, :n])
            assert torch.equal(store[1:1 + rows, :n], want)
            assert bool((store[0] == -7).all()) and bool((store[1 + rows:] == -7).all()) and bool((store[:, n:] == -7).all())


@pytest.mark.parametrize("rows,n,k", [(5, 40, 300), (140, 150, 272), (520, 520, 640)])
def test_product_of_special_values(rows, n, k):
    """A NaN or an infinite scale stays in its own row or column; scales of blocks differ by whole range."""
    a, sa, w, sw, _ = _operands(rows, n, k, 6)
    clean = pa.matmul_fp8(a, sa, w, sw, dtype=torch.float32)
    bad = a.clone()
    bad.view(torch.uint8)[rows - 1, k - 1] = 0x7f
    got = pa.matmul_fp8(bad, sa, w, sw, dtype=torch.float32)
    assert bool(torch.isnan(got[rows - 1]).all()) and torch.equal(got[:rows - 1], clean[:rows - 1])
    bad = w.clone()
    bad.view(torch.uint8)[3, 0] = 0xff
    got = pa.matmul_fp8(a, sa, bad, sw, dtype=torch.float32)
    assert bool(torch.isnan(got[:, 3]).all()) and int(torch.isnan(got).sum()) == rows
    scales = sa.clone()
    scales[1, 2] = float("inf")
    got = pa.matmul_fp8(a, scales, w, sw, dtype=torch.float32)
    assert not bool(torch.isfinite(got[2]).any()) and torch.equal(got[3:], clean[3:])
    zero = pa.matmul_fp8(torch.zeros_like(a.view(torch.uint8)).view(E4M3), sa, w, sw)
    assert bool((zero == 0).all())


def test_product_behind_32_bit_offsets():
    """Rows further apart than 2^32 bytes between the first and the last, in each operand and in the output."""
    rows, n, k = 68, 66, 160
    a, sa, w, sw, _ = _operands(rows, n, k, 8)
    want = pa.matmul_fp8(a, sa, w, sw)
    far = 64 * 1024 * 1024 + 16                                     # bytes between rows: 4.3 GB from first to last
    store = torch.empty(far * (rows - 1) + k, dtype=torch.uint8, device=DEV)
    av = torch.as_strided(store, (rows, k), (far, 1))
    av.copy_(a.view(torch.uint8))
    wv = torch.as_strided(store, (n, k), (far, 1), 512)
    wv.copy_(w.view(torch.uint8))
    assert torch.equal(pa.matmul_fp8(av.view(E4M3), sa, wv.view(E4M3), sw), want)
    out = torch.empty(far * (rows - 1) + n, dtype=torch.bfloat16, device=DEV).as_strided((rows, n), (far, 1))
    assert torch.equal(pa.matmul_fp8(a, sa, w, sw, out=out), want)


def test_rows_behind_32_bit_offsets():
    rows, c = 70, 260
    far = 40 * 1024 * 1024
    store = torch.empty(far * (rows - 1) + 2 * c, dtype=torch.bfloat16, device=DEV)
    x = torch.as_strided(store, (rows, 2 * c), (far, 1))
    x.copy_(_normal((rows, 2 * c), 1, "bf16"))
    dense = x.contiguous()
    w = _normal((c,), 3, "f32", 0.3)
    q = torch.empty(64 * 1024 * 1024 * (rows - 1) + c, dtype=torch.uint8, device=DEV).as_strided((rows, c), (64 * 1024 * 1024, 1)).view(E4M3)
    s = torch.empty((blocks(c), rows), device=DEV)
    def same(want):
        assert torch.equal(q.contiguous().view(torch.uint8), want[0].contiguous().view(torch.uint8)) and torch.equal(s, want[1])

    pa.quantize_fp8(x, True, out=(q, s))
    same(pa.quantize_fp8(dense, True))
    pa.rms_norm_fp8(x[:, :c], w, residual=x[:, c:], sum_out=x[:, c:], out=(q, s))
    same(pa.rms_norm_fp8(dense[:, :c], w, residual=dense[:, c:]))
    assert torch.equal(x[:, c:], (dense[:, :c].float() + dense[:, c:].float()).bfloat16())


# ---------------------------------------------------------------------------------- as they are used
def _layer(x, residual, norm_w, gate_up, down, final_w, head, head_bias, frames):
    """A feed-forward layer, the last norm and the projection to the latent."""
    q, s, h = pa.rms_norm_fp8(x, norm_w, residual=residual)
    gu = pa.matmul_fp8(q, s, *gate_up)
    g, gs = pa.quantize_fp8(gu, gated=True)
    d = pa.matmul_fp8(g, gs, *down)
    q2, s2, h2 = pa.rms_norm_fp8(d, final_w, residual=h)
    return (q, s, h, gu, g, gs, d, q2, s2, h2), pa.matmul_fp8(q2, s2, *head, bias=head_bias, n_frames=frames)


def _layer_inputs(rows, c=320, f=704, latent=16, seed=0):
    x, r = _normal((rows, c), seed, "bf16", 0.3), _normal((rows, c), seed + 1, "bf16", 0.5)
    weights = [pa.quantize_weights_fp8(_normal(shape, 20 + i, "bf16", 0.2) * shape[1] ** -0.5) for i, shape in enumerate([(2 * f, c), (c, f), (latent, c)])]
    return x, r, 1 + 0.1 * _normal((c,), 5, "f32"), weights[0], weights[1], 1 + 0.1 * _normal((c,), 6, "f32"), weights[2], _normal((latent,), 7, "f32", 0.0)


def test_a_layer_and_the_decode_behind_it():
    clips, frames = 2, 25
    args = _layer_inputs(clips * frames, latent=64)
    (q, s, h, gu, g, gs, d, q2, s2, h2), z = _layer(*args, frames)
    x, r, nw, up, down, fw, head, hb = args
    cpu = lambda t: t.cpu().double()                          # noqa: E731
    # each step against its definition, from the step before as it is
    y = cpu(x) + cpu(r)
    y = y / torch.sqrt((y * y).mean(1, keepdim=True) + 1e-6) * cpu(nw)
    check_quantized(q.cpu(), at_rows(cpu(s), y.shape[1]), at_rows(row_scales(y), y.shape[1]), y, REL_NORM)
    check_product(gu, *product(q, s, *up, None), q.shape[1], torch.bfloat16)
    y = cpu(gu)
    y = y[:, :704] * torch.sigmoid(y[:, :704]) * y[:, 704:]
    check_quantized(g.cpu(), at_rows(cpu(gs), 704), at_rows(row_scales(y), 704), y, REL_GATE)
    check_product(d, *product(g, gs, *down, None), 704, torch.bfloat16)
    y = cpu(d) + cpu(h)
    assert bool(((cpu(h2) - y).abs() <= (2.0 ** -8 + 2.0 ** -16) * y.abs()).all())
    y = y / torch.sqrt((y * y).mean(1, keepdim=True) + 1e-6) * cpu(fw)
    check_quantized(q2.cpu(), at_rows(cpu(s2), y.shape[1]), at_rows(row_scales(y), y.shape[1]), y, REL_NORM)
    check_product(z.transpose(1, 2).reshape(clips * frames, 64), *product(q2, s2, *head, hb), 320, torch.bfloat16)
    # the latent goes into the decode as it is
    spec = di.DecoderSpec(64, (2, 2), (64, 32), (1, 3))
    vae = pa.DemonVAE(spec, di.make_weights(spec, 0, bf16=True), dtype="bf16", max_frames=frames, max_clips=clips, max_extended_frames=400)
    same = pa.matmul_fp8(q2, s2, *head, bias=hb).view(clips, frames, 64).transpose(1, 2).contiguous()
    assert torch.equal(vae.decode_windowed(z, window=8), vae.decode_windowed(same, window=8))
    vae.close()


def test_one_row_at_a_time_gives_the_rows_of_a_batch():
    """Sums of a row's products may be taken in another order for other numbers of rows; quantised rows do not depend on their number at all."""
    args = _layer_inputs(40)
    steps, z = _layer(*args, 0)
    x, r, nw, up = args[:4]
    for m in (0, 17, 39):
        q, s, h = pa.rms_norm_fp8(x[m:m + 1], nw, residual=r[m:m + 1])
        assert torch.equal(q.view(torch.uint8), steps[0][m:m + 1].view(torch.uint8)) and torch.equal(s, steps[1][:, m:m + 1]) and torch.equal(h, steps[2][m:m + 1])
        check_product(pa.matmul_fp8(q, s, *up), *product(q, s, *up, None), 320, torch.bfloat16)
        g, gs = pa.quantize_fp8(steps[3][m:m + 1], gated=True)
        assert torch.equal(g.view(torch.uint8), steps[4][m:m + 1].view(torch.uint8)) and torch.equal(gs, steps[5][:, m:m + 1])


@pytest.mark.parametrize("rows", [1, 50, 600])
def test_a_captured_layer_replays_on_new_inputs(rows):
    args = _layer_inputs(rows, seed=3)
    x, r = args[0].clone(), args[1].clone()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            steps, z = _layer(x, r, *args[2:], 0)
    for i in range(4):
        fresh = _layer_inputs(rows, seed=30 + i)
        x.copy_(fresh[0])
        r.copy_(fresh[1])
        want_steps, want = _layer(fresh[0], fresh[1], *args[2:], 0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(z, want) and all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(steps, want_steps))


def test_two_streams_at_once_and_repeated_calls_give_the_same_bits():
    args = [_layer_inputs(300, seed=s) for s in (1, 2)]
    want = [_layer(*a, 0)[1] for a in args]
    streams = [torch.cuda.Stream() for _ in args]
    torch.cuda.synchronize()
    for _ in range(5):
        got = []
        for a, st in zip(args, streams):
            with torch.cuda.stream(st):
                got.append(_layer(*a, 0)[1])
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_tensors_of_another_device_than_the_current_one():
    if torch.cuda.device_count() < 2:
        pytest.skip("one GPU")
    x = _normal((5, 300), 1, "bf16")
    q, s = pa.quantize_fp8(x)
    q1, s1 = pa.quantize_fp8(x.to("cuda:1"))
    assert torch.equal(s, s1.to(DEV)) and torch.equal(q.view(torch.uint8), q1.to(DEV).view(torch.uint8))


def test_wrong_tensors_are_refused():
    a, sa, w, sw, bias = _operands(4, 8, 200)
    x = torch.zeros((4, 200), device=DEV)
    bad = [lambda: pa.matmul_fp8(a, sa, w[:, :199], sw), lambda: pa.matmul_fp8(a, sa[:1], w, sw), lambda: pa.matmul_fp8(a, sa.t().contiguous().t(), w, sw),
           lambda: pa.matmul_fp8(a, sa, w, sw[:, :1]), lambda: pa.matmul_fp8(a, sa, w, sw, bias=bias[:7]), lambda: pa.matmul_fp8(a, sa, w, sw, n_frames=3),
           lambda: pa.matmul_fp8(a.t(), sa, w, sw), lambda: pa.matmul_fp8(a, sa, w, sw, out=torch.zeros((4, 7), device=DEV)),
           lambda: pa.matmul_fp8(a, sa, w, sw, dtype=torch.float32, out=torch.zeros((4, 8), dtype=torch.bfloat16, device=DEV)),
           lambda: pa.matmul_fp8(a.float(), sa, w, sw), lambda: pa.quantize_fp8(x[:, :199], gated=True), lambda: pa.quantize_fp8(x.t()),
           lambda: pa.quantize_fp8(x, out=(torch.empty((4, 199), dtype=E4M3, device=DEV), torch.empty((2, 4), device=DEV))),
           lambda: pa.rms_norm_fp8(x, torch.ones(199, device=DEV)), lambda: pa.rms_norm_fp8(x, torch.ones(200, device=DEV), residual=x.bfloat16()),
           lambda: pa.quantize_weights_fp8(x, out=(torch.empty((4, 200), dtype=E4M3, device=DEV), torch.empty((2, 1), device=DEV)))]
    for call in bad:
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: pa.quantize_fp8(x[:0]), lambda: pa.rms_norm_fp8(x[:0], torch.ones(200, device=DEV)), lambda: pa.matmul_fp8(a[:0], sa[:, :0], w, sw),
                 lambda: pa.quantize_weights_fp8(x[:, :0])):
        with pytest.raises(pa.DemonError) as e:
            call()
        assert e.value.status == pa.DEMON_ERR_INVALID_ARG
    with pytest.raises(pa.DemonError):                               # written rows that overlap
        pa.matmul_fp8(a, sa, w, sw, out=torch.zeros(64, device=DEV).as_strided((4, 8), (4, 1)))


# 256 x 256 tiles, in rounds where K is a multiple of 128 from 256 on: a last round cut in parts or not, ragged edges, K of 1, 2, 3 and more blocks
@pytest.mark.parametrize("rows,n,k", [(4096, 4096, 100), (4096, 4096, 128), (4100, 4090, 136), (4096, 4096, 144), (4096, 4096, 392), (4096, 4096, 400), (8200, 4400, 272), (4096, 4096, 256), (4100, 4090, 384), (4097, 4352, 256), (5000, 6200, 512), (2050, 8200, 640), (8200, 8200, 256)])
def test_product_of_many_tiles(rows, n, k):
    g = torch.Generator().manual_seed(rows + n + k)
    whole = lambda *shape: torch.randint(-4, 5, shape, generator=g).float().to(E4M3).to(DEV)      # noqa: E731
    powers = lambda *shape: torch.exp2(torch.randint(-1, 2, shape, generator=g).float()).to(DEV)  # noqa: E731
    for again in range(2):
        aligned = -(-k // 16) * 16
        a, w, sa, sw = laid_out(whole(rows, k), aligned), laid_out(whole(n, k), aligned), powers(blocks(k), rows), powers(blocks(n), blocks(k))
        bias = torch.randint(-9, 10, (n,), generator=g).float().to(DEV)
        # whole numbers of quarters below 2^24: fp32 has them exactly, and so has a product of fp32 matrices
        want = (a.float() * at_rows(sa, k)) @ (w.float() * at_weights(sw, n, k)).t()
        assert float(want.abs().max()) < 2 ** 14
        for b in (None, bias):
            got = pa.matmul_fp8(a, sa, w, sw, bias=b)
            assert torch.equal(got, (want if b is None else want + b).bfloat16())
    if rows % 5 == 0:
        latent = pa.matmul_fp8(a, sa, w, sw, n_frames=rows // 5)
        assert torch.equal(latent, want.bfloat16().view(5, rows // 5, n).transpose(1, 2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n,k", [(300, 600, 128), (300, 600, 256), (300, 600, 384), (300, 600, 400), (1300, 2000, 656), (1400, 1900, 1152), (500, 2100, 512), (150, 4000, 1040),
                                      (40, 8200, 384), (70, 8200, 2064), (700, 700, 127)])
def test_product_of_few_tiles_with_k_in_two_groups(rows, n, k, dtype):
    """One block of K, odd numbers of them, and a block that K ends in, where two groups of waves take the blocks in turn."""
    g = torch.Generator().manual_seed(rows + n + k)
    whole = lambda *shape: torch.randint(-4, 5, shape, generator=g).float().to(E4M3).to(DEV)      # noqa: E731
    powers = lambda *shape: torch.exp2(torch.randint(-1, 2, shape, generator=g).float()).to(DEV)  # noqa: E731
    a, w, sa, sw = whole(rows, k), whole(n, k), powers(blocks(k), rows), powers(blocks(n), blocks(k))
    want = (a.float() * at_rows(sa, k)) @ (w.float() * at_weights(sw, n, k)).t()
    aligned = -(-k // 16) * 16
    got = pa.matmul_fp8(laid_out(a, aligned), sa, laid_out(w, aligned), sw, dtype=TORCH[dtype])
    assert torch.equal(got, want.to(TORCH[dtype]))
    bad = a.clone()
    bad.view(torch.uint8)[5, k - 1] = 0x7f
    got = pa.matmul_fp8(laid_out(bad, aligned), sa, laid_out(w, aligned), sw, dtype=TORCH[dtype])
    assert bool(torch.isnan(got[5]).all()) and int(torch.isnan(got).sum()) == n and torch.equal(got[6:], want[6:].to(TORCH[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", [(3, 70), (100, 150), (700, 700), (2300, 2100)])
@pytest.mark.parametrize("k", [1, 7, 15, 16, 17, 31, 48, 113, 127, 129, 143, 160, 255, 272, 383, 399])
def test_product_of_every_end_of_k(rows, n, k, dtype):
    """K ends in every place of a block and of a piece; the bytes behind each row are NaN, and so are those before the first and behind the last."""
    g = torch.Generator().manual_seed(rows + n + k)
    whole = lambda *shape: torch.randint(-4, 5, shape, generator=g).float().to(E4M3).to(DEV)      # noqa: E731
    powers = lambda *shape: torch.exp2(torch.randint(-1, 2, shape, generator=g).float()).to(DEV)  # noqa: E731
    a, w, sa, sw = whole(rows, k), whole(n, k), powers(blocks(k), rows), powers(blocks(n), blocks(k))
    want = ((a.float() * at_rows(sa, k)) @ (w.float() * at_weights(sw, n, k)).t()).to(TORCH[dtype])
    for stride, before in ((-(-k // 16) * 16, 16), (k, 0), (k + 5, 3)):
        assert torch.equal(pa.matmul_fp8(laid_out(a, stride, before), sa, laid_out(w, stride, before), sw, dtype=TORCH[dtype]), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", [(1460, 2000), (2950, 2040), (740, 2010), (5900, 705), (1000, 3800)])
@pytest.mark.parametrize("k", [128, 272, 1111, 1152])
def test_product_of_counts_of_rows_between_those_of_the_square_tiles(rows, n, k, dtype):
    """Tiles of 96 rows, one a compute unit and more, with rows and columns that end inside a tile; bias and the latent layout with them."""
    g = torch.Generator().manual_seed(rows + n + k)
    whole = lambda *shape: torch.randint(-4, 5, shape, generator=g).float().to(E4M3).to(DEV)      # noqa: E731
    powers = lambda *shape: torch.exp2(torch.randint(-1, 2, shape, generator=g).float()).to(DEV)  # noqa: E731
    a, w, sa, sw = whole(rows, k), whole(n, k), powers(blocks(k), rows), powers(blocks(n), blocks(k))
    bias = torch.randint(-9, 10, (n,), generator=g).float().to(DEV)
    want = ((a.float() * at_rows(sa, k)) @ (w.float() * at_weights(sw, n, k)).t() + bias).to(TORCH[dtype])
    aligned = -(-k // 16) * 16
    la, lw = laid_out(a, aligned), laid_out(w, aligned)
    assert torch.equal(pa.matmul_fp8(la, sa, lw, sw, bias=bias, dtype=TORCH[dtype]), want)
    latent = pa.matmul_fp8(la, sa, lw, sw, bias=bias, dtype=TORCH[dtype], n_frames=rows // 5)
    assert torch.equal(latent, want.view(5, rows // 5, n).transpose(1, 2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n,k", [(1, 4097, 128), (1, 4113, 1111), (3, 4200, 15), (9, 5000, 300), (16, 8200, 2064), (2, 4500, 8192), (15, 4103, 4500), (16, 4096, 1200)])
def test_product_of_few_rows_with_many_weights(rows, n, k, dtype):
    """Up to a tile of rows with more weight rows than one workgroup a compute unit takes; the bytes behind each row are NaN, and so are those before the first and behind the last."""
    g = torch.Generator().manual_seed(rows + n + k)
    whole = lambda *shape: torch.randint(-4, 5, shape, generator=g).float().to(E4M3).to(DEV)      # noqa: E731
    powers = lambda *shape: torch.exp2(torch.randint(-1, 2, shape, generator=g).float()).to(DEV)  # noqa: E731
    a, w, sa, sw = whole(rows, k), whole(n, k), powers(blocks(k), rows), powers(blocks(n), blocks(k))
    bias = torch.randint(-9, 10, (n,), generator=g).float().to(DEV)
    want = ((a.double() * at_rows(sa, k)) @ (w.double() * at_weights(sw, n, k)).t() + bias).float()
    assert float(want.abs().max()) < 2 ** 14                         # whole numbers of quarters: fp32 has every sum exactly
    for stride, before in ((-(-k // 16) * 16, 16), (k, 0), (k + 5, 3)):
        got = pa.matmul_fp8(laid_out(a, stride, before), sa, laid_out(w, stride, before), sw, bias=bias, dtype=TORCH[dtype])
        assert torch.equal(got, want.to(TORCH[dtype]))
    latent = pa.matmul_fp8(a, sa, w, sw, bias=bias, dtype=TORCH[dtype], n_frames=1)
    assert torch.equal(latent, want.to(TORCH[dtype]).view(rows, n, 1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,n", [(420, 1104), (700, 1030), (1800, 1100), (1500, 2048), (2300, 2100)])
@pytest.mark.parametrize("k", [640, 700, 1152, 1279, 1291])
def test_product_of_operands_at_any_address(rows, n, k, dtype):
    """Every tile for operands that are not 16 bytes apart, K in one and in two groups of waves; what lies around the rows is NaN."""
    g = torch.Generator().manual_seed(rows + n + k)
    whole = lambda *shape: torch.randint(-4, 5, shape, generator=g).float().to(E4M3).to(DEV)      # noqa: E731
    powers = lambda *shape: torch.exp2(torch.randint(-1, 2, shape, generator=g).float()).to(DEV)  # noqa: E731
    a, w, sa, sw = whole(rows, k), whole(n, k), powers(blocks(k), rows), powers(blocks(n), blocks(k))
    want = ((a.float() * at_rows(sa, k)) @ (w.float() * at_weights(sw, n, k)).t()).to(TORCH[dtype])
    for stride, before in ((k | 1, 0), (k + 5, 3)):
        assert torch.equal(pa.matmul_fp8(laid_out(a, stride, before), sa, laid_out(w, stride, before), sw, dtype=TORCH[dtype]), want)
