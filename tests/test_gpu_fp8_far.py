"""8-bit products whose operands' or outputs' rows lie as far apart as their kernels' offsets reach, and further."""
import pytest
import torch

import paper_2605_28657_amd as pa
from fp8_util import E4M3, at_rows, at_weights, blocks

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FAR = 1 << 22                       # from here on tiles of 256 rows are not taken: their offsets have 32 bits


def _whole(rows, n, k):
    g = torch.Generator().manual_seed(rows + n + k)
    whole = lambda *shape: torch.randint(-4, 5, shape, generator=g).float().to(E4M3).to(DEV)      # noqa: E731
    powers = lambda *shape: torch.exp2(torch.randint(-1, 2, shape, generator=g).float()).to(DEV)  # noqa: E731
    a, w, sa, sw = whole(rows, k), whole(n, k), powers(blocks(k), rows), powers(blocks(n), blocks(k))
    want = (a.float() * at_rows(sa, k)) @ (w.float() * at_weights(sw, n, k)).t()
    assert float(want.abs().max()) < 2 ** 14                         # quarters: fp32 has every sum exactly
    return a, sa, w, sw, want


def _apart(q, stride, before=0):
    """q's rows `stride` bytes apart, NaN before and behind each."""
    rows, k = q.shape
    store = torch.empty(before + 16 + stride * (rows - 1) + k + 16, dtype=torch.uint8, device=DEV)
    torch.as_strided(store, (rows, k + 32), (stride, 1), before).fill_(0x7f)
    view = torch.as_strided(store, (rows, k), (stride, 1), before + 16)
    view.copy_(q.view(torch.uint8))
    return view.view(E4M3)


@pytest.mark.parametrize("a_stride,w_stride,before", [
    (FAR - 16, FAR - 16, 0), (FAR - 16, 416, 0), (416, FAR - 16, 0), (FAR - 15, FAR - 15, 3), (FAR - 1, 417, 0), (417, FAR - 1, 0),
    (FAR, FAR, 0), (FAR + 16, 416, 0), (416, FAR + 16, 0), (FAR + 1, FAR + 3, 1)])
def test_operands(a_stride, w_stride, before):
    """Sizes that take tiles where the rows lie near each other; the first and the last weight row are 4.6 GB apart."""
    rows, n, k = 272, 1100, 384
    a, sa, w, sw, want = _whole(rows, n, k)
    av, wv = _apart(a, a_stride, before), _apart(w, w_stride, before)
    for kw in (dict(), dict(fp32_sums=True), dict(dtype=torch.float32)):
        assert torch.equal(pa.matmul_fp8(av, sa, wv, sw, **kw), want.to(kw.get("dtype", torch.bfloat16)))


@pytest.mark.parametrize("a_stride,w_stride", [(FAR - 16, 144), (144, FAR - 16)])
def test_operands_of_the_largest_tiles(a_stride, w_stride):
    """256 rows a tile at the largest stride, in one launch whose rows end 17 GB behind the first; K ends inside its second block."""
    rows, n, k = 4100, 4090, 144
    a, sa, w, sw, want = _whole(rows, n, k)
    av, wv = (_apart(a, a_stride) if a_stride >= FAR - 16 else a), (_apart(w, w_stride) if w_stride >= FAR - 16 else w)
    assert torch.equal(pa.matmul_fp8(av, sa, wv, sw), want.bfloat16())


@pytest.mark.parametrize("rows,n,k,stride", [(272, 1100, 384, 1 << 23), (272, 1100, 384, (1 << 23) + 3), (4100, 4090, 256, 1 << 20), (4100, 4090, 200, (1 << 20) + 1)])
def test_outputs(rows, n, k, stride):
    """The last output row more than 4 GB behind the first, from tiles; what lies beside a row stays."""
    a, sa, w, sw, want = _whole(rows, n, k)
    store = torch.empty((rows - 1) * stride + n + 8, dtype=torch.bfloat16, device=DEV)
    around = torch.as_strided(store, (rows, n + 8), (stride, 1))
    for kw in (dict(), dict(fp32_sums=True)):
        around.fill_(-7)
        pa.matmul_fp8(a, sa, w, sw, out=around[:, 4:4 + n], **kw)
        assert torch.equal(around[:, 4:4 + n], want.bfloat16())
        assert bool((around[:, :4] == -7).all()) and bool((around[:, 4 + n:] == -7).all())
