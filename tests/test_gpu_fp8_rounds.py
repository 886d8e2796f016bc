"""8-bit products of more of the largest tiles than there are compute units, where K is two blocks of which the second one is cut: a tile's requests for the next tile begin
in its first block and leave out the pieces behind K in its second."""
import pytest
import torch

import paper_2605_28657_amd as pa
from fp8_util import E4M3, at_rows, at_weights, blocks, laid_out

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("rows,n", [(8200, 8200), (9000, 4200), (4097, 16400)])
@pytest.mark.parametrize("k", [144, 240, 272])
def test_product(rows, n, k):
    g = torch.Generator().manual_seed(rows + n + k)
    whole = lambda *shape: torch.randint(-4, 5, shape, generator=g).float().to(E4M3).to(DEV)      # noqa: E731
    powers = lambda *shape: torch.exp2(torch.randint(-1, 2, shape, generator=g).float()).to(DEV)  # noqa: E731
    a, w, sa, sw = whole(rows, k), whole(n, k), powers(blocks(k), rows), powers(blocks(n), blocks(k))
    bias = torch.randint(-9, 10, (n,), generator=g).float().to(DEV)
    want = (a.float() * at_rows(sa, k)) @ (w.float() * at_weights(sw, n, k)).t()
    assert float(want.abs().max()) < 2 ** 14                         # quarters: fp32 has every sum exactly
    av, wv = laid_out(a, k + 16, 16), laid_out(w, k + 16, 16)        # the bytes behind each row are NaN
    for b in (None, bias):
        for _ in range(2):
            assert torch.equal(pa.matmul_fp8(av, sa, wv, sw, bias=b), (want if b is None else want + b).bfloat16())
