"""Products of more outputs than one launch has threads for are UNSUPPORTED, whatever kernel they would take.  Every call here is refused before a launch."""
import ctypes

import pytest

import paper_2605_28657_amd as pa

P = ctypes.c_void_p(4096)          # never read
FAR = 1 << 22


@pytest.mark.parametrize("entry", ["demon_vae_matmul_fp8", "demon_vae_matmul_fp8_fp32_sums"])
@pytest.mark.parametrize("dtype", [pa.DEMON_BF16, pa.DEMON_F32])
@pytest.mark.parametrize("rows,n,k,a_stride,w_stride", [
    (1 << 24, 1 << 24, 256, 256, 256), (1 << 24, 1 << 24, 100, 100, 100), (1 << 24, 1 << 24, 256, 257, 256),
    (1 << 20, 1 << 12, 256, FAR, 256), (1 << 20, 1 << 12, 256, 256, FAR), ((1 << 20) - 15, (1 << 12) - 31, 256, FAR, FAR), (1 << 24, 1 << 24, 1 << 24, 1 << 24, 1 << 24)])
def test_too_many_outputs(entry, dtype, rows, n, k, a_stride, w_stride):
    rc = getattr(pa.load_library(), entry)(P, a_stride, P, rows, P, w_stride, P, None, rows, n, k, 0, dtype, P, n, None)
    assert rc == pa.DEMON_ERR_UNSUPPORTED and "outputs" in pa.demon_vae_last_error()


@pytest.mark.parametrize("change,status", [
    (dict(a=None), 1), (dict(a_scale=None), 1), (dict(w=None), 1), (dict(w_scale=None), 1), (dict(out=None), 1), (dict(rows=0), 1), (dict(n=0), 1), (dict(k=-1), 1),
    (dict(dtype=2), 1), (dict(a_stride=-1), 1), (dict(w_stride=-1), 1), (dict(a_scale_stride=3), 1), (dict(out_stride=7), 1), (dict(n_frames=-1), 1), (dict(n_frames=3), 1),
    (dict(k=(1 << 24) + 1), 2), (dict(rows=(1 << 24) + 1, a_scale_stride=1 << 25), 2), (dict(n=(1 << 24) + 1, out_stride=1 << 25), 2)])
def test_fp32_sums_refuse_what_the_product_refuses(change, status):
    given = dict(a=P, a_stride=256, a_scale=P, a_scale_stride=4, w=P, w_stride=256, w_scale=P, bias=None, rows=4, n=8, k=256, n_frames=0, dtype=pa.DEMON_BF16,
                 out=P, out_stride=8, stream=None)
    for entry in (pa.load_library().demon_vae_matmul_fp8, pa.load_library().demon_vae_matmul_fp8_fp32_sums):
        assert entry(*dict(given, **change).values()) == status and pa.demon_vae_last_error()
