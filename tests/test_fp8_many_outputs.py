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
