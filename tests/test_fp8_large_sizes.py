"""Sizes of 2^31 and more of the 8-bit operators are refused as they are, not as what is left of them in 32 bits.  Nothing here has memory behind it."""
import pytest
import torch

import paper_2605_28657_amd as pa

E4M3, P, BIG = torch.float8_e4m3fn, 4096, [1 << 31, (1 << 32) + 1, (1 << 32) + 5]


def _rows(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def _product(rows, n, k, **more):
    blocks = -(-k // 128)
    return pa.matmul_fp8(_rows(rows, k, dtype=E4M3), _rows(blocks, rows, dtype=torch.float32), _rows(n, k, dtype=E4M3),
                         _rows(-(-n // 128), blocks, dtype=torch.float32), **more)


@pytest.mark.parametrize("big", BIG)
def test_tensors_are_refused(big):
    calls = [lambda: pa.quantize_fp8(_rows(1, big)), lambda: pa.quantize_fp8(_rows(big, 1)), lambda: pa.quantize_fp8(_rows(1, 2 * big), gated=True),
             lambda: pa.quantize_fp8(_rows(1, 128).expand(big, 128)),
             lambda: pa.rms_norm_fp8(_rows(1, big), _rows(big, dtype=torch.float32)), lambda: pa.rms_norm_fp8(_rows(big, 1), _rows(1, dtype=torch.float32)),
             lambda: pa.quantize_weights_fp8(_rows(1, big)), lambda: pa.quantize_weights_fp8(_rows(big, 1)),
             lambda: _product(big, 1, 1), lambda: _product(1, big, 1), lambda: _product(1, 1, big), lambda: _product(1, 1, big, fp32_sums=True)]
    for call in calls:
        with pytest.raises(pa.DemonError) as e:
            call()
        assert e.value.status == pa.DEMON_ERR_UNSUPPORTED


@pytest.mark.parametrize("big", BIG)
def test_sizes_are_refused(big):
    product = [P, 16, P, 1 << 40, P, 16, P, 0, 4, 4, 4, 0, pa.DEMON_BF16, P, 1 << 40]
    calls = [(pa.demon_vae_quantize_fp8, [P, 0, 4, 4, 0, pa.DEMON_F32, P, 1 << 40, P, 1 << 40], (2, 3)),
             (pa.demon_vae_rms_norm_fp8, [P, 0, 0, 0, P, 4, 4, 1e-6, pa.DEMON_F32, 0, 0, P, 1 << 40, P, 1 << 40], (5, 6)),
             (pa.demon_vae_quantize_weights_fp8, [P, 0, 4, 4, pa.DEMON_F32, P, 1 << 40, P], (2, 3)),
             (pa.demon_vae_matmul_fp8, product, (8, 9, 10, 11)), (pa.demon_vae_matmul_fp8_fp32_sums, product, (8, 9, 10, 11))]
    for fn, args, sizes in calls:
        for i in sizes:
            with pytest.raises(pa.DemonError) as e:
                fn(*args[:i], big, *args[i + 1:])
            assert e.value.status == pa.DEMON_ERR_UNSUPPORTED
