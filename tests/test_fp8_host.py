"""The 8-bit operators without a GPU: refused arguments (checked before anything is launched) and tensors that are not on a GPU."""
import ctypes

import pytest
import torch

import paper_2605_28657_amd as pa

INVALID, UNSUPPORTED = pa.DEMON_ERR_INVALID_ARG, pa.DEMON_ERR_UNSUPPORTED
P = ctypes.c_void_p(4096)          # never read: every call here is refused before a launch


def _call(name, given, change):
    args = dict(given, **change)
    fn = getattr(pa.load_library(), name)
    assert set(args) == set(given)
    rc = fn(*args.values())
    return rc, pa.demon_vae_last_error()


QUANTIZE = dict(x=P, x_stride=256, rows=4, channels=256, gated=0, dtype=pa.DEMON_BF16, q=P, q_stride=256, scale=P, scale_stride=4, stream=None)
NORM = dict(x=P, x_stride=256, residual=P, residual_stride=256, weight=P, rows=4, channels=256, eps=1e-6, dtype=pa.DEMON_BF16, sum=P, sum_stride=256,
            q=P, q_stride=256, scale=P, scale_stride=4, stream=None)
WEIGHTS = dict(w=P, w_stride=256, n=4, k=256, dtype=pa.DEMON_F32, q=P, q_stride=256, scale=P, stream=None)
MATMUL = dict(a=P, a_stride=256, a_scale=P, a_scale_stride=4, w=P, w_stride=256, w_scale=P, bias=None, rows=4, n=8, k=256, n_frames=0,
              dtype=pa.DEMON_BF16, out=P, out_stride=8, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(rows=0), INVALID), (dict(rows=-1), INVALID),
    (dict(channels=0), INVALID), (dict(dtype=2), INVALID), (dict(dtype=-1), INVALID), (dict(x_stride=-1), INVALID), (dict(q_stride=255), INVALID),
    (dict(scale_stride=3), INVALID), (dict(channels=(1 << 24) + 1, q_stride=1 << 25), UNSUPPORTED), (dict(rows=1 << 22, scale_stride=1 << 22), UNSUPPORTED)])
def test_quantize_refuses(change, status):
    rc, message = _call("demon_vae_quantize_fp8", QUANTIZE, change)
    assert rc == status and message


@pytest.mark.parametrize("change,status", [
    (dict(x=None), INVALID), (dict(weight=None), INVALID), (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(rows=0), INVALID),
    (dict(channels=0), INVALID), (dict(dtype=7), INVALID), (dict(eps=-1e-6), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(eps=float("inf")), INVALID), (dict(x_stride=-256), INVALID), (dict(residual_stride=-256), INVALID), (dict(sum_stride=255), INVALID),
    (dict(x_stride=512), INVALID),                                      # sum in place of x with another stride
    (dict(x=ctypes.c_void_p(8192), residual_stride=512), INVALID),      # the same for the residual
    (dict(q_stride=1), INVALID), (dict(scale_stride=0), INVALID),
    (dict(rows=1 << 22, scale_stride=1 << 22), UNSUPPORTED), (dict(channels=32769, x_stride=32769, residual_stride=32769, sum_stride=32769, q_stride=32769), UNSUPPORTED)])
def test_norm_refuses(change, status):
    rc, message = _call("demon_vae_rms_norm_fp8", NORM, change)
    assert rc == status and message


@pytest.mark.parametrize("change,status", [
    (dict(w=None), INVALID), (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(n=0), INVALID), (dict(k=0), INVALID), (dict(dtype=2), INVALID),
    (dict(w_stride=-1), INVALID), (dict(q_stride=255), INVALID), (dict(n=(1 << 24) + 1), UNSUPPORTED),
    (dict(n=1 << 24, k=1 << 24, q_stride=1 << 24), UNSUPPORTED), (dict(n=1 << 19, k=1 << 19, q_stride=1 << 19), UNSUPPORTED)])
def test_weights_refuse(change, status):
    rc, message = _call("demon_vae_quantize_weights_fp8", WEIGHTS, change)
    assert rc == status and message


@pytest.mark.parametrize("change,status", [
    (dict(a=None), INVALID), (dict(a_scale=None), INVALID), (dict(w=None), INVALID), (dict(w_scale=None), INVALID), (dict(out=None), INVALID),
    (dict(rows=0), INVALID), (dict(n=0), INVALID), (dict(k=0), INVALID), (dict(dtype=2), INVALID), (dict(a_stride=-1), INVALID),
    (dict(w_stride=-1), INVALID), (dict(a_scale_stride=3), INVALID), (dict(out_stride=7), INVALID), (dict(n_frames=-1), INVALID),
    (dict(n_frames=3), INVALID), (dict(n_frames=8), INVALID), (dict(k=(1 << 24) + 1), UNSUPPORTED),
    (dict(rows=(1 << 24) + 1, a_scale_stride=1 << 25), UNSUPPORTED), (dict(n=(1 << 24) + 1, out_stride=1 << 25), UNSUPPORTED)])
def test_matmul_refuses(change, status):
    rc, message = _call("demon_vae_matmul_fp8", MATMUL, change)
    assert rc == status and message


def test_tensors_that_are_not_on_a_gpu_are_refused():
    x = torch.zeros(4, 256)
    q = torch.zeros(4, 256, dtype=torch.float8_e4m3fn)
    s = torch.zeros(2, 4)
    with pytest.raises(AssertionError):
        pa.quantize_fp8(x)
    with pytest.raises(AssertionError):
        pa.rms_norm_fp8(x, torch.ones(256))
    with pytest.raises(AssertionError):
        pa.quantize_weights_fp8(x)
    with pytest.raises(AssertionError):
        pa.matmul_fp8(q, s, q, torch.zeros(1, 2))
    with pytest.raises(KeyError):
        pa.quantize_fp8(x.half())


def test_kernels_keep_their_sums_in_registers():
    """Sums and operands of the products live in registers; in scratch memory they would make a round trip in every block of K."""
    from test_kernel_sources import _resources
    res = {n: r for n, r in _resources().items() if "matmul_" in n or "rms_norm_kernel" in n or "quantize_" in n}
    assert len(res) > 40
    assert {n: r for n, r in res.items() if r != (0, 0)} == {}
