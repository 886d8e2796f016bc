"""Arguments that do not fit are refused by the Python entry points also where Python runs without its assert statements (-O)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
import paper_2605_28657_amd as pa

E4M3 = torch.float8_e4m3fn
x, w = torch.zeros(4, 256), torch.ones(256)
a, sa, m, sm = torch.zeros(4, 200, dtype=E4M3), torch.zeros(2, 4), torch.zeros(8, 200, dtype=E4M3), torch.zeros(1, 2)
calls = [lambda: pa.quantize_fp8(x), lambda: pa.quantize_fp8(x.t()), lambda: pa.quantize_fp8(x[:, :255], gated=True),
         lambda: pa.quantize_fp8(x, out=(torch.zeros(4, 255, dtype=E4M3), torch.zeros(2, 4))),
         lambda: pa.rms_norm_fp8(x, w), lambda: pa.rms_norm_fp8(x, w[:255]), lambda: pa.rms_norm_fp8(x, w, residual=x[:3]),
         lambda: pa.rms_norm_fp8(x, w, sum_out=x[:, :255]), lambda: pa.quantize_weights_fp8(x), lambda: pa.quantize_weights_fp8(x, out=(m, sm)),
         lambda: pa.matmul_fp8(a, sa, m, sm), lambda: pa.matmul_fp8(a, sa, m[:, :199], sm), lambda: pa.matmul_fp8(a, sa[:1], m, sm),
         lambda: pa.matmul_fp8(a, sa, m, sm[:, :1]), lambda: pa.matmul_fp8(a, sa, m, sm, bias=w[:7]), lambda: pa.matmul_fp8(a, sa, m, sm, n_frames=3),
         lambda: pa.matmul_fp8(a, sa, m, sm, out=torch.zeros(4, 7)), lambda: pa.matmul_fp8(x, sa, m, sm),
         lambda: pa.latent_similarity(x, x), lambda: pa.latent_similarity(x, x[:3]), lambda: pa.crossfade(x, x)]
for i, call in enumerate(calls):
    try:
        call()
    except AssertionError:
        continue
    except Exception as e:
        sys.exit("call %d: %r" % (i, e))
    sys.exit("call %d was taken" % i)
print("refused", len(calls))
"""


def test_checks_do_not_go_with_the_assert_statements():
    for flags in ([], ["-O"]):
        done = subprocess.run([sys.executable, *flags, "-c", PROGRAM, ROOT], capture_output=True, text=True, timeout=300)
        assert done.returncode == 0 and done.stdout.strip() == "refused 21", (flags, done.stderr[-500:])
