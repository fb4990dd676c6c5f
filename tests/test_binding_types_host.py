"""The binding on a torch that does not have the types of 4-bit codes and of powers of two: everything else works, and so do bytes."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_PROGRAM = """
import torch
for name in ("float8_e8m0fnu", "float4_e2m1fn_x2"):
    if hasattr(torch, name):
        delattr(torch, name)
from paper_2407_08608_amd import binding
binding._native = None
x, i = torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((2, 2), dtype=torch.int32)
codes, powers = torch.zeros((4, 2, 16, 32), dtype=torch.uint8), torch.zeros((4, 2, 16, 2), dtype=torch.uint8)
# past the types, and refused for where the tensors are
for call in (lambda: binding.fa_fwd(x, x, x, 0.1, False), lambda: binding.fa_cache_write(x[:2], x[:2], x, x, i, i[0]), lambda: binding.fa_cache_read(x, x, i, i[0], 3),
             lambda: binding.fa_cache_copy(codes, codes, i[0], i[0], k_scales=powers, v_scales=powers), lambda: binding.fa_fwd_cache(x[:2], x, x, i, i[0], 0.1)):
    try:
        call()
    except ValueError as e:
        print(e)
    else:
        raise SystemExit("not refused")
print("done", binding._in_four_bits(codes, powers), binding._in_four_bits(codes, None), binding._in_four_bits(x, None))
"""


def test_a_torch_without_the_newest_types():
    r = subprocess.run([sys.executable, "-c", _PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=240)
    assert r.returncode == 0, r.stderr
    lines = r.stdout.strip().splitlines()
    assert lines[-1] == "done True False False" and len(lines) == 6 and all("device" in x or "cuda" in x.lower() for x in lines[:5]), lines
