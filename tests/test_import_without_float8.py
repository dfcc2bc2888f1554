"""The package on a torch that lacks the 8-bit cache's types: everything but Kv8Pool works."""
import os
import subprocess
import sys

PROGRAM = """
import torch
for name in ("float8_e4m3fn", "float8_e8m0fnu"):
    if hasattr(torch, name):
        delattr(torch, name)
import paper_2609_27233_gb300 as umim
assert umim.umim_decode_attention and umim.paged_kv
for make in (lambda: umim.Kv8Pool.zeros(1, 2, 1, 64, "cpu"),
             lambda: umim.Kv8Pool(torch.zeros((1, 2, 2, 1, 16, 64)), torch.zeros((1, 2, 2, 1, 16)))):
    try:
        make()
    except RuntimeError as e:
        assert "float8" in str(e), e
    else:
        raise AssertionError("made a cache without its types")
print("fine")
"""


def test_import_without_the_8_bit_types():
    root = os.path.join(os.path.dirname(os.path.abspath(__file__)), os.pardir)
    p = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout.strip() == "fine", p.stderr
