"""The compiler's report on the 8-bit products: their register splits are chosen so that (almost) nothing spills."""
import os
import re
import subprocess

from paper_1705_09056_b200 import build


def test_products_of_8_bit_layers_do_not_spill(tmp_path):
    src = os.path.join(build.CSRC, "fp8_linear.cu")
    flags = [f for f in build.FLAGS if not f.startswith("--use_fast_math")]
    r = subprocess.run([build._nvcc(), *flags, "-Xptxas", "-v", "-c", src, "-o", str(tmp_path / "x.o")], stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    found = re.findall(r"Function properties for (\S*fp8_gemm_kernel\S*)\s+\d+ bytes stack frame, (\d+) bytes spill stores, (\d+)", r.stdout)
    assert len(found) >= 8
    for name, stores, loads in found:
        most = 4 if "ILi0ELi256ELb1E" in name else 0          # the pair of CTAs: one register
        assert int(stores) <= most and int(loads) <= most, (name, stores, loads)
