"""desc.max_ctas bounds the CTAs of each attention kernel over the 8-bit cache (on the host, with the runtime faked: what
the launchers ask for), and a bounded call gives the same result."""
import os
import subprocess

import pytest

from kv8_util import check
from paper_2402_02082_gb300 import binding as gb
from paper_2402_02082_gb300 import build
from test_kv8_attn import call, expect, make

HERE = os.path.dirname(os.path.abspath(__file__))
# B, H, H_kv, D, keys, n, tree
CALLS = [(1, 2, 2, 128, 100, 1, 0), (4, 32, 32, 128, 4096, 1, 0), (2, 8, 2, 64, 3000, 5, 1), (4, 32, 8, 128, 16384, 33, 1),
         (8, 40, 40, 128, 2000, 26, 1), (1, 256, 1, 128, 5000, 1, 0), (2, 16, 4, 64, 700, 64, 1)]
BOUNDS = [1, 2, 3, 4, 7, 64, 151, 1000]


@pytest.mark.parametrize("source,launcher,f32", [("kv8_few.cu", "launch_kv8_few", 0),
                                                 ("kv8_attn_tc.cu", "launch_kv8_attn_tc", 0),
                                                 ("kv8_attn_fma.cu", "launch_kv8_attn_fma", 1)])
def test_ctas(tmp_path, source, launcher, f32):
    exe = str(tmp_path / "check")
    cmd = [build.nvcc(), "-gencode", "arch=compute_103a,code=compute_103a", "-std=c++17", "-O0",
           "--expt-relaxed-constexpr", "-I", build.CSRC, "-I", build.INCLUDE, "-I", HERE, f'-DSOURCE="{source}"',
           f"-DCALL={launcher}", os.path.join(HERE, "kv8_bound_check.cu"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    lines = [(*c, f32, most) for c in CALLS for most in BOUNDS]
    r = subprocess.run([exe], input="\n".join(" ".join(map(str, x)) for x in lines), capture_output=True, text=True,
                       timeout=60)
    got = [int(x) for x in r.stdout.split()]
    assert r.returncode == 0 and len(got) == len(lines)
    assert any(got)
    for (_, H, H_kv, _, _, n, _, _, most), ctas in zip(lines, got):
        rows = n * H // H_kv
        # a slab of more than 64 query rows is so many row tiles, side by side
        least = -(-rows // 64) if source == "kv8_attn_tc.cu" else 1
        assert ctas <= max(most, least), (H, H_kv, n, most, ctas)
        assert ctas > 0 or source == "kv8_few.cu"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv,n", [(3, 3, 1), (4, 2, 9), (8, 2, 33)])
def test_results(dtype, H, H_kv, n):
    build.build()
    gb.lib()
    c = make(H + n, 2, H, H_kv, 128, [700, 41], n, dtype, n > 1)
    want = expect(c)
    for max_ctas in (1, 2, 3, 5, 8, 1000):
        check(call(c, max_ctas=max_ctas), *want, dtype)
