"""What the launches of the real-valued ends' calls read and write, on the CPU: tests/host/real_ends_extents.cpp takes the HIP runtime's
place and follows every launch of the host code (built with AddressSanitizer and UBSan) through the workspace and the outputs."""
import os
import subprocess

import pytest

from paper_1804_02941_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def follow(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("extents") / "real_ends_extents")
    flags = [f for f in build.FLAGS if f not in ("-shared", "-fPIC") and not f.startswith("-Rpass")]
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-g",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-I", os.path.join(ROOT, "include"), "-I", build.CSRC,
           *[os.path.join(build.CSRC, s) for s in ("head.hip", "product16.hip", "small32.hip", "w4.hip")],
           os.path.join(ROOT, "tests", "host", "real_ends_extents.cpp"), "-o", exe]
    p = subprocess.run(cmd, capture_output=True, text=True)
    assert p.returncode == 0, p.stdout[-3000:] + p.stderr[-3000:]

    def run(*args):
        p = subprocess.run([exe, *map(str, args)], capture_output=True, text=True, timeout=600)
        assert p.returncode == 0, p.stdout[-3000:] + p.stderr[-3000:]
        return p.stdout
    return run


# Heads of bf16 and fp32 whose gradient's products are large tiles with a last round that is not full, some with room for shares of
# one product, of a full piece or of none: several pieces, one piece, up to 128 tokens.
HEADS = [(8192, 2048, 50257, BF16), (2048, 8192, 128256, BF16), (2048, 7168, 128256, BF16), (6144, 5120, 131072, BF16), (1632, 3796, 6071, BF16),
         (2048, 6144, 128000, F32), (65, 8256, 4097, BF16), (1162, 2832, 7768, BF16), (215, 4071, 1024, BF16), (7731, 2365, 1168, BF16),
         (8192, 2048, 50304, BF16), (8192, 2048, 131072, BF16), (2048, 4096, 32768, BF16), (1999, 1000, 50021, BF16), (256, 512, 250, F32)]


@pytest.mark.parametrize("sizes", HEADS)
def test_a_head_stays_within_its_workspace(follow, sizes):
    follow("head", *sizes)


@pytest.mark.parametrize("seed", [1, 2, 3])
def test_calls_of_any_size_stay_within_their_workspaces(follow, seed):
    assert " 0 faults" in follow(20000, seed)
