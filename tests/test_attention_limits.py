"""Calls at the limits of a launch and of a workspace: 2^32 threads do not fit one, and are refused before anything is enqueued.  No GPU."""
import os
import subprocess

import pytest
import torch

from paper_2505_14638_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
P = 0x10000          # a non-NULL, aligned dummy address; never dereferenced on the paths tested here
SHAPE = 2


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_14638_amd import build
        build.build()
    return B.lib()


def test_launches_of_two_to_the_32_threads_are_refused(L):
    # 2^24 pages of 16 bytes, each a workgroup of its own
    assert L.w4a8_cache_copy_pages(P, 1, 0, 1 << 24, 16, 16, P, P, 1 << 24, None) == SHAPE
    # 2^20 sequences of 16 heads, a workgroup each at least
    assert L.w4a8_attention_prompt(P, 2048, P, 128, P, 128, P, 1 << 20, 1, 16, 1, 128, 1, 0.1, P, 2048, None, None) == SHAPE
    # 2^23 tokens of 128 heads, four threads a head
    assert L.w4a8_rope_cache_write(P, 8192, 1 << 23, 64, 32, 64, P, 100, 0, P, P, P, 4096, None, 0, P, P, 0, None, 1 << 24, 32 * 16 * 64, 16, None) == SHAPE


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_every_accepted_launch_fits(tmp_path):
    """The front end with stubs in the place of the launchers: sizes on either side of the limits, grids as the launchers form them."""
    exe = str(tmp_path / "attention_limits")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", os.path.join(ROOT, "paper_2505_14638_amd", "csrc", "api_attention.hip"),
           os.path.join(ROOT, "tests", "host_sanitizer", "attention_limits.cpp"), "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert build.returncode == 0, build.stdout[-4000:]
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120)
    assert run.returncode == 0 and "all checks passed" in run.stdout, run.stdout[-4000:]


def test_a_workspace_with_holes_is_refused(L):
    """Every second byte of a buffer, and one byte seen many times, have fewer bytes behind their address than elements."""
    q, cache = torch.zeros((2, 4, 64), dtype=torch.bfloat16), torch.zeros((5, 2, 16, 64), dtype=torch.bfloat16)
    tables, lengths = torch.zeros((2, 1), dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    for work in (torch.zeros(1 << 16, dtype=torch.uint8)[::2], torch.zeros(1, dtype=torch.uint8).expand(1 << 16)):
        with pytest.raises(ValueError, match="workspace"):
            B.attention_decode(q, cache, cache, tables, lengths, workspace=work)
