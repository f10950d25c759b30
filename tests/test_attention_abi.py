"""Host-side checks of the attention entry points: bad arguments are refused before anything is launched, the binding refuses what does not
belong together, and the front end runs clean under the host sanitizers.  No GPU."""
import math
import os
import subprocess

import pytest
import torch

from paper_2505_14638_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests", "host_sanitizer")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
P = 0x10000          # a non-NULL, aligned dummy address; never dereferenced on the paths tested here
OK, NULL, SHAPE, DTYPE, ALIGN, WORKSPACE = 0, 1, 2, 4, 6, 7


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(B.LIB_PATH):
        from paper_2505_14638_amd import build
        build.build()
    return B.lib()


def caller(f, order, ok):
    assert list(ok) == order.split()
    return lambda **kw: f(*{**ok, **kw}.values())


def test_rope_cache_write_refusals(L):
    ok = dict(qkv=P, T=0, ldqkv=1024, H=4, HK=2, D=128, table=P, rows=100, rope=0, positions=P, slots=P, q=P, ldq=512, k=P, ldk=256, kc=P, vc=P,
              dtype=0, scales=P, pages=10, stride=4096, page=16, stream=None)
    call = caller(L.w4a8_rope_cache_write, " ".join(ok), ok)
    assert call() == OK                                          # no tokens: nothing to do
    live = dict(T=3)
    for key in ("qkv", "table", "positions", "slots", "q", "kc", "vc"):
        assert call(**live, **{key: 0}) == NULL, key
    assert call(**live, dtype=1, scales=0) == NULL
    assert call(rope=2) == DTYPE and call(rope=-1) == DTYPE and call(dtype=2) == DTYPE
    assert call(D=96) == SHAPE and call(D=256) == SHAPE and call(H=5) == SHAPE and call(H=1) == SHAPE and call(HK=0) == SHAPE and call(HK=-2) == SHAPE
    assert call(page=8) == SHAPE and call(page=48) == SHAPE and call(page=2048) == SHAPE and call(pages=0) == SHAPE
    assert call(pages=1 << 27) == SHAPE and call(stride=4095) == SHAPE and call(stride=4100) == ALIGN and call(dtype=1, stride=4104) == ALIGN
    assert call(T=-1) == SHAPE and call(T=(1 << 24) + 1) == SHAPE and call(rows=0) == SHAPE
    assert call(**live, ldqkv=1016) == SHAPE and call(**live, ldqkv=1028) == ALIGN and call(**live, ldqkv=1 << 20) == SHAPE
    assert call(**live, ldq=504) == SHAPE and call(**live, ldk=248) == SHAPE and call(**live, qkv=P + 8) == ALIGN
    for key in ("table", "kc", "vc", "q", "k"):
        assert call(**live, **{key: P + 8}) == ALIGN, key
    for key in ("positions", "slots", "scales"):
        assert call(**live, **{key: P + 2}) == ALIGN, key


def test_attention_prompt_refusals(L):
    ok = dict(q=P, ldq=512, k=P, ldk=256, v=P, ldv=256, starts=P, n=0, T=5, H=4, HK=2, D=128, causal=1, scale=0.1, y=P, ldy=512, y_scale=None,
              stream=None)
    call = caller(L.w4a8_attention_prompt, " ".join(ok), ok)
    assert call() == OK and call(n=1, T=0) == OK
    live = dict(n=1)
    for key in ("q", "k", "v", "starts", "y"):
        assert call(**live, **{key: 0}) == NULL, key
    assert call(D=32) == SHAPE and call(H=3) == SHAPE and call(HK=0) == SHAPE and call(H=8192) == SHAPE
    assert call(causal=2) == DTYPE
    for scale in (0.0, -1.0, math.inf, math.nan, 1e31):
        assert call(scale=scale) == SHAPE, scale
    assert call(n=-1) == SHAPE and call(T=-1) == SHAPE and call(T=(1 << 24) + 1) == SHAPE and call(n=1 << 20, H=64) == SHAPE
    for key in ("ldq", "ldk", "ldv", "ldy"):
        assert call(**live, **{key: 128}) == SHAPE and call(**live, **{key: 516}) == ALIGN and call(**live, **{key: 1 << 20}) == SHAPE, key
    assert call(**live, ldy=520, y_scale=P) == ALIGN             # bytes here
    for key in ("q", "k", "v", "y"):
        assert call(**live, **{key: P + 8}) == ALIGN, key
    assert call(**live, starts=P + 2) == ALIGN and call(**live, y_scale=P + 1) == ALIGN


def test_attention_decode_refusals(L):
    ok = dict(q=P, ldq=512, n=0, H=4, HK=2, D=128, kc=P, vc=P, dtype=0, scales=P, pages=10, stride=4096, page=16, tables=P, width=4, ld=4, lengths=P,
              prefix_pages=P, prefix=0, scale=0.1, y=P, ldy=512, y_scale=None, ws=P, ws_bytes=1 << 40, stream=None)
    call = caller(L.w4a8_attention_decode, " ".join(ok), ok)
    assert call() == OK
    live = dict(n=2, prefix=20)
    for key in ("q", "kc", "vc", "tables", "lengths", "prefix_pages", "y", "ws"):
        assert call(**live, **{key: 0}) == NULL, key
    assert call(**live, dtype=1, scales=0) == NULL
    assert call(D=96) == SHAPE and call(H=3) == SHAPE and call(page=24) == SHAPE and call(dtype=7) == DTYPE and call(scale=-1.0) == SHAPE
    assert call(n=-1) == SHAPE and call(n=1 << 17) == SHAPE and call(width=-1) == SHAPE and call(width=1 << 27, ld=1 << 27) == SHAPE
    assert call(ld=3) == SHAPE and call(prefix=-1) == SHAPE and call(prefix=1 << 31) == SHAPE
    assert call(stride=4095) == SHAPE and call(stride=4100) == ALIGN
    assert call(**live, ldq=516) == ALIGN and call(**live, ldy=504) == SHAPE and call(**live, q=P + 2) == ALIGN and call(**live, ws=P + 8) == ALIGN
    for key in ("tables", "lengths", "prefix_pages", "scales", "y_scale"):
        assert call(**live, **{key: P + 2}) == ALIGN, key
    need = L.w4a8_attention_decode_workspace_bytes(2, 4, 2, 128, 16, 4, 20)
    assert need > 0 and need % 16 == 0 and call(**live, ws_bytes=need - 1) == WORKSPACE


def test_attention_decode_workspace(L):
    f = B.attention_decode_workspace_bytes
    assert f(0, 4, 2, 128, 16, 4) == 0 and f(2, 3, 2, 128, 16, 4) == 0 and f(2, 4, 2, 128, 17, 4) == 0
    assert f(4096, 32, 8, 128, 16, 8) == 0                       # enough sequences: every row is finished by one workgroup
    row = (128 + 2) * 4
    for n in (1, 7, 64, 500):
        for width in (1, 3, 100, 4000):
            for prefix in (0, 1, 5000, 100000):
                need = f(n, 32, 8, 128, 16, width, prefix)
                assert need % (n * 32 * row) == 0 and need // (n * 32 * row) <= 128
                assert prefix == 0 or need >= 2 * n * 32 * row    # the prefix's part and the sequence's own


def test_cache_copy_pages_refusals(L):
    ok = dict(cache=P, planes=2, plane_stride=1 << 16, pages=8, stride=4096, size=4096, src=P, dst=P, n=0, stream=None)
    call = caller(L.w4a8_cache_copy_pages, " ".join(ok), ok)
    assert call() == OK and call(n=3, planes=0) == OK
    for key in ("cache", "src", "dst"):
        assert call(n=1, **{key: 0}) == NULL, key
    assert call(planes=-1) == SHAPE and call(planes=65536) == SHAPE and call(pages=0) == SHAPE and call(n=9) == SHAPE and call(n=-1) == SHAPE
    assert call(size=0) == SHAPE and call(stride=4080) == SHAPE and call(plane_stride=-16) == SHAPE and call(stride=1 << 50) == SHAPE
    assert call(size=4088) == ALIGN and call(stride=4104) == ALIGN and call(plane_stride=8) == ALIGN
    assert call(n=1, cache=P + 8) == ALIGN and call(n=1, src=P + 2) == ALIGN


def test_binding_refuses_what_does_not_belong_together(L):
    def bf(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16)

    def i32(*values):
        return torch.tensor(values, dtype=torch.int32)

    q, k, cache = bf(6, 4, 64), bf(6, 2, 64), bf(5, 2, 16, 64)
    for bad in (lambda: B.attention_prompt(q, k, k, i32(0, 6)),                                    # not on a GPU
                lambda: B.attention_prompt(q.float(), k, k, i32(0, 6)),
                lambda: B.attention_prompt(q, k, bf(6, 4, 64), i32(0, 6)),
                lambda: B.attention_prompt(q, bf(5, 2, 64), bf(5, 2, 64), i32(0, 6)),
                lambda: B.attention_prompt(q.transpose(1, 2).contiguous().transpose(1, 2), k, k, i32(0, 6)),
                lambda: B.attention_prompt(q, k, k, torch.tensor([0, 6])),
                lambda: B.attention_prompt(q, k, k, i32()),
                lambda: B.attention_decode(q, cache, cache, i32(0), i32(1)),
                lambda: B.attention_decode(q, cache, cache[:4], i32(*range(6)).view(6, 1), i32(*range(6))),
                lambda: B.attention_decode(q, cache, cache, i32(*range(6)).view(6, 1), i32(1)),
                lambda: B.attention_decode(q, cache.to(torch.uint8), cache.to(torch.uint8), i32(*range(6)).view(6, 1), i32(*range(6))),   # no scales
                lambda: B.attention_decode(q, cache, cache, i32(*range(6)).view(6, 1), i32(*range(6)), prefix_pages=i32(0), prefix_length=17),
                lambda: B.attention_decode(q, cache.transpose(1, 2), cache.transpose(1, 2), i32(*range(6)).view(6, 1), i32(*range(6))),
                lambda: B.rope_cache_write(bf(6, 500), torch.zeros(9, 64), i32(*range(6)), i32(*range(6)), cache, cache),
                lambda: B.rope_cache_write(bf(6, 512), torch.zeros(9, 32), i32(*range(6)), i32(*range(6)), cache, cache),
                lambda: B.rope_cache_write(bf(6, 512), torch.zeros(9, 64), i32(*range(5)), i32(*range(6)), cache, cache),
                lambda: B.cache_copy_pages(bf(2, 5, 16, 64).transpose(2, 3), i32(0), i32(1)),
                lambda: B.cache_copy_pages(bf(2, 5, 16, 64), i32(0), i32(1, 2))):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
def test_front_end_under_address_and_undefined_behavior_sanitizers(tmp_path):
    exe = str(tmp_path / "attention_driver")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", os.path.join(ROOT, "paper_2505_14638_amd", "csrc", "api_attention.hip"),
           os.path.join(HERE, "attention_driver.cpp"), "-o", exe]
    build = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=600)
    assert build.returncode == 0, build.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0")        # the HIP runtime's own start-up allocations are not ours
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=120, env=env)
    assert run.returncode == 0 and "all checks passed" in run.stdout, run.stdout[-4000:]
