"""Host side of fls_quantize and fls_fp8_gemm: sizes and refusals, before anything is launched.  Needs no GPU."""
import os

import pytest


@pytest.fixture(scope="module")
def fls():
    import paper_2309_10285_amd as f
    from paper_2309_10285_amd import _build

    if not os.path.exists(f.LIB_PATH):
        _build.build()
    return f


def test_sizes(fls):
    assert [fls.scale_stride(k) for k in (16, 128, 512, 528, 7168)] == [4, 4, 4, 8, 56]
    # control area, 64 MiB of sums, X in e4m3 (up to 64 columns: whole steps of 128 k for 16, 32 or 64), its scales
    assert fls.fls_fp8_workspace_bytes(1024, 1024, 8) == (4 << 20) + (64 << 20) + 16 * 1024 + 64
    assert fls.fls_fp8_workspace_bytes(1, 16, 33) == (4 << 20) + (64 << 20) + 64 * 128 + 144
    assert fls.fls_fp8_workspace_bytes(1000, 1040, 65) == (4 << 20) + (64 << 20) + 65 * 1040 + 784
    for M, K, N in ((0, 16, 1), (1, 0, 1), (1, 24, 1), (1, 8, 1), (1, 16, 0), (1, 16, 8193), ((1 << 21) + 1, 16, 1), (1, (1 << 22) + 16, 1),
                    (128, 1 << 22, 256), (1 << 21, 16, 512), (-1, 16, 1)):
        assert fls.fls_fp8_workspace_bytes(M, K, N) == 0
        with pytest.raises(fls.FlsError) as e:
            fls.ensure_fp8_workspace(M, K, N)
        assert e.value.code == fls.EINVAL


def test_refusals_need_no_device(fls):
    L = fls.lib()
    for args in ((None, 1, 16, 16, 16), (16, 1, 16, None, 16), (16, 1, 16, 16, None), (16, 0, 16, 16, 16), (16, 1, 17, 16, 16), (16, 1, 8, 16, 16),
                 (16, (1 << 21) + 1, 16, 16, 16), (16, 1, (1 << 22) + 16, 16, 16)):
        assert L.fls_quantize(*args, None) == fls.EINVAL
    for args in ((8, 1, 16, 16, 16), (16, 1, 16, 8, 16), (16, 1, 16, 16, 24)):
        assert L.fls_quantize(*args, None) == fls.EALIGN
    good = [16, 16, 16, 16, 1, 16, 1]
    for i in range(4):
        assert L.fls_fp8_gemm(*[None if j == i else a for j, a in enumerate(good)], None) == fls.EINVAL
        assert L.fls_fp8_gemm(*[24 if j == i else a for j, a in enumerate(good)], None) == fls.EALIGN
    assert L.fls_fp8_gemm(16, 16, 16, 16, 1, 20, 1, None) == fls.EINVAL
    assert L.fls_fp8_gemm(16, 16, 16, 16, 1, 16, 8193, None) == fls.EINVAL


def test_slices_stay_inside_the_room_for_their_sums(fls):
    """Also where K is longer than what one workgroup of the stream kernel takes (256 steps of 128)."""
    import ctypes

    L, out = fls.lib(), (ctypes.c_uint32 * 4)()
    for M in (1, 100, 7168, 50257, 1 << 21):
        for K in (16, 1040, 7168, 32768, 32784, 49152, 1 << 20, 1 << 22):
            for N in (1, 16, 17, 64, 65, 300, 8192):
                if fls.fls_fp8_workspace_bytes(M, K, N) == 0:
                    continue
                L.fls_internal_fp8_plan(M, K, N, 256, out)
                which, tile_m, tile_n, slices = out
                assert slices >= 1 and (slices == 1 or slices * M * N * 4 <= 64 << 20)
                assert which == 2 or (N <= 64 and tile_m in (16, 32, 64) and slices * 256 * 128 >= K)
                assert which != 0 or (N <= 16 and slices == 1)
                assert which != 2 or (tile_m, tile_n) in ((256, 256), (256, 128), (128, 128))
