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
    # control area, 64 MiB of sums, X in e4m3, its scales
    assert fls.fls_fp8_workspace_bytes(1024, 1024, 8) == (4 << 20) + (64 << 20) + 8 * 1024 + 64
    assert fls.fls_fp8_workspace_bytes(1, 16, 3) == (4 << 20) + (64 << 20) + 48 + 16
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
