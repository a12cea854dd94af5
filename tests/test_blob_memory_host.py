"""Which blobs the binding makes the library forget when their memory is freed, with a recorder in the library's place.  Needs no GPU."""
import os

import pytest


@pytest.fixture()
def fls(monkeypatch):
    import torch

    import paper_2309_10285_amd as f
    from paper_2309_10285_amd import _build

    if not os.path.exists(f.LIB_PATH):
        _build.build()
    real = f.lib()

    class Library:
        forgotten, remembered = [], []
        fls_compress_bound, fls_compress_bound_v2 = real.fls_compress_bound, real.fls_compress_bound_v2

        def fls_compress(self, W, M, K, out, *rest):
            self.remembered.append(out)
            return 0

        def fls_compress_v2(self, W, M, K, out, *rest):
            self.remembered.append(out)
            return 0

        def fls_spmm(self, blob, *rest):
            self.remembered.append(blob)
            return 0

        def fls_forget(self, at):
            self.forgotten.append(at)

    library = Library()
    monkeypatch.setattr(f, "lib", lambda: library)
    monkeypatch.setattr(f, "_stream", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)  # host memory, as far as the binding can tell
    return f


def operands(torch):
    return torch.zeros(128, 32, dtype=torch.float16), torch.zeros(4, 32, dtype=torch.float16), torch.zeros(4, 128, dtype=torch.float16)


@pytest.mark.parametrize("compress", ["fls_compress", "fls_compress_v2"])
def test_memory_of_the_callers(fls, compress):
    import torch

    W, _, _ = operands(torch)
    arena = torch.empty(1 << 20, dtype=torch.uint8)
    at = [arena.data_ptr(), arena.data_ptr() + 4096]
    for _ in range(3):  # again into the same memory: forgotten once
        for i in (0, 1):
            blob, _ = getattr(fls, compress)(W, out=arena[4096 * i:4096 * i + 4096])
    assert fls.lib().remembered == at * 3
    del arena
    assert fls.lib().forgotten == []  # a view is left
    del blob
    assert sorted(fls.lib().forgotten) == at


def test_memory_of_the_bindings(fls):
    import torch

    W, _, _ = operands(torch)
    blob, _ = fls.fls_compress(W)
    at = fls.lib().remembered
    assert len(at) == 1 and fls.lib().forgotten == []
    del blob
    assert fls.lib().forgotten == at


@pytest.mark.parametrize("prepared", [False, True])
def test_a_copy_that_was_multiplied(fls, prepared):
    """The library remembers a blob when it first sees it, whoever put it there."""
    import torch

    _, X, C = operands(torch)
    blob = torch.zeros(4096, dtype=torch.uint8)
    at = blob.data_ptr()
    if prepared:
        call = fls.prepare_spmm(blob, X, C, 128, 32, 4)
        call()
        del call
    else:
        for _ in range(3):
            fls.fls_spmm(blob, X, C, 128, 32, 4)
    assert fls.lib().forgotten == []
    del blob
    assert fls.lib().forgotten == [at]


def test_memory_that_is_handed_out_again(fls):
    """What lies at an address later is forgotten in its turn."""
    import torch

    _, X, C = operands(torch)
    seen = []
    for _ in range(4):
        blob = torch.zeros(1 << 16, dtype=torch.uint8)
        seen.append(blob.data_ptr())
        fls.fls_spmm(blob, X, C, 128, 32, 4)
        del blob
        assert fls.lib().forgotten == seen
