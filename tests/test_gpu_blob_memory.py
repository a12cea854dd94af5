"""The library's memory of blob addresses when a blob's memory is freed and handed out again."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fls():
    import torch

    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2309_10285_amd as f

    f.lib()
    return f


@pytest.mark.parametrize("N", [8, 48, 200])
def test_a_blob_of_the_other_version_in_memory_that_was_freed(fls, N):
    """Version 1 is compressed and freed; the same memory then holds a copy of the same matrix in version 2."""
    import torch

    M, K = 640, 3040
    gen = torch.Generator(device="cuda").manual_seed(N)
    W = torch.randn(M, K, generator=gen, device="cuda").half()
    W[torch.rand(M, K, generator=gen, device="cuda") < 0.7] = 0
    X, C = torch.randn(N, K, generator=gen, device="cuda").half(), torch.empty(N, M, dtype=torch.float16, device="cuda")
    ref = X.double() @ W.double().T
    close = lambda: ((C.double() - ref).abs().max() <= 2e-3 * ref.abs().max()).item()  # noqa: E731
    fls.ensure_workspace(M, K, N)
    second, _ = fls.fls_compress_v2(W)
    first, _ = fls.fls_compress(W)
    kept = first[:64].view(torch.int8)  # as long as any view is left the memory is the blob's
    fls.fls_spmm(first, X, C, M, K, N)
    assert close()
    address, size = first.data_ptr(), first.untyped_storage().nbytes()
    del first, kept
    held, place = [], None
    for _ in range(50):
        place = torch.empty(size, dtype=torch.uint8, device="cuda")
        if place.data_ptr() == address:
            break
        held.append(place)
    else:
        pytest.skip("the allocator did not hand the memory out again")
    place[:second.numel()].copy_(second)
    fls.fls_spmm(place, X, C, M, K, N)
    assert close()
    fls.fls_forget(place)


@pytest.mark.parametrize("N", [8, 48, 200])
@pytest.mark.parametrize("how", ["out", "copy", "prepared"])
def test_a_blob_that_the_caller_placed(fls, how, N):
    """The same for memory that the caller gave fls_compress, and for a copy of a blob that the library saw in a product first."""
    import torch

    M, K = 640, 3040
    gen = torch.Generator(device="cuda").manual_seed(N + len(how))
    W = torch.randn(M, K, generator=gen, device="cuda").half()
    W[torch.rand(M, K, generator=gen, device="cuda") < 0.7] = 0
    X, C = torch.randn(N, K, generator=gen, device="cuda").half(), torch.empty(N, M, dtype=torch.float16, device="cuda")
    ref = X.double() @ W.double().T
    close = lambda: ((C.double() - ref).abs().max() <= 2e-3 * ref.abs().max()).item()  # noqa: E731
    fls.ensure_workspace(M, K, N)
    blobs = [fls.fls_compress(W)[0], fls.fls_compress_v2(W)[0]]
    size, address, held = fls.fls_compress_bound(M, K), None, []
    for version in (0, 1, 0, 1):
        for _ in range(50):
            place = torch.empty(size, dtype=torch.uint8, device="cuda")
            if address in (None, place.data_ptr()):
                break
            held.append(place)
        else:
            pytest.skip("the allocator did not hand the memory out again")
        address = place.data_ptr()
        if how == "out" and version == 0:
            fls.fls_compress(W, out=place)
        else:
            place[:blobs[version].numel()].copy_(blobs[version])
        C.zero_()
        if how == "prepared":
            call = fls.prepare_spmm(place, X, C, M, K, N)
            call()
            del call
        else:
            fls.fls_spmm(place, X, C, M, K, N)
        assert close()
        del place
