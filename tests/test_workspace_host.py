"""What the binding's ensure_... functions make and keep, with memory that exists in name only.  Needs no GPU."""
import os

import pytest


@pytest.fixture()
def fls(monkeypatch):
    import torch

    import paper_2309_10285_amd as f
    from paper_2309_10285_amd import _build

    if not os.path.exists(f.LIB_PATH):
        _build.build()
    empty, made = torch.empty, []

    def on_no_device(size, *args, device=None, **kwargs):
        if device != "cuda":
            return empty(size, *args, device=device, **kwargs)
        made.append(size)
        return empty(size, *args, device="meta", **kwargs)

    monkeypatch.setattr(f, "_ws_tensor", None)
    monkeypatch.setattr(f, "_ws_made", [])
    monkeypatch.setattr(f, "fls_set_workspace", lambda ws: monkeypatch.setattr(f, "_ws_tensor", ws))
    monkeypatch.setattr(torch, "empty", on_no_device)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: f.capturing, raising=True)
    monkeypatch.setattr(f, "capturing", False, raising=False)
    f.made = made
    yield f
    del f.made


def ensures(fls):
    """ensure_... and ..._workspace_bytes of growing shapes, for each of the three."""
    import torch

    Q, K = torch.zeros(1, 64, 128, device="meta"), torch.zeros(1 << 20, 8, 128, device="meta")
    q = lambda n: torch.zeros(n + 1, device="meta")  # noqa: E731
    return [(lambda n: fls.ensure_workspace(12288, 49152, n), lambda n: fls.fls_workspace_bytes(12288, 49152, n), range(40, 4000, 37)),
            (lambda n: fls.ensure_fp8_workspace(12288, 49152, n), lambda n: fls.fls_fp8_workspace_bytes(12288, 49152, n), range(40, 4000, 37)),
            (lambda n: fls.ensure_attention_workspace(Q.expand(n, 64, 128), K, q(n), 1, 1 << 20),
             lambda n: fls.fls_attention_workspace_bytes(Q.expand(n, 64, 128), K, n, 1, 1 << 20), range(1, 9))]


@pytest.mark.parametrize("which", range(3), ids=["products", "fp8", "attention"])
def test_what_growing_shapes_leave_behind_is_bounded(fls, which):
    """Workspaces stay alive for the graphs that were recorded with them: sizes are powers of two, under twice what is needed, and a larger one is
    twice as large at least, so all of them are under twice the largest."""
    ensure, need, steps = ensures(fls)[which]
    for n in steps:
        ensure(n)
        assert fls._ws_tensor.numel() >= need(n)
        kept = sum(t.numel() for t in fls._ws_made)
        assert kept < 4 * max(need(m) for m in steps if m <= n)
    assert fls.made == [t.numel() for t in fls._ws_made]
    assert fls.made == sorted(set(fls.made))
    before = list(fls.made)
    for n in steps:  # what is there is large enough for all of them
        ensure(n)
    assert fls.made == before


@pytest.mark.parametrize("which", range(3), ids=["products", "fp8", "attention"])
def test_none_is_made_while_a_graph_is_recorded(fls, which):
    """It would be memory of the graph's own, cleared only when the graph is replayed."""
    ensure, need, steps = ensures(fls)[which]
    fls.capturing = True
    with pytest.raises(fls.FlsError) as e:
        ensure(steps[0])
    assert e.value.code == fls.EWORKSPACE and fls.made == [] and fls._ws_tensor is None
    fls.capturing = False
    ensure(steps[-1])
    made = list(fls.made)
    fls.capturing = True
    ensure(steps[0])  # large enough already
    assert fls.made == made


def test_in_turn_with_a_callers_own_workspace(fls):
    import torch

    for _ in range(5):
        fls.fls_set_workspace(torch.zeros(1 << 20, dtype=torch.uint8, device="meta"))
        fls.ensure_workspace(1024, 1024, 8)
        small = fls._ws_tensor
        fls.ensure_fp8_workspace(1024, 1024, 8)
        assert fls._ws_tensor.numel() > small.numel()
    assert len(fls._ws_made) == 2


@pytest.mark.parametrize("operator", ["fp8", "attention"])
@pytest.mark.parametrize("prepared", [False, True])
def test_a_workspace_on_another_device_is_refused(monkeypatch, operator, prepared):
    """There is one workspace; a call on a second GPU must not write its sums into the first one's memory.  Host tensors, as far as the binding can tell on the current GPU."""
    import torch

    import paper_2309_10285_amd as f

    launched = []

    class Library:
        def fls_fp8_gemm(self, *args):
            launched.append(args)
            return 0

        fls_attention = fls_fp8_gemm
        fls_strerror = staticmethod(lambda code: b"")

    class Workspace:
        def __init__(self, device):
            self.device = device

        def get_device(self):
            return self.device

    here = torch.zeros(1).get_device()
    library = Library()
    monkeypatch.setattr(f, "lib", lambda: library)
    monkeypatch.setattr(f, "_stream", lambda: 0)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: here)
    half = lambda *s: torch.zeros(s, dtype=torch.float16)  # noqa: E731
    ints = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    if operator == "fp8":
        args = (torch.zeros(8, 128, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(8, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu), half(2, 128), half(2, 8), 8, 128, 2)
        call = (lambda: f.prepare_fp8_gemm(*args)()) if prepared else lambda: f.fls_fp8_gemm(*args)
    else:
        args = (half(2, 2, 64), half(5, 1, 64), half(5, 1, 64), half(2, 2, 64), ints(0, 2), ints(0), ints(5), 2, 5, 1.0)
        call = (lambda: f.prepare_attention(*args)()) if prepared else lambda: f.fls_attention(*args)
    for several, workspace, fine in ((False, Workspace(here), True), (True, Workspace(here), True), (True, None, True), (True, Workspace(here + 1), False)):
        monkeypatch.setattr(f, "_several_devices", several)
        monkeypatch.setattr(f, "_ws_tensor", workspace)
        del launched[:]
        if fine:
            call()
            assert len(launched) == 1
        else:
            with pytest.raises(f.FlsError) as e:
                call()
            assert e.value.code == f.EWORKSPACE and launched == []
