"""Host side of fls_attention: sizes and refusals, before anything is launched.  Needs no GPU."""
import os

import pytest

GOOD = dict(q_rows=100, k_rows=300, q_row=512, q_head=64, k_row=128, k_head=64, v_row=128, v_head=64, o_row=512, o_head=64, sequences=3, heads=8, kv_heads=2,
            head_dim=64, max_q=50, max_k=200, scale=0.125)


@pytest.fixture(scope="module")
def fls():
    import paper_2309_10285_amd as f
    from paper_2309_10285_amd import _build

    if not os.path.exists(f.LIB_PATH):
        _build.build()
    return f


def shape(fls, **changed):
    return fls._ATTENTION_LAYOUT.pack(*{**GOOD, **changed}.values())


def test_workspace(fls):
    size = lambda **c: fls.lib().fls_attention_workspace_bytes(shape(fls, **c))  # noqa: E731
    area = 4 << 20
    assert size() == area                                                  # 50 queries, 200 keys: one chunk
    assert size(k_rows=1 << 20, max_q=1, max_k=100000, sequences=1) > area  # one token behind many keys: chunks
    assert size(k_rows=1 << 20, max_k=100000) > area                       # 100 queries of 8 heads: chunks too
    assert size(q_rows=0) == area and size(sequences=0) == area and size(max_q=0) == area and size(max_k=0) == area and size(k_rows=0) == area
    # bounded: a thousand and some workgroups, 128 rows of at most 130 values each
    for rows in (1, 7, 100, 1000, 30000, 1000000):
        for heads, kv in ((1, 1), (64, 8), (96, 96)):
            for sequences, max_q in ((1, rows), (rows, 1), (3, 17)):
                c = dict(q_rows=rows, sequences=sequences, max_q=max_q, heads=heads, kv_heads=kv, head_dim=128, k_rows=1 << 30, max_k=1 << 28,
                         q_row=0, o_row=heads * 128, o_head=128)
                assert area <= size(**c) <= area + 2048 * 128 * 130 * 4 + 16


BAD = [dict(q_rows=-1), dict(k_rows=-1), dict(q_rows=(1 << 31) - 1), dict(k_rows=(1 << 31) - 1), dict(heads=0), dict(kv_heads=0), dict(kv_heads=3), dict(heads=-8), dict(heads=65544),
       dict(head_dim=0), dict(head_dim=65), dict(head_dim=136), dict(head_dim=-8), dict(max_q=-1), dict(max_k=-1), dict(max_q=1 << 31), dict(max_k=1 << 31), dict(scale=0.0), dict(scale=-1.0),
       dict(scale=float("inf")), dict(scale=float("nan")), dict(sequences=-1), dict(sequences=(1 << 24) + 1), dict(q_row=513), dict(k_row=-8),
       dict(v_row=(1 << 22) + 8), dict(k_head=(1 << 40) + 8), dict(v_head=4), dict(o_head=32), dict(o_row=448), dict(o_row=0), dict(o_head=0),
       dict(scale=2.1e38), dict(sequences=1 << 24, heads=64, kv_heads=64, max_q=1, o_row=4096), dict(sequences=1 << 24, max_q=100),
       dict(q_rows=(1 << 31) - 2, heads=65536, kv_heads=65536, o_row=1 << 22, max_q=1 << 30)]


@pytest.mark.parametrize("bad", BAD, ids=[",".join(b) + str(i) for i, b in enumerate(BAD)])
def test_shapes_refused(fls, bad):
    L = fls.lib()
    assert L.fls_attention_workspace_bytes(shape(fls, **bad)) == 0
    assert L.fls_attention(16, 16, 16, 16, 16, 16, 16, 16, shape(fls, **bad), None) == fls.EINVAL


def test_pointers_refused(fls):
    L = fls.lib()
    assert L.fls_attention_workspace_bytes(None) == 0
    good = [16, 16, 16, 16, 16, 16, 16, 16, shape(fls), None]
    for i in (0, 1, 2, 3, 5, 6, 7, 8):
        assert L.fls_attention(*[None if j == i else a for j, a in enumerate(good)]) == fls.EINVAL
    for i in (0, 1, 2, 3):
        assert L.fls_attention(*[24 if j == i else a for j, a in enumerate(good)]) == fls.EALIGN
    for i in (4, 5, 6, 7):
        assert L.fls_attention(*[18 if j == i else a for j, a in enumerate(good)]) == fls.EALIGN
    # heads after one another, each a block of rows, is a layout as well; in places of one row or one head strides do not matter
    for ok in (dict(o_row=64, o_head=6400), dict(q_rows=1, o_row=0), dict(heads=1, kv_heads=1, o_head=0)):
        assert L.fls_attention_workspace_bytes(shape(fls, **ok)) > 0


def test_nothing_to_do(fls):
    """No query: nothing is launched and no pointer is looked at; no shape is let through for it."""
    L = fls.lib()
    for none in (dict(q_rows=0), dict(sequences=0), dict(max_q=0)):
        assert L.fls_attention(*[None] * 8, shape(fls, **none), None) == fls.OK
        assert L.fls_attention(*[None] * 8, shape(fls, head_dim=65, **none), None) == fls.EINVAL
    for i in (0, 3, 5, 6, 7):  # K and V may be null where there are no keys, the others not
        args = [16, None, None, 16, 16, 16, 16, 16, shape(fls, k_rows=0), None]
        assert L.fls_attention(*[None if j == i else a for j, a in enumerate(args)]) == fls.EINVAL


def test_the_binding_refuses_what_is_not_on_the_gpu(fls):
    import torch

    Q, n = torch.zeros(1, 1, 64, dtype=torch.float16), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(AssertionError):
        fls.fls_attention(Q, Q, Q, Q, torch.zeros(2, dtype=torch.int32), n, n, 1, 1, 1.0)
    with pytest.raises(AssertionError):
        fls.fls_quantize(Q[0])


def test_the_limits_that_the_header_names(fls):
    """The last that is taken, the first that is not."""
    size = lambda **c: fls.lib().fls_attention_workspace_bytes(shape(fls, **c))  # noqa: E731
    big = (1 << 31) - 1
    for last, step, rest in ((("k_rows", big - 1), 1, {}), (("q_rows", big - 1), 1, dict(max_q=1)), (("max_q", big - 1), 1, {}), (("max_k", (1 << 31) - 4098), 1, {}),
                             (("sequences", 1 << 24), 1, dict(heads=1, kv_heads=1, max_q=1)), (("heads", 65536), 2, dict(q_rows=1, max_q=1)), (("k_row", 1 << 22), 8, {}),
                             (("v_head", 1 << 40), 8, {}), (("head_dim", 128), 8, dict(o_head=128, o_row=1024)), (("scale", 2e38), 1e37, {})):
        name, value = last
        assert size(**{**rest, name: value}) > 0, name
        assert size(**{**rest, name: value + step}) == 0, name


def test_a_search_without_end_is_refused(fls):
    """With many queries a workgroup looks through the sequences for its own: workgroups times sequences are bounded, at some 20 seconds.  One query to a sequence needs no search."""
    size = lambda **c: fls.lib().fls_attention_workspace_bytes(shape(fls, **c))  # noqa: E731
    n = 1 << 20
    many = dict(q_rows=n, sequences=n, max_q=100, kv_heads=1, o_row=512)
    assert ((n // 128 + n) * 4) * n <= 1 << 43 < ((n // 128 + n) * 8) * n
    assert size(**many, heads=4) > 0
    assert size(**many, heads=8) == 0
    assert size(**{**many, "sequences": n // 2}, heads=8) > 0
    assert size(**{**many, "max_q": 1}, heads=8) > 0
