"""How fls_attention cuts a call: which kernel, chunks of keys, and the GPU's CUs in both.  Needs no GPU."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def plan():
    import paper_2309_10285_amd as f
    from paper_2309_10285_amd import _build

    if not os.path.exists(f.LIB_PATH):
        _build.build()
    L = f.lib()

    def plan(q_rows, sequences, heads, kv_heads, dim, max_q, max_k, cus=256):
        out = (ctypes.c_uint32 * 6)()
        L.fls_internal_attention_plan(q_rows, sequences, heads, kv_heads, dim, max_q, max_k, cus, out)
        return dict(zip(("few", "chunk", "chunks", "units", "waves", "tile"), out))

    return plan


def test_few_queries_share_the_keys_out_to_one_workgroup_a_cu(plan):
    for cus in (32, 64, 128, 256):
        for sequences, kv_heads in ((1, 8), (1, 1), (4, 8), (16, 2)):
            p = plan(sequences, sequences, 2 * kv_heads, kv_heads, 128, 1, 100000, cus)
            busy = sequences * kv_heads
            wanted = max(1, min(cus // busy, 391))
            chunk = -(-(-(-100000 // wanted)) // 128) * 128
            assert (p["few"], p["chunk"], p["chunks"]) == (1, chunk, -(-100000 // chunk))
            assert p["units"] == busy * p["chunks"] and p["waves"] == (4 if p["units"] <= cus else 2)


def test_many_queries_fill_no_more_than_four_workgroups_a_cu(plan):
    for cus in (32, 64, 128, 256):
        for q_rows in (40, 129, 512, 2000, 9000):
            for heads in (1, 6, 32, 64):
                for max_k in (100, 1000, 9000, 100000):
                    p = plan(q_rows, 1, heads, heads, 128, q_rows, max_k, cus)
                    assert p["few"] == 0 and p["chunk"] % 128 == 0 and (p["chunks"] - 1) * p["chunk"] < max_k <= p["chunks"] * p["chunk"]
                    assert p["chunks"] == 1 or -(-q_rows // 128) * heads * p["chunks"] <= 4 * cus
                    assert p["units"] == (q_rows // 128 + 1) * heads * p["chunks"]
                    assert p["tile"] == (32 if p["units"] > 4 * cus and max_k <= 2048 else 64)


def test_chunks_of_many_queries_as_measured(plan):
    """Behind 512, 2512 and 8512 keys, 512 queries: 64 heads in one, two and two chunks, 32 heads behind 8512 in four; half of the CUs with half of the heads cut as
    all of them do."""
    chunks = lambda heads, max_k, cus=256: plan(512, 1, heads, heads, 128, 512, max_k, cus)["chunks"]  # noqa: E731
    assert [chunks(64, 512 + k) for k in (512, 2512, 8512)] == [1, 2, 2] and chunks(32, 9024) == 4
    for heads, max_k in ((64, 1024), (64, 9024), (32, 9024), (16, 30000)):
        for less in (2, 4, 8):
            assert chunks(heads // less, max_k, 256 // less) == chunks(heads, max_k)


@pytest.mark.parametrize("rep", [1, 2, 3, 4, 5, 8, 13, 64])
def test_what_counts_as_few_queries(plan, rep):
    """As the header says: max_q x r <= 32; or r >= 4, max_k > 512 and max_q x r <= 32 (r / 2)."""
    few = lambda max_q, max_k, rows=1 << 20: plan(rows, 3, 2 * rep, 2, 64, max_q, max_k)["few"]  # noqa: E731
    for max_q in range(1, 70):
        assert few(max_q, 512) == (max_q * rep <= 32)
        assert few(max_q, 513) == (max_q * rep <= 32 or (rep >= 4 and max_q * rep <= 32 * (rep // 2)))
    most = max(q for q in range(1, 70) if few(q, 513))
    assert most == {1: 32, 2: 16, 3: 10, 4: 16, 5: 12, 8: 16, 13: 14, 64: 16}[rep]
