"""fls_attention against its definition in 64 bits.

Bounds, for a query with S = the largest scale |q| . |k| of its keys, n keys, and A = sum of weights times |v|:
  a score is a sum of head_dim products in fp32: off by at most (head_dim + 8) 2^-24 S, a few roundings of its own among them;
  a weight by as much again for the exponential's argument, and by 2^-21 for what the hardware's 2^x leaves;
  weights are rounded to fp16 for the product with V: half a step, 2^-11 of a weight; they are powers 2^(s - m + 7) of an m that is at most the largest
  score, so those under fp16's normal range, 2^-14, are off by at most 2^-25 / 2^7 of a weight at m, 2^-32 of the largest;
  sums over the keys in fp32: (n + 64) 2^-24;  O is rounded once: 2^-11 of it, 2^-25 below fp16's normal range.
"""
import math

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


def reference(Q, K, V, q_start, k_start, k_len, scale):
    """O, lse and how far each may be off, of the rows of sequences; the others are NaN in `off`."""
    import torch

    rows, H, D = Q.shape
    rep = H // K.shape[1]
    O, off = torch.zeros(rows, H, D, dtype=torch.float64, device="cuda"), torch.full((rows, H, D), math.nan, dtype=torch.float64, device="cuda")
    lse, lse_off = torch.full((H, rows), -math.inf, dtype=torch.float64, device="cuda"), torch.full((H, rows), math.nan, dtype=torch.float64, device="cuda")
    for b in range(len(k_len)):
        q0, q1, k0, nk = q_start[b], q_start[b + 1], k_start[b], k_len[b]
        nq = q1 - q0
        if nq == 0:
            continue
        hidden = torch.arange(nk, device="cuda") > torch.arange(nq, device="cuda")[:, None] + nk - nq
        for h in range(H):
            q, k, v = Q[q0:q1, h].double(), K[k0:k0 + nk, h // rep].double(), V[k0:k0 + nk, h // rep].double()
            s = (q @ k.T * scale).masked_fill(hidden, -math.inf)
            size = (q.abs() @ k.T.abs() * scale).masked_fill(hidden, 0.0).amax(1) if nk else torch.zeros(nq, dtype=torch.float64, device="cuda")
            top = s.amax(1, keepdim=True).clamp(min=-1e300) if nk else torch.zeros(nq, 1, dtype=torch.float64, device="cuda")
            p = torch.exp(s - top)
            total = p.sum(1, keepdim=True)
            w = p / torch.where(total > 0, total, 1.0)
            seen = ~hidden
            v0 = torch.where(torch.isfinite(v), v, 0.0)
            O[q0:q1, h] = w @ v0
            if not torch.isfinite(v).all():  # inf and NaN of the keys that are seen
                for code, add in ((v == math.inf, math.inf), (v == -math.inf, -math.inf), (torch.isnan(v), math.nan)):
                    O[q0:q1, h] += torch.where(seen.double() @ code.double() > 0, add, 0.0)
            lse[h, q0:q1] = (top + total.log())[:, 0]
            score = (D + 8) * 2.0 ** -24 * size
            A = w @ v0.abs()
            off[q0:q1, h] = 2.0 ** -11 * O[q0:q1, h].abs().nan_to_num(0, 0, 0) + (2.0 ** -11 + 2 * (2 * score + 2.0 ** -21 + (nk + 64) * 2.0 ** -24))[:, None] * A + 2.0 ** -25 + 2.0 ** -32 * v0.abs().sum(0) if nk else 0.0
            lse_off[h, q0:q1] = 2 * score + 2.0 ** -21 + (nk + 64) * 2.0 ** -24 + 2.0 ** -22 * lse[h, q0:q1].abs().nan_to_num(0, 0, 0)
    return O, off, lse, lse_off


def check(O, lse, ref, fill=5.0):
    import torch

    want, off, want_lse, lse_off = ref
    of_none = torch.isnan(off)
    assert (O[of_none] == fill).all(), "rows of no sequence were written"
    got, special = O.double(), ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got) & ~of_none, torch.isnan(want) & ~of_none)
    assert torch.equal(got[special & ~torch.isnan(want)], want[special & ~torch.isnan(want)])
    plain = ~of_none & ~special
    bad = (got - want).abs()[plain] > off[plain]
    assert not bad.any(), (int(bad.sum()), float(((got - want).abs()[plain] / off[plain]).max()))
    if lse is not None:
        none = torch.isnan(lse_off)
        assert (lse[none] == fill).all()
        empty = torch.isinf(want_lse) & ~none
        assert (lse[empty] == -math.inf).all()
        rest = ~none & ~empty
        assert ((lse.double() - want_lse).abs()[rest] <= lse_off[rest]).all()


def ints(v):
    import torch

    return torch.tensor(v, dtype=torch.int32, device="cuda")


def starts(counts, first=0, slack=0):
    at = [first]
    for n in counts:
        at.append(at[-1] + n + slack)
    return at


def attend(fls, Q, K, V, q_start, k_start, k_len, scale, O=None, with_lse=True, max_q=None, max_k=None):
    import torch

    rows, H, D = Q.shape
    O = torch.full((rows, H, D), 5.0, dtype=torch.float16, device="cuda") if O is None else O
    lse = torch.full((H, rows), 5.0, dtype=torch.float32, device="cuda") if with_lse else None
    mq = max([b - a for a, b in zip(q_start, q_start[1:])] + [0]) if max_q is None else max_q
    mk = max(list(k_len) + [0]) if max_k is None else max_k
    fls.ensure_attention_workspace(Q, K, ints(q_start), mq, mk)
    fls.fls_attention(Q, K, V, O, ints(q_start), ints(k_start), ints(k_len), mq, mk, scale, lse)
    torch.cuda.synchronize()
    return O, lse


def case(H, G, D, nq, nk, seed=0, q_first=0, slack=0, spread=2.0):
    import torch

    gen = torch.Generator(device="cuda").manual_seed(1000 + seed)
    q_start, k_start = starts(nq, q_first), starts(nk, 3, slack)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    Q = (randn(q_start[-1] + q_first, H, D) * spread).half()
    K, V = randn(k_start[-1] + 2, G, D).half(), randn(k_start[-1] + 2, G, D).half()
    return Q, K, V, q_start, k_start[:-1], list(nk)


# heads, key heads, head_dim, queries and keys of each sequence
CASES = [
    (1, 1, 64, [1], [1]), (2, 1, 64, [1, 1, 1], [1, 2, 33]), (4, 4, 8, [1], [40]), (16, 16, 64, [1], [201]), (8, 2, 128, [1, 1, 1, 1], [31, 32, 65, 700]),
    (6, 2, 80, [1, 0, 1], [129, 50, 257]), (64, 8, 128, [1], [5000]), (3, 3, 96, [1, 1], [20000, 130]), (40, 1, 64, [1, 1], [500, 64]), (8, 1, 72, [4, 2, 1], [300, 2, 17]),
    (5, 5, 128, [3, 1], [3, 900]), (4, 1, 64, [16, 9], [16, 2000]), (12, 4, 40, [7, 21, 20], [1000, 21, 19]),
    (2, 2, 64, [128], [128]), (2, 1, 128, [127, 1, 129, 64], [127, 1, 129, 64]), (1, 1, 128, [256], [256]), (3, 3, 80, [65, 100], [65, 100]), (2, 2, 96, [33, 200], [333, 900]),
    (4, 2, 128, [100], [6000]), (2, 1, 64, [150, 140], [9000, 140]), (1, 1, 16, [130], [131]), (7, 7, 128, [257, 70, 300], [257, 1070, 301]), (2, 2, 128, [1000], [1000]),
    # fewer keys than queries: the first queries see none; no keys; no queries
    (2, 1, 64, [5, 3], [2, 0]), (2, 2, 128, [200, 150, 90], [100, 0, 1]), (1, 1, 64, [129], [64]), (2, 1, 128, [0, 0], [10, 0]), (2, 2, 64, [0, 300, 0, 1], [7, 300, 0, 5]),
]


@pytest.mark.parametrize("H,G,D,nq,nk", CASES, ids=[f"{c[0]}x{c[1]}x{c[2]}-q{max(c[3])}-k{max(c[4])}" for c in CASES])
def test_against_the_definition(fls, H, G, D, nq, nk):
    Q, K, V, q_start, k_start, k_len = case(H, G, D, nq, nk, seed=len(nq) + D, q_first=2, slack=5)
    scale = D ** -0.5
    O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, scale)
    check(O, lse, reference(Q, K, V, q_start, k_start, k_len, scale))
    again, lse2 = attend(fls, Q, K, V, q_start, k_start, k_len, scale)
    import torch

    assert torch.equal(again, O) and torch.equal(lse, lse2)


@pytest.mark.parametrize("nq", [[1], [2, 1], [150]])
@pytest.mark.parametrize("n", [1, 3])
def test_one_key_gives_its_values(fls, nq, n):
    """The weight of the only key that is seen is exactly 1."""
    import torch

    Q, K, V, q_start, k_start, _ = case(4, 2, 64, nq, [1] * len(nq), seed=n)
    O, _ = attend(fls, Q, K, V, q_start, k_start, [1] * len(nq), 0.3)
    for b in range(len(nq)):
        assert torch.equal(O[q_start[b + 1] - 1], V[k_start[b]].repeat_interleave(2, 0))
        assert (O[q_start[b]:q_start[b + 1] - 1] == 0).all()


LAYOUTS = ["fused", "heads first", "cache of heads", "wide rows", "one key row"]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("nq,past", [([1, 1], [70, 300]), ([140, 30], [0, 0]), ([3, 2], [40, 9])])
def test_layouts(fls, layout, nq, past):
    import torch

    H, G, D = 6, 2, 80
    gen = torch.Generator(device="cuda").manual_seed(len(layout) + nq[0])
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda").half()  # noqa: E731
    nk = [a + b for a, b in zip(nq, past)]
    q_start, rows, keys = starts(nq), sum(nq), sum(nk)
    k_start, O = starts(nk)[:-1], None
    if layout == "fused":
        qkv = randn(keys, H + 2 * G, D)
        Q, K, V = qkv[:rows, :H], qkv[:, H:H + G], qkv[:, H + G:]
    elif layout == "heads first":
        Q, K, V = randn(H, rows, D).transpose(0, 1), randn(G, keys, D).transpose(0, 1), randn(G, keys, D).transpose(0, 1)
        O = torch.full((H, rows, D), 5.0, dtype=torch.float16, device="cuda").transpose(0, 1)
    elif layout == "cache of heads":  # [sequence][head][capacity][D] read as rows
        Q, K, V = randn(rows, H, D), randn(keys, G, D + 16)[..., :D], randn(keys, G, D + 8)[..., 8:]
    elif layout == "wide rows":
        Q, K, V = randn(rows, H + 3, D)[:, 2:2 + H], randn(keys, 3 * G, D)[:, ::3], randn(keys, 5, G, D)[:, 4]
        O = torch.full((rows, 2 * H, D), 5.0, dtype=torch.float16, device="cuda")[:, H:]
    else:  # every key the same: a row stride of 0
        Q, K, V = randn(rows, H, D), randn(1, G, D).expand(keys, G, D), randn(1, G, D).expand(keys, G, D)
    O, lse = attend(fls, Q, K, V, q_start, k_start, nk, 0.1, O=O)
    check(O, lse, reference(Q, K, V, q_start, k_start, nk, 0.1))
    attend(fls, Q, K, V, q_start, k_start, nk, 0.1, with_lse=False)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nq,nk", [([1, 1], [100, 9000]), ([4, 3], [70, 6]), ([150, 64], [150, 70]), ([100], [7000])])
def test_what_is_not_seen_does_not_matter(fls, D, nq, nk):
    """Infinities and NaN in rows beside the sequences and in keys that only later queries see."""
    import torch

    Q, K, V, q_start, k_start, k_len = case(4, 2, D, nq, nk, seed=3, q_first=1, slack=40)
    want = torch.full_like(K[:, 0, 0], True, dtype=torch.bool)
    for a, n in zip(k_start, k_len):
        want[a:a + n] = False
    K[want], V[want] = math.nan, math.inf
    K[want.nonzero()[0]] = math.inf
    Q[0] = math.nan
    O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.1)
    assert torch.isfinite(O[1:q_start[-1]]).all() and torch.isfinite(lse[:, 1:q_start[-1]]).all()
    check(O[1:], lse[:, 1:].contiguous(), reference(Q[1:], K, V, [a - 1 for a in q_start], k_start, k_len, 0.1))
    # values that some queries see: inf, -inf, NaN and both infinities in different columns
    last = k_start[0] + k_len[0] - 1
    for back, (at, x) in enumerate(((0, math.inf), (1, -math.inf), (2, math.nan), (3, math.inf), (3, -math.inf))):
        if back < k_len[0]:
            V[last - back, back % 2, at] = x
    O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.1)
    check(O[1:], lse[:, 1:].contiguous(), reference(Q[1:], K, V, [a - 1 for a in q_start], k_start, k_len, 0.1))


def test_large_and_equal_scores(fls):
    """One score far above the others, all equal, a growing sequence (the largest changes with every key), fp16's largest values."""
    import torch

    for nq, nk in (([1], [1000]), ([200], [200]), ([8], [3000])):
        Q, K, V, q_start, k_start, k_len = case(2, 1, 64, nq, nk, seed=8)
        for what in ("equal", "growing", "falling", "far", "largest"):
            if what == "equal":
                K[:] = 1.0
            elif what in ("growing", "falling"):
                Q[:], K[:] = 1.0, 0.0
                ramp = torch.arange(K.shape[0], device="cuda").half() / 8
                K[:, 0, 0] = ramp if what == "growing" else ramp.flip(0)
            elif what == "far":
                K[:] = -30.0
                K[k_start[0] + 1] = 30.0
            else:
                Q[:], K[:] = 65504.0, 65504.0
                K[k_start[0]] = -65504.0
            scale = 2.0 ** -20 if what == "largest" else 0.125
            O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, scale)
            check(O, lse, reference(Q, K, V, q_start, k_start, k_len, scale))


def test_not_a_number_in_a_query_or_a_key(fls):
    import torch

    for nq, nk in (([1, 2], [50, 40]), ([140, 130], [140, 500]), ([1], [6000])):
        Q, K, V, q_start, k_start, k_len = case(2, 2, 64, nq, nk, seed=1)
        Q[q_start[1] - 1, 0, 5] = math.nan
        O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.1)
        bad = torch.zeros_like(O, dtype=torch.bool)
        bad[q_start[1] - 1, 0] = True
        assert torch.equal(torch.isnan(O), bad) and torch.equal(torch.isnan(lse).T, bad[..., 0])
        Q[q_start[1] - 1, 0, 5] = 0.0
        K[:, 1] = math.nan
        O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.1)
        assert torch.isnan(O[:, 1]).all() and torch.isfinite(O[:, 0]).all() and torch.isnan(lse[1]).all()


def test_offsets_past_32_bits(fls):
    """Keys and values more than 4 GB behind the start of a cache."""
    import torch

    H, G, D, rows = 4, 2, 64, 2300
    cache = torch.empty(rows, 1 << 20, dtype=torch.float16, device="cuda")
    K, V = cache[:, 4096:4096 + G * D].view(rows, G, D), cache[:, (1 << 20) - G * D:].view(rows, G, D)
    gen = torch.Generator(device="cuda").manual_seed(4)
    for nq, nk in (([1, 1], [130, 90]), ([130], [140])):
        Q = torch.randn(sum(nq), H, D, generator=gen, device="cuda").half()
        k_start = [2150, 2160][:len(nk)]
        for a, n in zip(k_start, nk):
            K[a:a + n] = torch.randn(n, G, D, generator=gen, device="cuda").half()
            V[a:a + n] = torch.randn(n, G, D, generator=gen, device="cuda").half()
        O, lse = attend(fls, Q, K, V, starts(nq), k_start, nk, 0.2)
        check(O, lse, reference(Q, K, V, starts(nq), k_start, nk, 0.2))


def test_lengths_that_lie_outside_the_tensors(fls):
    """Nothing outside is read or written: such a sequence has no queries, or only the keys that there are."""
    import torch

    for nq, nk in (([2, 2, 2], [50, 60, 70]), ([140, 150, 130], [140, 160, 170])):
        Q, K, V, q_start, k_start, k_len = case(2, 1, 64, nq, nk, seed=6)
        base, _ = attend(fls, Q, K, V, q_start, k_start, k_len, 0.1)
        mq, mk = max(nq), max(nk)
        for change in (dict(k_len=[50, -3, 70]), dict(k_start=[3, -1, k_start[2]]), dict(k_start=[3, 1 << 30, k_start[2]]), dict(q=[0, nq[0], 1 << 30, 1 << 30]),
                       dict(q=[0, nq[0], -5, -5]), dict(q=[0, nq[0], 0, 0])):
            O, _ = attend(fls, Q, K, V, change.get("q", q_start), change.get("k_start", k_start), change.get("k_len", k_len), 0.1, max_q=mq, max_k=mk)
            assert torch.isfinite(O).all()
            if "q" in change or nk[0] == 50:
                assert torch.equal(O[:nq[0]], base[:nq[0]]) or "q" in change
        long = list(k_len)
        long[2] += 1000  # past the end: the keys that there are, in front of it
        O, lse = attend(fls, Q, K, V, q_start, k_start, long, 0.1, max_k=3000)
        there = K.shape[0] - k_start[2]
        check(O, lse, reference(Q, K, V, q_start, k_start, [k_len[0], k_len[1], there], 0.1))


@pytest.mark.parametrize("nq,nk", [([1, 1, 1], [300, 20, 4000]), ([130, 5, 260], [130, 900, 400])])
def test_in_a_graph_with_other_lengths(fls, nq, nk):
    import torch

    H, G, D = 8, 4, 128
    Q, K, V, q_start, k_start, k_len = case(H, G, D, nq, nk, seed=11)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        qs, ks, kl = ints(q_start), ints(k_start), ints(k_len)
        mq, mk = max(nq), max(nk)
        fls.ensure_attention_workspace(Q, K, qs, mq, mk)
        O, P = torch.zeros_like(Q), torch.zeros_like(Q)
        lse, lse2 = torch.zeros(H, Q.shape[0], device="cuda"), torch.zeros(H, Q.shape[0], device="cuda")
        fls.fls_attention(Q, K, V, O, qs, ks, kl, mq, mk, 0.1, lse)
        call = fls.prepare_attention(Q, K, V, P, qs, ks, kl, mq, mk, 0.1, lse2)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
        for i in range(4):
            kl.copy_(ints([max(1, n - 17 * i) for n in k_len]))
            Q.mul_(0.9)
            graph.replay()
            fls.fls_attention(Q, K, V, O, qs, ks, kl, mq, mk, 0.1, lse)
            side.synchronize()
            assert torch.equal(O, P) and torch.equal(lse, lse2) and O.abs().max() > 0


def test_a_layer_on_prompts_and_then_token_by_token(fls):
    """QKV product, attention, output projection: first the prompts, K and V going to the slabs of a cache, then single tokens.  Every step against the
    same step in 64 bits on what the step before it gave, and the single tokens against the whole sequence at once."""
    import torch

    hidden, H, G, D = 512, 8, 2, 64
    gen = torch.Generator(device="cuda").manual_seed(21)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    Wqkv, Wo = (randn((H + 2 * G) * D, hidden) * hidden ** -0.5).half(), (randn(hidden, H * D) * (H * D) ** -0.5).half()
    qkv8, o8 = fls.fls_quantize(Wqkv), fls.fls_quantize(Wo)
    lens, steps = [37, 150, 1], 3
    total, capacity = sum(lens), max(lens) + steps
    x = randn(total + steps * len(lens), hidden).half()  # prompts, then a token of each sequence per step
    cache_k, cache_v = torch.zeros(len(lens) * capacity, G, D, dtype=torch.float16, device="cuda"), torch.zeros(len(lens) * capacity, G, D, dtype=torch.float16, device="cuda")
    slabs = [b * capacity for b in range(len(lens))]

    def layer(x, q_start, k_len, max_q):
        rows = x.shape[0]
        C = torch.empty(rows, (H + 2 * G) * D, dtype=torch.float16, device="cuda")
        fls.ensure_fp8_workspace(C.shape[1], hidden, rows)
        fls.fls_fp8_gemm(*qkv8, x, C, C.shape[1], hidden, rows)
        qkv = C.view(rows, H + 2 * G, D)
        at = torch.cat([torch.arange(slabs[b] + k_len[b] - (q_start[b + 1] - q_start[b]), slabs[b] + k_len[b]) for b in range(len(lens))]).cuda()
        cache_k[at], cache_v[at] = qkv[:, H:H + G], qkv[:, H + G:]
        O = torch.empty(rows, H, D, dtype=torch.float16, device="cuda")
        fls.ensure_attention_workspace(qkv[:, :H], cache_k, ints(q_start), max_q, max(k_len))
        fls.fls_attention(qkv[:, :H], cache_k, cache_v, O, ints(q_start), ints(slabs), ints(k_len), max_q, max(k_len), D ** -0.5)
        check(O, None, reference(qkv[:, :H], cache_k, cache_v, q_start, slabs, k_len, D ** -0.5))
        if max_q > 1:  # a prompt's keys are the QKV product's own rows
            P = torch.empty_like(O)
            fls.fls_attention(qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:], P, ints(q_start), ints(q_start[:-1]), ints(k_len), max_q, max(k_len), D ** -0.5)
            assert torch.equal(O, P)
        out = torch.empty(rows, hidden, dtype=torch.float16, device="cuda")
        fls.fls_fp8_gemm(*o8, O.view(rows, H * D), out, hidden, H * D, rows)
        return C, O, out

    C, O, out = layer(x[:total], starts(lens), list(lens), max(lens))
    for (W, src, got) in ((Wqkv, x[:total], C), (Wo, O.view(total, -1), out)):
        ref = src.double() @ W.double().T
        assert (got.double() - ref).norm() <= 2 ** 0.5 * 2.0 ** -4 / 3 ** 0.5 * ref.norm()  # two operands rounded to e4m3
    for i in range(steps):
        now = x[total + i * len(lens):total + (i + 1) * len(lens)]
        layer(now, starts([1] * len(lens)), [n + i + 1 for n in lens], 1)
    # all tokens of the longest sequence at once, from the cache: the same as what came step by step
    b = 1
    n = lens[b] + steps
    whole = torch.cat([x[37:37 + lens[b]]] + [x[total + i * len(lens) + b][None] for i in range(steps)])
    C = torch.empty(n, (H + 2 * G) * D, dtype=torch.float16, device="cuda")
    fls.ensure_fp8_workspace(C.shape[1], hidden, n)
    fls.fls_fp8_gemm(*qkv8, whole, C, C.shape[1], hidden, n)
    K = C.view(n, H + 2 * G, D)[:, H:H + G]
    assert (K.double() - cache_k[slabs[b]:slabs[b] + n].double()).norm() <= 2.0 ** -10 * K.double().norm()


@pytest.mark.parametrize("H,G,D,nq,nk", [
    (2, 1, 64, [n % 3 for n in range(200)], [5 * n % 71 + 2 for n in range(200)]),                                   # single tokens and pairs
    (1, 1, 128, [70] + [n % 2 for n in range(150)] + [40], [75] + [7 * n % 400 + 1 for n in range(150)] + [3000]),   # 128 queries to a workgroup, chunks
    (3, 3, 80, [130 if n % 40 == 7 else n % 2 for n in range(131)] + [300], [3 * n % 200 for n in range(131)] + [310]),
], ids=["few", "chunks", "tiles"])
def test_more_sequences_than_a_wave_has_lanes(fls, H, G, D, nq, nk):
    import torch

    Q, K, V, q_start, k_start, k_len = case(H, G, D, nq, nk, seed=len(nq), q_first=3, slack=1)
    O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.2)
    check(O, lse, reference(Q, K, V, q_start, k_start, k_len, 0.2))
    # the same where max_q and max_k promise more than there is: other kernels, other chunks
    for mq, mk in ((max(nq) * 100, max(nk)), (max(nq), 20000), (1 << 20, 1 << 28)):
        P, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.2, max_q=mq, max_k=mk)
        check(P, lse, reference(Q, K, V, q_start, k_start, k_len, 0.2))


@pytest.mark.parametrize("H,G,D,nq,nk", [
    (64, 1, 64, [16, 3, 9], [700, 3, 2000]), (32, 4, 128, [16, 1, 13], [600, 900, 13]), (24, 2, 80, [15], [9000]), (33, 1, 96, [15, 2], [1500, 1]), (13, 1, 128, [12, 14], [7000, 14]),
    (64, 1, 64, [17, 3], [700, 3]), (32, 4, 128, [16, 9], [500, 512]), (32, 4, 128, [16, 9], [500, 513]), (8, 2, 40, [16], [2000]), (8, 2, 40, [17], [2000]),
])
def test_rows_of_many_heads_that_share_keys(fls, H, G, D, nq, nk):
    """Several workgroups of 32 rows to a key head, and the other kernel where it takes over."""
    Q, K, V, q_start, k_start, k_len = case(H, G, D, nq, nk, seed=H + D, q_first=1, slack=2)
    O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, D ** -0.5)
    check(O, lse, reference(Q, K, V, q_start, k_start, k_len, D ** -0.5))


@pytest.mark.parametrize("D", [128, 104])
@pytest.mark.parametrize("G", [64, 16])
def test_many_workgroups(fls, D, G):
    """More than four workgroups to a CU, with tiles of their own: ragged lengths, fewer keys than queries, none, and values that are not finite in keys that are not seen or seen by some."""
    import random

    import torch

    r = random.Random(D + G)
    nq = [r.choice((0, 1, 33, 128, 129, 200, r.randint(2, 260))) for _ in range(22)] + [100, 150]
    nk = [max(0, n + r.choice((0, 0, 1, 31, 64, 700, -n // 2, -n))) for n in nq[:-2]] + [100, 2048]
    Q, K, V, q_start, k_start, k_len = case(64, G, D, nq, nk, seed=D, q_first=1, slack=3)
    O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.1)
    check(O, lse, reference(Q, K, V, q_start, k_start, k_len, 0.1))
    outside = torch.ones(K.shape[0], dtype=torch.bool, device="cuda")
    for at, n in zip(k_start, k_len):
        outside[at:at + n] = False
    K[outside], V[outside] = math.nan, math.inf
    for b in (22, 23):  # keys that the last few queries see
        last = k_start[b] + k_len[b] - 1
        V[last, 3, 7], V[last - 1, 5, 8], V[last - 40, 7, 9], K[last - 2, 0] = math.inf, math.nan, -math.inf, -1000.0
    O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.1)
    check(O, lse, reference(Q, K, V, q_start, k_start, k_len, 0.1))


def test_sequences_that_share_keys_and_are_cut(fls):
    """Two sequences on the same keys (a shared prefix); and max_q, max_k below what a sequence has: its first so many of each."""
    Q, K, V, q_start, _, _ = case(4, 2, 64, [3, 2, 140], [400], seed=13)
    for mq, mk in ((140, 300), (140, 100), (64, 300), (2, 33)):
        k_start, k_len = [3, 3, 20], [300, 200, 250]
        O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, 0.2, max_q=mq, max_k=mk)
        for b in range(3):
            n, cut = min(q_start[b + 1] - q_start[b], mq), min(k_len[b], mk)
            rows = slice(q_start[b], q_start[b] + n)
            check(O[rows], lse[:, rows].contiguous(), reference(Q[rows], K, V, [0, n], [k_start[b]], [cut], 0.2))
            assert (O[q_start[b] + n:q_start[b + 1]] == 5).all()


def test_nothing_to_attend(fls):
    import torch

    e = lambda *s: torch.empty(s, dtype=torch.float16, device="cuda")  # noqa: E731
    O = torch.full((3, 2, 64), 5.0, dtype=torch.float16, device="cuda")
    fls.ensure_attention_workspace(O, e(0, 1, 64), ints([0, 3]), 3, 0)
    assert fls.fls_attention(e(0, 2, 64), e(0, 1, 64), e(0, 1, 64), e(0, 2, 64), ints([0, 0]), ints([0]), ints([0]), 0, 0, 1.0).shape == (0, 2, 64)
    assert (fls.fls_attention(e(3, 2, 64), e(7, 1, 64), e(7, 1, 64), O, ints([0]), ints([]), ints([]), 3, 7, 1.0) == 5).all()  # no sequence
    for max_k in (0, 9):  # no key
        lse = torch.zeros(2, 3, device="cuda")
        O.fill_(5.0)
        fls.fls_attention(e(3, 2, 64), e(0, 1, 64), e(0, 1, 64), O, ints([0, 3]), ints([0]), ints([0]), 3, max_k, 1.0, lse)
        assert (O == 0).all() and (lse == -math.inf).all()


def test_very_many_sequences(fls):
    """More workgroups than a grid has in one direction: single tokens with one key each, whose values are the result."""
    import torch

    n, H, D = 300000, 32, 8
    gen = torch.Generator(device="cuda").manual_seed(2)
    Q = torch.randn(n, H, D, generator=gen, device="cuda").half()
    V = torch.randn(1000, H, D, generator=gen, device="cuda").half()
    k_start = torch.randint(0, 1000, (n,), generator=gen, device="cuda", dtype=torch.int32)
    q_start, k_len = torch.arange(n + 1, device="cuda", dtype=torch.int32), torch.ones(n, device="cuda", dtype=torch.int32)
    O = torch.zeros_like(Q)
    fls.ensure_attention_workspace(Q, V, q_start, 1, 1)
    fls.fls_attention(Q, V, V, O, q_start, k_start, k_len, 1, 1, 1.0)
    assert torch.equal(O, V[k_start.long()])


@pytest.mark.parametrize("seed", range(24))
def test_drawn(fls, seed):
    """Shapes and lengths drawn over what the call takes."""
    import random

    r = random.Random(seed)
    G = r.choice((1, 1, 2, 3, 5))
    H, D = G * r.choice((1, 1, 2, 3, 4, 7, 8, 13)), 8 * r.randint(1, 16)
    longest = r.choice((1, 1, 2, 5, 16, 64, 200, 700))
    nq = [r.randint(0, longest) if r.random() < 0.8 else longest for _ in range(r.choice((1, 1, 2, 3, 7, 12)))]
    nk = [max(0, n + r.choice((0, 0, 1, 63, 64, 300, 5000, -1, -n // 2))) for n in nq]
    Q, K, V, q_start, k_start, k_len = case(H, G, D, nq, nk, seed=seed, q_first=r.choice((0, 1)), slack=r.choice((0, 3)), spread=r.choice((0.1, 1.0, 4.0)))
    scale = r.choice((1.0, D ** -0.5, 0.01))
    O, lse = attend(fls, Q, K, V, q_start, k_start, k_len, scale)
    check(O, lse, reference(Q, K, V, q_start, k_start, k_len, scale))


def test_a_graph_keeps_its_workspace(fls):
    """A call that was recorded before a larger workspace was made writes its partial sums where it did."""
    import torch

    Q, K, V, q_start, k_start, k_len = case(2, 1, 64, [1, 1], [9000, 8000], seed=17)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        qs, ks, kl = ints(q_start), ints(k_start), ints(k_len)
        fls._ws_tensor = None  # as in a new process
        fls.ensure_attention_workspace(Q, K, qs, 1, 9000)
        O, P = torch.zeros_like(Q), torch.zeros_like(Q)
        fls.fls_attention(Q, K, V, O, qs, ks, kl, 1, 9000, 0.1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            fls.fls_attention(Q, K, V, P, qs, ks, kl, 1, 9000, 0.1)
            with pytest.raises(fls.FlsError) as e:  # a larger one cannot be made here
                fls.ensure_fp8_workspace(128, 1 << 17, 64)
            assert e.value.code == fls.EWORKSPACE
        size = fls._ws_tensor.numel()
        fls.ensure_fp8_workspace(128, 1 << 17, 64)
        assert fls._ws_tensor.numel() > size
        others = [torch.full((size,), 0x7f, dtype=torch.uint8, device="cuda") for _ in range(3)]
        for i in range(3):
            P.zero_()
            graph.replay()
            side.synchronize()
            assert torch.equal(O, P) and all((t == 0x7f).all() for t in others)


def test_refusals_in_the_binding(fls):
    import torch

    Q, K, V, q_start, k_start, k_len = case(2, 1, 64, [2], [5])
    args = lambda **c: [c.get("Q", Q), c.get("K", K), c.get("V", V), c.get("O", torch.empty_like(Q)), c.get("qs", ints(q_start)), ints(k_start), ints(k_len), 2, 5, c.get("scale", 1.0)]  # noqa: E731
    for bad in (dict(Q=Q.float()), dict(K=K.cpu()), dict(V=V[:-1]), dict(O=torch.empty_like(Q)[:1]), dict(qs=ints(q_start).long()), dict(qs=ints(q_start + q_start)),
                dict(Q=Q.transpose(1, 2))):
        with pytest.raises(AssertionError):
            fls.fls_attention(*args(**bad))
    for bad in (dict(scale=0.0), dict(O=torch.empty(1, 2, 64, dtype=torch.float16, device="cuda").expand(*Q.shape)), dict(Q=torch.empty(Q.shape[0], 2, 68, dtype=torch.float16, device="cuda")[..., :64])):
        with pytest.raises(fls.FlsError) as e:
            fls.fls_attention(*args(**bad))
        assert e.value.code == fls.EINVAL


def test_tensors_of_another_device_are_refused(fls, monkeypatch):
    """As on a machine with two of them, of which the other one is the current one."""
    import torch

    Q, K, V, q_start, k_start, k_len = case(2, 1, 64, [2], [5])
    call = lambda: fls.fls_attention(Q, K, V, torch.empty_like(Q), ints(q_start), ints(k_start), ints(k_len), 2, 5, 1.0)  # noqa: E731
    W = torch.zeros(8, 128, dtype=torch.float16, device="cuda")
    Wq, Ws = fls.fls_quantize(W)
    fls.ensure_fp8_workspace(8, 128, 8)
    product = lambda: fls.fls_fp8_gemm(Wq, Ws, W, torch.empty(8, 8, dtype=torch.float16, device="cuda"), 8, 128, 8)  # noqa: E731
    monkeypatch.setattr(fls, "_several_devices", True)
    for f in (call, product, lambda: fls.fls_quantize(W)):
        f()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for f in (call, product, lambda: fls.fls_quantize(W)):
        with pytest.raises(AssertionError):
            f()


@pytest.mark.parametrize("D", [72, 80, 96])
@pytest.mark.parametrize("nq,nk", [([1, 1], [100, 9000]), ([4, 3], [70, 6]), ([150, 64], [150, 70]), ([100], [7000]), ([3] * 150, [5 + n for n in range(150)])])
def test_what_is_not_seen_does_not_matter_in_heads_of_up_to_96(fls, D, nq, nk):
    """Kernels of their own: 96 values in a row of 128."""
    test_what_is_not_seen_does_not_matter(fls, D, nq, nk)


LOW, HIGH = -(1 << 31), (1 << 31) - 1


@pytest.mark.parametrize("H,G,D,nq,nk", [(2, 1, 64, [2, 2, 2], [50, 60, 70]), (4, 2, 96, [1, 2, 1], [9000, 3000, 40]), (2, 2, 128, [1] * 150, [40] * 150), (2, 1, 64, [140, 150, 130], [140, 160, 170]),
                                         (2, 1, 80, [100, 90, 160], [6000, 90, 500]), (96, 96, 128, [300, 260, 500], [300, 260, 600]), (1, 1, 128, [70] + [2] * 70 + [60], [75] + [9] * 70 + [60])],
                         ids=["few", "few chunks", "few of two waves", "many", "many chunks", "many small tiles", "more than lanes"])
def test_lengths_outside_the_tensors_against_the_definition(fls, H, G, D, nq, nk):
    """A sequence whose queries are not all inside has none and its rows stay as they were; one whose keys begin outside has none, one whose keys reach past the end has those up to there."""
    import torch

    Q, K, V, q_start, k_start, k_len = case(H, G, D, nq, nk, seed=D, slack=3)
    rows, k_rows, n, mq, mk = Q.shape[0], K.shape[0], len(nq), max(nq), max(nk) + 100
    at = lambda values, i, x: values[:i % len(values)] + [x] + values[i % len(values) + 1:]  # noqa: E731
    changes = [dict(k_len=at(k_len, i, x)) for i, x in ((1, -3), (0, LOW), (n - 1, 0), (n - 1, HIGH), (n - 1, nk[-1] + 90))]
    changes += [dict(k_start=at(k_start, i, x)) for i, x in ((0, -1), (1, k_rows), (n - 1, HIGH), (1, LOW), (0, k_rows - 1), (n - 1, k_rows - 5))]
    changes += [dict(k_start=at(k_start, 1, HIGH), k_len=at(k_len, 1, HIGH)), dict(k_start=[-1] * n)]
    changes += [dict(q_start=q) for q in (at(q_start, 0, -5), at(q_start, 0, LOW), [-7, -2] + q_start[2:], at(q_start, n, rows + 1), at(q_start, n, HIGH), q_start[:2] + [1 << 30] * (n - 1),
                                          q_start[:2] + [rows] * (n - 1) if q_start[1] + mq >= rows else q_start[:2] + [q_start[1]] * (n - 1), [LOW] * n + [HIGH], [rows] * (n + 1), [-9] * (n + 1))]
    for change in changes:
        q, k, length = change.get("q_start", q_start), change.get("k_start", k_start), change.get("k_len", k_len)
        assert all(a <= b for a, b in zip(q, q[1:]))
        O, lse = attend(fls, Q, K, V, q, k, length, 0.1, max_q=mq, max_k=mk)
        untouched = torch.ones(rows, dtype=torch.bool, device="cuda")
        for b in range(n):
            if not (0 <= q[b] < q[b + 1] <= rows):
                continue
            count = min(q[b + 1] - q[b], mq)
            keys = min(length[b], k_rows - k[b], mk) if 0 <= k[b] < k_rows and length[b] > 0 else 0
            there = slice(q[b], q[b] + count)
            untouched[there] = False
            check(O[there], lse[:, there].contiguous(), reference(Q[there], K, V, [0, count], [k[b] if keys else 0], [keys], 0.1))
        assert (O[untouched] == 5).all() and (lse[:, untouched] == 5).all()
