"""What a decoder layer runs beside the compressed products: cases, plain forms and exact values of

  fp8        C = W . X with W in 8-bit floating point (e4m3, a power-of-two scale for each 128 consecutive k of a row) and X
             quantised the same way on the fly: matrices, and prompts, for which sparsity does not pay.
  quantize   dense W -> e4m3 and scales: run once per matrix when a model is loaded.
  attention  what lies between the QKV product and the output projection: causal, grouped heads, packed sequences of different
             lengths.  A prompt's Q, K and V are read where the QKV product put them ("fused"); a chunk of a prompt or a single
             token behind a stored prefix reads K and V from a cache in which every sequence has a slab of rows ("cache").

Weights are N(0, 0.02), activations N(0, 1) with some channels twenty times as large, as outlier channels of a model are;
queries are scaled so that scores spread by about two.  All of it is drawn on the GPU from the seed alone; the lengths of a case's
sequences are part of the case.
"""
import math
import random

import torch

own = False

BLOCK = 128          # consecutive k that share a scale
E4M3_MAX = 448.0
SLAB_SLACK = 37      # rows of a sequence's slab behind its last key
MOST_PRODUCTS = 12288 * 12288 * 4096
MOST_SCORES = 64 * 8192 * 8192              # heads x queries x keys, sequences padded to the longest
MOST_KEYS = 64 * 2048 * 56 * 128            # values of K, sequences padded to the longest


def _fp8(name, M, K, N):
    return {"name": name, "op": "fp8", "M": M, "K": K, "N": N}


def _attention(name, layout, sequences, heads, kv_heads, dim, q, past, lengths):
    """`q`, `past`: least and most queries of a sequence and keys before them; `lengths`: which lengths between them."""
    return {"name": name, "op": "attention", "layout": layout, "sequences": sequences, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "q_least": q[0], "q_most": q[1], "past_least": past[0], "past_most": past[1], "lengths": lengths}


def listed():
    return [
        # one sequence in a decode step of a small model: nothing but latency
        _attention("attention-1-token-h16-d64", "cache", 1, 16, 16, 64, (1, 1), (200, 200), 1),
        # a decode step of a 30B-shaped model, batch of 64, every head with keys of its own
        _attention("attention-decode-64-h56", "cache", 64, 56, 56, 128, (1, 1), (300, 2047), 2),
        # a decode step behind long documents, eight query heads to a key head
        _attention("attention-decode-long-64-8", "cache", 4, 64, 8, 128, (1, 1), (20000, 65000), 3),
        # prompts read in chunks, some behind a stored prefix; a head size that fills no matrix instruction
        _attention("attention-chunks-h32-d80", "cache", 3, 32, 32, 80, (100, 700), (0, 3000), 4),
        # a batch of prompts of a 30B-shaped model
        _attention("attention-prompts-h56", "fused", 8, 56, 56, 128, (17, 1500), (0, 0), 5),
        # one long prompt, grouped heads: the largest
        _attention("attention-prompt-8192-64-8", "fused", 1, 64, 8, 128, (8192, 8192), (0, 0), 6),
        # a small projection of a single token: nothing but latency
        _fp8("fp8-1024x1024-n1", 1024, 1024, 1),
        # a vocabulary's rows (an odd number) for an odd batch: the stream of a decode step
        _fp8("fp8-50257x7168-n13", 50257, 7168, 13),
        # a prompt of 1000 tokens (no multiple of any tile) through an FFN down-projection
        _fp8("fp8-7168x28672-n1000", 7168, 28672, 1000),
        # a long prompt: the largest
        _fp8("fp8-12288x12288-n4096", 12288, 12288, 4096),
        # model loading: an FFN up-projection, and a matrix with no round size
        {"name": "quantize-28672x7168", "op": "quantize", "M": 28672, "K": 7168},
        {"name": "quantize-999x1040", "op": "quantize", "M": 999, "K": 1040},
    ]


def _log_int(rng, lo, hi, step=1):
    """An integer in [lo, hi], a multiple of `step`, spread over the logarithm."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return min(hi // step * step, max(-(-lo // step) * step, int(v) // step * step))


def draw(rng):
    """One more case: the listed kinds over their ranges, odd sizes among them."""
    kind = rng.choices(["fp8", "quantize", "prompts", "chunks", "decode"], weights=[4, 1, 2, 2, 3])[0]
    if kind in ("fp8", "quantize"):
        M = _log_int(rng, 500, 51200, rng.choice([1, 16, 128]))
        K = _log_int(rng, 512, min(49152, 28672 * 7168 // M if kind == "quantize" else 12288 * 49152 // M), rng.choice([16, 32, 128]))
        if kind == "quantize":
            return {"op": "quantize", "M": M, "K": K}
        return {"op": "fp8", "M": M, "K": K, "N": _log_int(rng, 1, min(4096, MOST_PRODUCTS // (M * K)))}
    kv_heads, dim = _log_int(rng, 1, 32), rng.choice([64, 80, 96, 128])
    heads = kv_heads * rng.choice([1, 1, 2, 4, 8])
    layout, sequences = "cache", _log_int(rng, 1, 64 if kind == "decode" else 16)
    if kind == "prompts":
        layout, past = "fused", (0, 0)
        most = _log_int(rng, 1, max(1, min(4096, int(math.sqrt(MOST_SCORES // 8 // (sequences * heads))))))
        q = (max(1, most // rng.choice([1, 2, 8, 50])), most)
    elif kind == "chunks":
        most = _log_int(rng, 2, 1024)
        q, far = (max(1, most // rng.choice([1, 3, 20])), most), _log_int(rng, 1, 8192)
        far = min(far, MOST_SCORES // 8 // (sequences * heads * most), MOST_KEYS // (sequences * kv_heads * dim) - most)
        past = (rng.choice([0, far // 2, far]), far)
    else:
        q, far = (1, 1), max(1, min(_log_int(rng, 16, 60000), MOST_KEYS // (sequences * kv_heads * dim) - 1))
        past = (rng.choice([1, max(1, far // 4), far]), far)
    c = _attention("", layout, sequences, heads, kv_heads, dim, q, past, rng.randrange(1 << 30))
    del c["name"]
    return c


def _lengths(case):
    """Queries and keys of each sequence."""
    rng = random.Random(case["lengths"])
    nq = [rng.randint(case["q_least"], case["q_most"]) for _ in range(case["sequences"])]
    return nq, [n + rng.randint(case["past_least"], case["past_most"]) for n in nq]


def _starts(counts, slack=0):
    at = [0]
    for n in counts:
        at.append(at[-1] + n + slack)
    return at


def _scale_bytes(blocks):
    return -(-blocks // 4) * 4


def _quantize(x):
    """e4m3 values of x [rows, K] and the scales, bytes of an exponent: the smallest power of two that brings a block of 128 to at
    most 448.  A row's scales are filled up to a multiple of four with scales of one."""
    rows, K = x.shape
    blocks = -(-K // BLOCK)
    b = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - K)).view(rows, blocks, BLOCK)
    most = b.abs().amax(-1)
    half, e = torch.frexp(most)  # most = half * 2^e, half in [1/2, 1); 448 = 7/8 * 2^9
    e = torch.where(most > 0, e - 9 + (half > 0.875).int(), 0)
    down = ((127 - e) << 23).to(torch.int32).view(torch.float32)  # 2^-e
    q = (b * down[..., None]).to(torch.float8_e4m3fn).view(rows, blocks * BLOCK)[:, :K]
    s = torch.full((rows, _scale_bytes(blocks)), 127, dtype=torch.uint8, device=x.device)
    s[:, :blocks] = (e + 127).to(torch.uint8)
    return q.contiguous(), s.view(torch.float8_e8m0fnu)


def _values(q, s):
    """What quantised rows stand for, in fp32 (exactly)."""
    rows, K = q.shape
    scale = (s.view(torch.uint8).int() << 23).view(torch.float32)
    return q.float() * scale.repeat_interleave(BLOCK, dim=1)[:, :K]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    if case["op"] == "quantize":
        return {"case": case, "W": (randn(case["M"], case["K"]) * 0.02).half()}
    if case["op"] == "fp8":
        M, K, N = case["M"], case["K"], case["N"]
        channels = torch.where(torch.rand(K, generator=gen, device="cuda") < 0.002, 20.0, 1.0)
        X = (randn(N, K) * channels).half()
        Wq, Ws = torch.empty(M, K, dtype=torch.float8_e4m3fn, device="cuda"), []
        for r in range(0, M, 4096):  # a piece at a time: the matrix in fp32 would be eight times its size
            q, s = _quantize((randn(min(4096, M - r), K) * 0.02).half())
            Wq[r:r + 4096] = q
            Ws.append(s.view(torch.uint8))
        return {"case": case, "Wq": Wq, "Ws": torch.cat(Ws).view(torch.float8_e8m0fnu), "X": X,
                "C": torch.empty(N, M, dtype=torch.float16, device="cuda")}
    nq, nk = _lengths(case)
    H, G, D = case["heads"], case["kv_heads"], case["dim"]
    q_start = _starts(nq)
    if case["layout"] == "fused":  # C of the QKV product: a row per token, Q's heads, K's, V's
        qkv = randn(q_start[-1], H + 2 * G, D)
        qkv[:, :H] *= 2.0
        qkv = qkv.half()
        Q, K, V = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
        k_start = q_start[:-1]
    else:
        k_start = _starts(nk, SLAB_SLACK)
        Q, K, V = (randn(q_start[-1], H, D) * 2.0).half(), randn(k_start[-1], G, D).half(), randn(k_start[-1], G, D).half()
        k_start = k_start[:-1]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"case": case, "Q": Q, "K": K, "V": V, "q_start": ints(q_start), "k_start": ints(k_start), "k_len": ints(nk), "max_q": max(nq), "max_k": max(nk),
            "scale": 1.0 / math.sqrt(D), "O": torch.empty(q_start[-1], H, D, dtype=torch.float16, device="cuda"),
            "lse": torch.empty(H, q_start[-1], dtype=torch.float32, device="cuda")}


def _plain_attention(s):
    """All sequences padded to the longest, scores as a whole."""
    Q, K, V, q_start, mq, mk = s["Q"], s["K"], s["V"], s["q_start"].long(), s["max_q"], s["max_k"]
    (rows, H, D), G = Q.shape, K.shape[1]
    nq, nk = q_start[1:] - q_start[:-1], s["k_len"].long()
    B, i, j = len(nq), torch.arange(mq, device="cuda"), torch.arange(mk, device="cuda")
    of_q = (q_start[:-1, None] + i).clamp(max=rows - 1)
    of_k = (s["k_start"].long()[:, None] + j).clamp(max=len(K) - 1)
    q = Q[of_q].float().view(B, mq, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(B * G, H // G * mq, D)
    k = K[of_k].permute(0, 2, 3, 1).float().contiguous().view(B * G, D, mk)
    v = torch.where((j < nk[:, None])[:, :, None, None], V[of_k].float(), 0.0).permute(0, 2, 1, 3).contiguous().view(B * G, mk, D)
    p = torch.bmm(q, k).view(B, G, H // G, mq, mk).mul_(s["scale"])
    seen = j <= (i + (nk - nq)[:, None])[:, :, None]  # [B, mq, mk]
    p.masked_fill_(~seen[:, None, None], -math.inf)
    top = p.amax(-1, keepdim=True).clamp(min=-3e38)  # a row that sees no key has a sum of zero
    p.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(B * G, H // G * mq, mk), v).view(B, G, H // G, mq, D) / torch.where(total > 0, total, 1.0)
    lse = (top + total.log())[..., 0].reshape(B, H, mq)
    b = torch.repeat_interleave(torch.arange(B, device="cuda"), nq, output_size=rows)
    at = torch.arange(rows, device="cuda") - q_start[b]
    return {"O": o.view(B, H, mq, D)[b, :, at].half(), "lse": lse[b, :, at].T.contiguous()}


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2309_10285_amd as fls

        if op == "quantize":
            return fls.fls_quantize(state["W"])
        if op == "fp8":
            M, K, N = state["case"]["M"], state["case"]["K"], state["case"]["N"]
            fls.ensure_fp8_workspace(M, K, N)
            return fls.fls_fp8_gemm(state["Wq"], state["Ws"], state["X"], state["C"], M, K, N)
        fls.ensure_attention_workspace(state["Q"], state["K"], state["q_start"], state["max_q"], state["max_k"])
        fls.fls_attention(state["Q"], state["K"], state["V"], state["O"], state["q_start"], state["k_start"], state["k_len"],
                          state["max_q"], state["max_k"], state["scale"], state["lse"])
        return {"O": state["O"], "lse": state["lse"]}
    if op == "quantize":
        return _quantize(state["W"])
    if op == "fp8":
        return torch.mm(_values(*_quantize(state["X"])), _values(state["Wq"], state["Ws"]).T).half()
    return _plain_attention(state)


def work(case):
    """Every input read once, every output written once; every visible pair of query and key once in each of the two products."""
    if case["op"] == "attention":
        nq, nk = _lengths(case)
        H, G, D = case["heads"], case["kv_heads"], case["dim"]
        pairs = sum(q * k - q * (q - 1) // 2 for q, k in zip(nq, nk))
        return {"bytes": 4.0 * sum(nq) * H * D + 4.0 * sum(nk) * G * D + 4.0 * sum(nq) * H, "flops": 4.0 * D * H * pairs}
    M, K = case["M"], case["K"]
    scales = M * _scale_bytes(-(-K // BLOCK))
    if case["op"] == "quantize":
        return {"bytes": 3.0 * M * K + scales, "flops": 0.0}
    N = case["N"]
    return {"bytes": 1.0 * M * K + scales + 2.0 * N * (M + K), "flops": 2.0 * M * K * N}


def _exact_quantize(x):
    """(e4m3 values, scales) in 64 bits: the scale by its definition, the rounding by the spacing of e4m3's values."""
    rows, K = x.shape
    blocks = -(-K // BLOCK)
    b = torch.zeros(rows, blocks * BLOCK, dtype=torch.float64, device=x.device)
    b[:, :K] = x.double()
    b = b.view(rows, blocks, BLOCK)
    most = b.abs().max(dim=-1).values
    e = torch.ceil(torch.log2(torch.where(most > 0, most, E4M3_MAX) / E4M3_MAX)) - 1.0  # log2 may be an ulp off: try from below
    e = torch.where(most * torch.exp2(-e) > E4M3_MAX, e + 1.0, e)
    e = torch.where(most * torch.exp2(-e) > E4M3_MAX, e + 1.0, e)
    e = torch.where(most > 0, e, 0.0)
    v = b * torch.exp2(-e)[..., None]
    binade = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(binade - 3.0)
    q = torch.round(v / step) * step  # to even where it is half way
    scales = torch.ones(rows, _scale_bytes(blocks), dtype=torch.float64, device=x.device)
    scales[:, :blocks] = torch.exp2(e)
    return q.view(rows, blocks * BLOCK)[:, :K], scales


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        pieces = [_exact_quantize(s["W"][r:r + 4096]) for r in range(0, case["M"], 4096)]
        return tuple(torch.cat([p[k] for p in pieces]) for k in (0, 1))
    if case["op"] == "fp8":
        wide = lambda t: t.repeat_interleave(BLOCK, dim=1)[:, :case["K"]]  # noqa: E731
        q, scales = _exact_quantize(s["X"])
        X, C = q * wide(scales), torch.empty(case["N"], case["M"], dtype=torch.float64, device="cuda")
        for r in range(0, case["M"], 4096):
            power = s["Ws"][r:r + 4096].view(torch.uint8).double() - 127.0
            C[:, r:r + 4096] = X @ (s["Wq"][r:r + 4096].double() * wide(torch.exp2(power))).T
        return C
    nq, nk = _lengths(case)
    H, D, rep = case["heads"], case["dim"], case["heads"] // case["kv_heads"]
    O, lse = torch.zeros(sum(nq), H, D, dtype=torch.float64, device="cuda"), torch.zeros(H, sum(nq), dtype=torch.float64, device="cuda")
    at, starts = 0, s["k_start"].tolist()
    for n, k, k0 in zip(nq, nk, starts):
        far = torch.arange(n, device="cuda")[:, None] + (k - n) < torch.arange(k, device="cuda")
        for g in range(case["kv_heads"]):
            key, value = s["K"][k0:k0 + k, g].double(), s["V"][k0:k0 + k, g].double()
            for h in range(g * rep, (g + 1) * rep):
                score = s["Q"][at:at + n, h].double() @ key.T * s["scale"]
                score[far] = -math.inf
                lse[h, at:at + n] = torch.logsumexp(score, dim=1)
                O[at:at + n, h] = torch.exp(score - lse[h, at:at + n, None]) @ value
        at += n
    return {"O": O, "lse": lse}
