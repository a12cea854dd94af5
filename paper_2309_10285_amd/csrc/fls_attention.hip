// fls_attention: causal softmax attention with grouped heads over packed sequences, in one pass over the keys.
//
//   s_ij = scale q_i . k_j for j <= i + keys - queries,   o_i = sum_j exp(s_ij) v_j / sum_j exp(s_ij)
//
// A query keeps a score m (times log2 e: powers of two are what the hardware computes), the sum l of 2^(s - m) and the sum o of
// 2^(s - m) v.  When a score exceeds m by more than kSlack, m becomes the largest score so far and l and o are multiplied by 2^(old - new); to
// do that for every new largest score would cost as much as a fifth of the other vector work.  All three are fp32; 2^(s - m) is rounded to
// fp16 for the product with v (to nearest, 2^-11 of it), raised by 2^kLift so that what is small beside the largest is not subnormal:
// at most 2^(kLift + kSlack), half of what fp16 holds.
//
// Both products are computed transposed, with 32x32x16 MFMAs: S^T = K Q^T gives lane l the column of query l & 31 and of 32 keys the rows
// 8 a + 4 (l >> 5) + b (a, b = 0 ... 3), so that the largest and the sum of a query's scores are found inside a lane and
// its neighbour 32 further.  In O^T = V^T P^T the same registers are the operand as they are: a lane's eight k may be any eight keys of 16, if
// V^T has the same, and those are read from row-major V in LDS by transposing reads of four keys (ds_read_b64_tr_b16).
//
// Keys and values go to LDS without passing through registers.  16-byte piece c of row r lies at place c ^ turn(r), so that
// eight lanes that read the same piece of eight rows find them in eight places, and the four rows of a transposing read as well.
#include "fls_device.h"
#include "fls_launch.h"

namespace fls {

typedef float float16v __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));

constexpr int kLift = 7, kSlack = 8;
constexpr uint32_t kNowhere = 0x80000000u;  // an offset past every buffer descriptor here: a load from it gives 0
constexpr float kInf = __builtin_inff();

struct AttentionParams {
  const _Float16 *Q, *K, *V;
  _Float16* O;
  float* lse;
  const int32_t *q_start, *k_start, *k_len;
  int64_t q_rows, k_rows, q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  uint32_t sequences, heads, rep, dim, max_q, max_k;
  uint32_t chunk, chunks;     // keys to a workgroup where they are split, and into how many at most
  uint32_t slots, units, row_blocks;
  float scale_log2;           // scale * log2 e
  float* part_o;              // [chunk][part row][head][DP] sums not yet divided; part rows: max_q to a sequence where there are few, else those of Q
  float* part_ml;             // [chunk][part row][head][2]
  uint64_t part_rows;
  uint32_t few;
  Divisor by_rep, by_chunks, by_chunk, by_row_blocks, by_kv_heads, by_slots, by_heads, by_max_q;
};

// A sequence, cut to the tensors it lies in: whatever the arrays hold, nothing outside is read or written.
struct Sequence {
  int64_t q0, k0;
  uint32_t nq, nk;
};

__device__ __forceinline__ Sequence sequence(const AttentionParams& p, uint32_t b) {
  const int64_t a = p.q_start[b], e = p.q_start[b + 1], k = p.k_start[b], n = p.k_len[b];
  Sequence s = {a, k, 0u, 0u};
  if (a >= 0 && e > a && e <= p.q_rows) s.nq = (uint32_t)(e - a);
  if (k >= 0 && n > 0 && k < p.k_rows) s.nk = (uint32_t)(n < p.k_rows - k ? n : p.k_rows - k);
  s.nq = min(s.nq, p.max_q);
  s.nk = min(s.nk, p.max_k);
  return s;
}

// Chunks that so many keys are cut into.  One chunk goes to O at once.
__device__ __forceinline__ uint32_t chunks_of(uint32_t keys, const AttentionParams& p) { return keys <= p.chunk ? 1u : divide((keys - 1u) >> 7, p.by_chunk) + 1u; }

// Head sizes are filled up to DP = 64, 96 or 128 with zeros; a row in LDS has 64 or 128 values.
template <int DP>
constexpr int kPitch = DP == 64 ? 64 : 128;

// Where a row's pieces lie.  128 values: 16 rows give a piece 16 places (256 B, all banks), four neighbouring rows four pieces 16 places.
// 64 values: the same of eight and four pairs of rows.
template <int DP>
__device__ __forceinline__ uint32_t turn(uint32_t row) {
  return DP == 64 ? (row >> 1 & 1u) << 2 | (row >> 2 & 3u) : (row & 3u) << 2 | (row >> 2 & 3u);
}

// ROWS rows to LDS by THREADS lanes; rows from `left` on and values from dim on are 0.
template <int DP, int ROWS, int THREADS, bool STREAM = false>
__device__ __forceinline__ void stage(const _Float16* first, int64_t row_stride, uint32_t left, uint32_t dim, uint32_t lds, uint32_t thread) {
  constexpr uint32_t kPieces = kPitch<DP> / 8, kStep = THREADS / kPieces;  // rows to a load of all lanes
  static_assert(ROWS % kStep == 0 && (kStep % 16 == 0 || 16 % kStep == 0), "whole loads");
  const uint32_t bytes = left == 0u ? 0u : (uint32_t)((min(left, (uint32_t)ROWS) - 1u) * row_stride * 2 + dim * 2u);
  const u32x4 buf = descriptor(first, bytes);
  const uint32_t wave = __builtin_amdgcn_readfirstlane(thread >> 6);
#pragma unroll
  for (int i = 0; i < ROWS / (int)kStep; ++i) {
    const uint32_t row = i * kStep + thread / kPieces, piece = (thread % kPieces) ^ turn<DP>(row);
    const uint32_t off = row * (uint32_t)(row_stride * 2) + piece * 16u;
    load_lds<16, STREAM>(buf, lds + i * THREADS * 16 + wave * 1024u, row < left && piece * 8u < dim ? off : kNowhere);
  }
}

// What a wave knows of its 32 queries: lane l of query l & 31.
template <int DP>
struct Wave {
  half8 q[DP / 16];
  float16v o[DP / 32];
  float m, l;
  int limit;  // last key the query sees, from the first key of the sequence on; below 0: none

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) o[d] = float16v{};
    m = -kInf;
    l = 0.f;
  }

  // `here`: whether this lane's query is one
  __device__ __forceinline__ void load(const _Float16* row, bool here, uint32_t dim, uint32_t lane) {
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      const uint32_t d = i * 16u + (lane >> 5) * 8u;
      q[i] = half8{};
      if (here && d < dim) q[i] = *(const half8*)(row + d);
    }
  }
};

__device__ __forceinline__ float across(float x, bool add) {  // with the lane 32 further
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, x), false, false);
  const uint32_t lower = r[0], upper = r[1];  // of r[1] itself, __builtin_bit_cast takes r[0]
  const float a = __builtin_bit_cast(float, lower), b = __builtin_bit_cast(float, upper);
  return add ? a + b : fmaxf(a, b);
}

// Where a lane begins to read in a tile of K or V, from its start on.  All its other places differ from that in bits that pieces lie in (and in whole rows), so
// they are one exclusive or away: kept in registers, they would be more than there are.  That is right for the address in LDS as well if no bit of the tile's
// start is among them: tiles begin at multiples of kTileAlign.
constexpr uint32_t kTileAlign = 256;  // a row of 128 values
template <int DP>
__device__ __forceinline__ uint32_t key_place(uint32_t lane) {
  const uint32_t row = lane & 31u;
  return row * (kPitch<DP> * 2) + ((turn<DP>(row) ^ (lane >> 5)) << 4);
}
template <int DP>
__device__ __forceinline__ uint32_t value_place(uint32_t lane) {
  const uint32_t row = 4u * (lane >> 5) + ((lane & 15u) >> 2), piece = 2u * ((lane >> 4) & 1u) + ((lane & 3u) >> 1);
  return row * (kPitch<DP> * 2) + ((piece ^ turn<DP>(row)) << 4) + (lane & 1u) * 8u;
}
__device__ __forceinline__ uint32_t place_in(uint32_t tile, uint32_t place) {
  uint32_t at = tile + place;
  asm volatile("" : "+v"(at));  // not known before the loop
  return at;
}

typedef const __attribute__((address_space(3))) half8* lds_half8;

// S^T of 32 B keys; `at`: key_place in their rows of K.  Block by block in turn: a product that waits for the one before it waits longer than it takes.
template <int DP, int B>
__device__ __forceinline__ void scores(const Wave<DP>& w, uint32_t at, float16v (&s)[B]) {
#pragma unroll
  for (int b = 0; b < B; ++b) s[b] = float16v{};
#pragma unroll
  for (uint32_t i = 0; i < DP / 16; ++i)
#pragma unroll
    for (int b = 0; b < B; ++b)
      s[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*(lds_half8)(uintptr_t)((at ^ (i << 5)) + b * (32 * kPitch<DP> * 2)), w.q[i], s[b], 0, 0, 0);
}

// Eight keys of V^T for 32 d: keys key + 4 (l >> 5) + 0 ... 3 and the same 8 further, as S^T has them; `at`: value_place.
template <int DP>
__device__ __forceinline__ half8 values(uint32_t at, uint32_t key, uint32_t d) {
  typedef __attribute__((address_space(3))) short4v* lds_ptr;
  constexpr uint32_t kRow = kPitch<DP> * 2;
  const short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)((at ^ (d << 1)) + key * kRow));
  const short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(uintptr_t)((at ^ (d << 1) ^ 32u) + (key + 8u) * kRow));
  return __builtin_bit_cast(half8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Key of score i of a lane.
__device__ __forceinline__ uint32_t key_of(int i, uint32_t lane) { return 8u * (i / 4) + 4u * (lane >> 5) + i % 4; }

// Makes m fit 32 B keys with these scores.
template <int DP, int B>
__device__ __forceinline__ void settle(Wave<DP>& w, const float16v (&s)[B], float scale_log2) {
  float top = s[0][0];
#pragma unroll
  for (int b = 0; b < B; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
  top = across(top, false) * scale_log2;
  if (!__any(top > w.m + kSlack)) return;
  const float m = fmaxf(w.m, top), down = m == -kInf ? 0.f : __builtin_amdgcn_exp2f(w.m - m);
  w.m = m;
  w.l *= down;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) w.o[d][i] *= down;
}

// Their weights in their place, added to l.
template <int DP, int B>
__device__ __forceinline__ void soften(Wave<DP>& w, float16v (&s)[B], float scale_log2) {
  const float base = w.m == -kInf ? 0.f : w.m - kLift;  // a query that has seen no key: its weights are 0, not NaN
  float sum = 0.f;
#pragma unroll
  for (int b = 0; b < B; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], scale_log2, -base));
      sum += s[b][i];
    }
  w.l += sum;  // of this lane's keys; both lanes' in the end
}

__device__ __forceinline__ half8 weights(const float16v& s, int half) {
  half8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (_Float16)s[half * 8 + i];
  return r;
}

template <int DP, int B>
__device__ __forceinline__ void add_values(Wave<DP>& w, const half8 (&p)[2 * B], uint32_t at) {
#pragma unroll
  for (int k = 0; k < 2 * B; ++k)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) w.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(values<DP>(at, k * 16u, d * 32u), p[k], w.o[d], 0, 0, 0);
}

// Does V in LDS hold an infinity or NaN?
template <int DP, int ROWS>
__device__ __forceinline__ bool any_not_finite(uint32_t tile, uint32_t lane) {
  uint32_t most = 0;  // magnitudes of two values; those of fp16 are ordered as their bits are
#pragma unroll 2
  for (int i = 0; i < ROWS * kPitch<DP> / 512; ++i) {
    const u32x4 v = *(const __attribute__((address_space(3))) u32x4*)(uintptr_t)(tile + (i * 64u + lane) * 16u);
#pragma unroll
    for (int e = 0; e < 4; ++e) most = max_u16(most, v[e] & 0x7fff7fffu);
  }
  return __any((most & 0xffffu) >= 0x7c00u || most >= 0x7c000000u);
}

// add_values where some queries do not see some keys whose values are not finite: a weight of 0 times those is NaN.  Query by query,
// with the values that the query does not see taken as 0; 32 times the work, for tiles that any_not_finite finds.
template <int DP, int B>
__device__ __forceinline__ void add_seen_values(Wave<DP>& w, const half8 (&p)[2 * B], uint32_t at, int key0, uint32_t lane) {
#pragma unroll 1
  for (uint32_t query = 0; query < 32u; ++query) {
    const int limit = __builtin_amdgcn_readlane(w.limit, query) - key0;
    const bool mine = (lane & 31u) == query;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      float16v o = {};
#pragma unroll
      for (int k = 0; k < 2 * B; ++k) {
        half8 v = values<DP>(at, k * 16u, d * 32u);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if ((int)(k / 2 * 32u + key_of((k & 1) * 8 + i, lane)) > limit) v[i] = (_Float16)0.f;
        o = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p[k], o, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) w.o[d][i] = mine ? w.o[d][i] + o[i] : w.o[d][i];
    }
  }
}

// One tile of 32 B keys from key0 on (relative to the sequence).  MASK: some query may not see some of them; CHECK: nor their values, be they not finite.
template <int DP, int B, bool MASK, bool CHECK>
__device__ __forceinline__ void attend(Wave<DP>& w, uint32_t k_tile, uint32_t v_tile, int key0, float scale_log2, uint32_t lane) {
  const uint32_t k_at = place_in(k_tile, key_place<DP>(lane)), v_at = place_in(v_tile, value_place<DP>(lane));
  float16v s[B];
  scores<DP, B>(w, k_at, s);
  if (MASK) {
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (key0 + (int)(b * 32u + key_of(i, lane)) > w.limit) s[b][i] = -kInf;
  }
  settle<DP, B>(w, s, scale_log2);
  soften<DP, B>(w, s, scale_log2);
  half8 p[2 * B];
#pragma unroll
  for (int k = 0; k < 2 * B; ++k) p[k] = weights(s[k / 2], k & 1);
  if (CHECK && any_not_finite<DP, 32 * B>(v_tile, lane)) add_seen_values<DP, B>(w, p, v_at, key0, lane);
  else add_values<DP, B>(w, p, v_at);
}

// 32 d of a lane's query: four in a row at 8 a + 4 (l >> 5)
template <int DP>
__device__ __forceinline__ void store_rows(const Wave<DP>& w, _Float16* row, float factor, uint32_t dim, uint32_t lane) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const uint32_t at = d * 32u + a * 8u + (lane >> 5) * 4u;
      if (at < dim)
        *(half4*)(row + at) = half4{(_Float16)(w.o[d][4 * a] * factor), (_Float16)(w.o[d][4 * a + 1] * factor), (_Float16)(w.o[d][4 * a + 2] * factor),
                                    (_Float16)(w.o[d][4 * a + 3] * factor)};
    }
}

__device__ __forceinline__ float log_sum(float m, float l) { return l > 0.f ? (m - kLift + __builtin_amdgcn_logf(l)) * 0.69314718055994531f : l == 0.f ? -kInf : l; }

// --- many queries to a sequence ------------------------------------------------------------------------------------------------
// A workgroup has 128 queries of a head, 32 to a wave; tiles of 32 or 64 keys go through LDS in two stages.  Tiles that every query sees
// come first, in a loop without a mask.  A prompt of 8192, 64 heads of 128 on 8: 1127 - 1190 us, 0.92 - 0.98 PFLOP/s, bound by power (1.8 GHz; the same cycles at 2.4 GHz, 851 us, with all inputs zero).  Eight prompts of
// 17 - 1500, 56 heads of 128: 194 us, of which queries and results some 30: a workgroup's start and end have only the others on its CU to hide behind.  Two fit in 64 KB of LDS each and 256
// registers; three in 32 KB and 168 registers, with rows of 64 values (8 prompts of 1024, 56 heads of 64, 119 -> 112 us, 64 of 128 63 -> 55) or tiles of 32 keys.

constexpr uint32_t kTileQ = 128;

// x of all lanes up to this one.
__device__ __forceinline__ uint32_t sum_up_to_lane(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);  // the lane before, in rows of 16
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);  // the last lane of the row before, for every second row
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);  // lane 31, for the upper half
  return x;
}

template <int DP, int KEYS>
__global__ __launch_bounds__(256, KEYS * kPitch<DP> <= 4096 ? 3 : 2) void attention_kernel(AttentionParams p) {
  constexpr int B = KEYS / 32, kBytes = KEYS * kPitch<DP> * 2;
  __shared__ __align__(kTileAlign) uint8_t stages[2][2 * kBytes];  // a tile of K, one of V
  static_assert(__alignof__(stages) % kTileAlign == 0 && kBytes / B % kTileAlign == 0, "tiles, and blocks of 32 keys in them");
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint32_t unit;
  if (!xcd_unit(p.units, unit)) return;
  // head by head and chunk by chunk, so that what runs at one time on an XCD reads the same keys
  const uint32_t whole = divide(unit, p.by_slots), slot = unit - whole * p.slots;
  const uint32_t head = divide(whole, p.by_chunks), c = whole - head * p.chunks;
  // Slots are counted over the sequences, one for each 128 queries; those left over lie at the end of a head.  (Slots that can be told from
  // q_start alone, with one to spare for each sequence, left every second one empty for sequences of 128: the CUs that the hardware gives those to had half the
  // work, and 64 such sequences took twice as long.)  A lane looks at one sequence; what is known of the one that has the slot comes from its lane.
  Sequence s = {0, 0, 0u, 0u};
  uint32_t passed = 0, first = 0;
  bool found = false;
  for (uint32_t at = 0; at < p.sequences && !found; at += 64u) {
    Sequence mine = sequence(p, min(at + lane, p.sequences - 1u));
    if (at + lane >= p.sequences) mine.nq = 0u;
    const uint32_t has = (mine.nq + kTileQ - 1u) / kTileQ, upto = passed + sum_up_to_lane(has);
    const uint64_t in = __ballot(slot >= upto - has && slot < upto);
    found = in != 0ull;
    if (found) {
      const uint32_t l = (uint32_t)__builtin_ctzll(in);
      s.q0 = (int32_t)__builtin_amdgcn_readlane((uint32_t)mine.q0, l);
      s.k0 = (int32_t)__builtin_amdgcn_readlane((uint32_t)mine.k0, l);
      s.nq = __builtin_amdgcn_readlane(mine.nq, l);
      s.nk = __builtin_amdgcn_readlane(mine.nk, l);
      // The last queries of a sequence, which see the most keys, come first.  Workgroups go to the four shader engines of an XCD in turn, whatever these
      // have to do: every second four slots are taken backwards, or the first engine always had the longest of four (8 sequences of 1024: 8 % slower).
      const uint32_t end = __builtin_amdgcn_readlane(upto, l), begin = end - __builtin_amdgcn_readlane(has, l), four = slot & ~3u;
      const uint32_t turned = (slot & 4u) == 0u ? slot : max(four, begin) + min(four + 4u, end) - 1u - slot;
      first = (end - 1u - turned) * kTileQ;
    }
    passed = __builtin_amdgcn_readlane(upto, 63);
  }
  if (!found) return;
  const int off = (int)s.nk - (int)s.nq;  // query i sees keys up to i + off

  Wave<DP> w;
  const uint32_t mine = first + wave * 32u + (lane & 31u);
  const bool here = mine < s.nq;
  const uint32_t g = divide(head, p.by_rep);
  w.limit = here ? (int)mine + off : -1;
  w.clear();

  const int last = (int)min(first + kTileQ, s.nq) - 1 + off;  // last key that the workgroup's last query sees,
  const int low = (int)first + off;                           // its first query,
  const bool idle = first + wave * 32u >= s.nq;  // a wave without queries only loads (17 queries of 64 heads on one: 88 -> 76 us)
  const int wave_low = low + (int)wave * 32, high = idle ? -1 : min(wave_low + 31, (int)s.nk - 1);  // the wave's first and last
  const uint32_t keys = last < 0 ? 0u : (uint32_t)last + 1u, parts = chunks_of(keys, p);
  if (c >= parts) return;  // no such chunk
  const uint32_t t0 = c * (p.chunk / KEYS), t1 = min((keys + KEYS - 1u) / KEYS, t0 + p.chunk / KEYS);
  const uint32_t full = low < 0 ? 0u : ((uint32_t)low + 1u) / KEYS;  // tiles that all see (the same for all waves)
  auto issue = [&](uint32_t t, uint32_t to) {
    const int64_t row = s.k0 + (int64_t)t * KEYS;
    const uint32_t left = s.nk - t * KEYS;
    stage<DP, KEYS, 256>(p.K + row * p.k_row + (int64_t)g * p.k_head, p.k_row, left, p.dim, to, threadIdx.x);
    stage<DP, KEYS, 256>(p.V + row * p.v_row + (int64_t)g * p.v_head, p.v_row, left, p.dim, to + kBytes, threadIdx.x);
  };
  const uint32_t lds = lds_at(stages);
  if (t0 < t1) issue(t0, lds);
  const _Float16* q_row = p.Q + (s.q0 + mine) * p.q_row + (int64_t)head * p.q_head;
  w.load(q_row, here, p.dim, lane);
  __builtin_amdgcn_s_waitcnt(0);  // the compiler's loads have come: it has nothing to wait for among the loop's
  uint32_t t = t0, now = 0;
  auto begin = [&]() {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // this wave's pieces of the tile are in LDS
    __syncthreads();                                  // everybody's are, and nobody reads the other stage any more
    if (t + 1u < t1) issue(t + 1u, lds + (now ^ 1u) * 2u * kBytes);
  };
  for (; t < (idle ? t0 : min(full, t1)); ++t, now ^= 1u) {
    begin();
    const uint32_t at = lds + now * 2u * kBytes;
    attend<DP, B, false, false>(w, at, at + kBytes, (int)(t * KEYS), p.scale_log2, lane);
  }
  for (; t < t1; ++t, now ^= 1u) {
    begin();
    const uint32_t at = lds + now * 2u * kBytes;
    const int key0 = (int)(t * KEYS);
    if (key0 <= high) attend<DP, B, true, false>(w, at, at + kBytes, key0, p.scale_log2, lane);
  }
  // Sums that are not finite may come from values that a query does not see, times a weight of 0.  That is found here, once, and then all is done again with
  // an eye on them: to look at every tile's values cost a tenth of short prompts.  A loop of its own, queries read again: what it needs in registers (and spills), the loops above need not
  // have (as one loop that runs twice: 8 prompts of 1024 200 us instead of 196).
  float odd = 0.f;  // NaN, if one is not finite
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) odd = __builtin_fmaf(w.o[d][i], 0.f, odd);
  if (__syncthreads_or(odd != 0.f && full < t1)) {
    w.clear();
    w.load(q_row, here, p.dim, lane);
    __builtin_amdgcn_s_waitcnt(0);
    issue(t0, lds);
    now = 0;
#pragma unroll 1
    for (t = t0; t < t1; ++t, now ^= 1u) {
      begin();
#pragma unroll 1
      for (uint32_t b = 0; b < (uint32_t)B; ++b) {
        const uint32_t at = lds + now * 2u * kBytes + b * (kBytes / B);
        const int key0 = (int)(t * KEYS + b * 32u);
        if (key0 <= high) attend<DP, 1, true, true>(w, at, at + kBytes, key0, p.scale_log2, lane);
      }
    }
    __syncthreads();
  }
  w.l = across(w.l, true);
  const int64_t row = s.q0 + mine;
  if (parts == 1u) {
    // Through LDS, so that 16 (8) lanes write a row: stores of the 8 bytes that a lane has of its query took a seventh of short prompts' time.  The caches
    // need not keep it (64 prompts of 128, 56 heads: 110.8 -> 107.7 us).  Queries gain nothing from coming in whole rows through LDS (124).
    constexpr uint32_t kRow = kPitch<DP> * 2, kPieces = kPitch<DP> / 8;
    const uint32_t mine_at = lds + wave * 32u * kRow;
    const float factor = w.l > 0.f ? 1.f / w.l : w.l;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int a = 0; a < 4; ++a)
        *(__attribute__((address_space(3))) half4*)(uintptr_t)(mine_at + (lane & 31u) * kRow + (((d * 4u + a) ^ (lane & (kPieces - 1u))) << 4) + (lane >> 5) * 8u) =
            half4{(_Float16)(w.o[d][4 * a] * factor), (_Float16)(w.o[d][4 * a + 1] * factor), (_Float16)(w.o[d][4 * a + 2] * factor), (_Float16)(w.o[d][4 * a + 3] * factor)};
#pragma unroll
    for (uint32_t i = 0; i < 32u * kPieces / 64u; ++i) {
      const uint32_t r = i * (64u / kPieces) + lane / kPieces, piece = lane % kPieces, query = first + wave * 32u + r;
      const half8 v = *(lds_half8)(uintptr_t)(mine_at + r * kRow + ((piece ^ (r & (kPieces - 1u))) << 4));
      if (query < s.nq && piece * 8u < p.dim) __builtin_nontemporal_store(v, (half8*)(p.O + (s.q0 + query) * p.o_row + (int64_t)head * p.o_head + piece * 8u));
    }
    if (here && p.lse && lane < 32u) p.lse[(int64_t)head * p.q_rows + row] = log_sum(w.m, w.l);
    return;
  }
  if (!here) return;
  const uint64_t at = ((uint64_t)c * p.part_rows + row) * p.heads + head;
  float* out = p.part_o + at * DP;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int a = 0; a < 4; ++a)
      *(float4v*)(out + d * 32 + a * 8 + (lane >> 5) * 4u) = float4v{w.o[d][4 * a], w.o[d][4 * a + 1], w.o[d][4 * a + 2], w.o[d][4 * a + 3]};
  if (lane < 32u) {
    p.part_ml[at * 2] = w.m;
    p.part_ml[at * 2 + 1] = w.l;
  }
}

// --- few queries to a sequence -------------------------------------------------------------------------------------------------
// Bound by the stream of keys and values (loads that the caches do not keep: 64 tokens behind 300 - 2047 keys, 56 heads of 128, 345 -> 313 us, 6.1 TB/s).  The queries of all heads that share a key head are the 32 columns of a wave; a workgroup has
// a chunk of a sequence's keys, its waves take tiles of 32 in turn, each with two stages of its own in LDS and no barrier, and add
// up what they have at the end.

constexpr uint32_t kFewKeys = 32;
constexpr uint32_t kGridRow = 1u << 23;  // workgroups: a grid has less than 2^32 threads in a direction

template <int DP, uint32_t WAVES>
__global__ __launch_bounds__(WAVES * 64) void attention_few_kernel(AttentionParams p) {
  constexpr int kBytes = kFewKeys * kPitch<DP> * 2;
  __shared__ __align__(kTileAlign) uint8_t stage0[WAVES][2 * kBytes], stage1[WAVES][2 * kBytes];
  static_assert(__alignof__(stage0) % kTileAlign == 0 && __alignof__(stage1) % kTileAlign == 0 && kBytes % kTileAlign == 0, "tiles");
  __shared__ float top[WAVES][32], sum[WAVES][32];
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // chunk outermost: sequences of one length run side by side
  const uint32_t kv_heads = p.heads / p.rep;
  const uint32_t u = blockIdx.y * gridDim.x + blockIdx.x;
  if (u >= p.units) return;
  const uint32_t x = divide(u, p.by_row_blocks), block = u - x * p.row_blocks;
  const uint32_t y = divide(x, p.by_kv_heads), g = x - y * kv_heads;
  const uint32_t b = divide(y, p.by_chunks), c = y - b * p.chunks;
  const Sequence s = sequence(p, b);
  const uint32_t rows = s.nq * p.rep;
  if (block * 32u >= rows) return;
  const uint32_t parts = chunks_of(s.nk, p), begin = c * p.chunk;
  if (c >= parts) return;  // no such chunk
  const uint32_t end = min(s.nk, begin + p.chunk);
  const int off = (int)s.nk - (int)s.nq;

  Wave<DP> w;
  const uint32_t packed = block * 32u + (lane & 31u), query = divide(packed, p.by_rep), head = g * p.rep + packed - query * p.rep;
  const bool here = packed < rows;
  w.limit = here ? (int)query + off : -1;
  w.clear();
  const int low = (int)divide(block * 32u, p.by_rep) + off;  // last key of the wave's first query

  const _Float16* K = p.K + s.k0 * p.k_row + (int64_t)g * p.k_head;
  const _Float16* V = p.V + s.k0 * p.v_row + (int64_t)g * p.v_head;
  auto issue = [&](uint32_t key, uint32_t to) {
    const uint32_t left = key < end ? end - key : 0u;
    stage<DP, kFewKeys, 64, true>(K + (int64_t)key * p.k_row, p.k_row, left, p.dim, to, lane);
    stage<DP, kFewKeys, 64, true>(V + (int64_t)key * p.v_row, p.v_row, left, p.dim, to + kBytes, lane);
  };
  constexpr uint32_t kStep = WAVES * kFewKeys;
  auto tile = [&](uint32_t key, uint32_t at) {
    // all but the other stage's loads, which were issued after this one's
    if (kPitch<DP> == 128) asm volatile("s_waitcnt vmcnt(16)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    if (key < end) {
      if ((int)(key + kFewKeys) - 1 <= low) attend<DP, 1, false, false>(w, at, at + kBytes, (int)key, p.scale_log2, lane);
      else attend<DP, 1, true, true>(w, at, at + kBytes, (int)key, p.scale_log2, lane);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile has been read
    issue(key + 2u * kStep, at);
  };
  uint32_t key = begin + wave * kFewKeys;
  const uint32_t lds0 = lds_at(stage0[wave]), lds1 = lds_at(stage1[wave]);
  issue(key, lds0);
  issue(key + kStep, lds1);
  w.load(p.Q + (s.q0 + query) * p.q_row + (int64_t)head * p.q_head, here, p.dim, lane);
  __builtin_amdgcn_s_waitcnt(0);  // the queries have come: the compiler has nothing to wait for among the loop's loads
  for (; key < end; key += 2u * kStep) {
    tile(key, lds0);
    tile(key + kStep, lds1);
  }
  __builtin_amdgcn_s_waitcnt(0);  // no load into LDS is left
  __syncthreads();

  // the waves' sums, brought to the largest of their m
  w.l = across(w.l, true);
  if (lane < 32u) top[wave][lane] = w.m;
  __syncthreads();
  float m = top[0][lane & 31u];
#pragma unroll
  for (uint32_t i = 1; i < WAVES; ++i) m = fmaxf(m, top[i][lane & 31u]);
  const float down = w.m == -kInf ? 0.f : __builtin_amdgcn_exp2f(w.m - m);
  if (lane < 32u) sum[wave][lane] = w.l * down;
  // [wave][d / 4][query][4], in the stages' place
  float* all = (float*)stage0;
  static_assert(sizeof(stage0) >= sizeof(float) * (WAVES - 1) * 32 * DP, "fits");
  if (wave != 0u) {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        const uint32_t quad = d * 8u + a * 2u + (lane >> 5);
        *(float4v*)(all + (((wave - 1u) * (DP / 4) + quad) * 32u + (lane & 31u)) * 4u) =
            float4v{w.o[d][4 * a] * down, w.o[d][4 * a + 1] * down, w.o[d][4 * a + 2] * down, w.o[d][4 * a + 3] * down};
      }
  }
  __syncthreads();
  if (wave != 0u || !here) return;
  float l = sum[0][lane & 31u];
#pragma unroll
  for (uint32_t i = 1; i < WAVES; ++i) l += sum[i][lane & 31u];
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const uint32_t quad = d * 8u + a * 2u + (lane >> 5);
#pragma unroll
      for (int e = 0; e < 4; ++e) w.o[d][4 * a + e] *= down;
#pragma unroll
      for (uint32_t i = 1; i < WAVES; ++i) {
        const float4v other = *(const float4v*)(all + (((i - 1u) * (DP / 4) + quad) * 32u + (lane & 31u)) * 4u);
#pragma unroll
        for (int e = 0; e < 4; ++e) w.o[d][4 * a + e] += other[e];
      }
    }
  const int64_t row = s.q0 + query;
  if (parts == 1u) {
    store_rows<DP>(w, p.O + row * p.o_row + (int64_t)head * p.o_head, l > 0.f ? 1.f / l : l, p.dim, lane);
    if (p.lse && lane < 32u) p.lse[(int64_t)head * p.q_rows + row] = log_sum(m, l);
    return;
  }
  const uint64_t at = ((uint64_t)c * p.part_rows + (uint64_t)b * p.max_q + query) * p.heads + head;
  float* out = p.part_o + at * DP;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int a = 0; a < 4; ++a)
      *(float4v*)(out + d * 32 + a * 8 + (lane >> 5) * 4u) = float4v{w.o[d][4 * a], w.o[d][4 * a + 1], w.o[d][4 * a + 2], w.o[d][4 * a + 3]};
  if (lane < 32u) {
    p.part_ml[at * 2] = m;
    p.part_ml[at * 2 + 1] = l;
  }
}

// --- chunks joined --------------------------------------------------------------------------------------------------------------
// 32 lanes have four d each of a query row and head, LANES of them side by side every LANES-th chunk; a block has 8 / LANES rows and heads.  The largest m
// of all chunks comes first, so that no load waits for another one's result.  Sums are added in a fixed order.  What has only one chunk of keys that it sees is in
// O already.  (Sums for all of it, and 8 lanes side by side for any number of rows: 64 heads, 2048 queries in three chunks, 307 us instead of 134.)
template <int DP, int LANES>
__global__ __launch_bounds__(256) void attention_join_kernel(AttentionParams p) {
  __shared__ float4v sum_o[8][32];
  __shared__ float sum_l[8];
  const uint32_t lane = threadIdx.x & 63u, part = threadIdx.x >> 5, mine = part % LANES;
  const uint32_t pair = blockIdx.x * (8u / LANES) + part / LANES;
  const uint32_t part_row = divide(pair, p.by_heads), head = pair - part_row * p.heads, d = (threadIdx.x & 31u) * 4u;
  uint32_t b = 0;
  if (p.few) {
    b = divide(part_row, p.by_max_q) + 1u;
  } else {
    for (uint32_t at = 0; at < p.sequences; at += 32u) {  // half a wave has one row
      const uint32_t i = at + (lane & 31u);
      const uint64_t begun = __ballot(i < p.sequences && p.q_start[min(i, p.sequences - 1u)] <= (int64_t)part_row);
      b += __popc((uint32_t)(begun >> (lane & 32u)));
    }
  }
  Sequence s = {0, 0, 0u, 0u};
  if (b > 0u && part_row < p.part_rows) s = sequence(p, b - 1u);
  const int64_t row = p.few ? s.q0 + (part_row - (b - 1u) * p.max_q) : (int64_t)part_row;
  // where there is one chunk, it is in O already
  uint32_t keys = s.nk;
  if (!p.few) keys = (uint32_t)max(0, (int)min(((uint32_t)(row - s.q0) | (kTileQ - 1u)) + 1u, s.nq) + (int)s.nk - (int)s.nq);  // of the row's workgroup
  const uint32_t n = chunks_of(keys, p);
  const bool there = row >= s.q0 && row < s.q0 + s.nq && n > 1u;
  const uint64_t first = (uint64_t)part_row * p.heads + head, step = p.part_rows * p.heads;
  float m = -kInf;
#pragma unroll 4
  for (uint32_t c = 0; c < (there ? n : 0u); ++c) m = fmaxf(m, p.part_ml[(first + c * step) * 2]);
  float l = 0.f;
  float4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (uint32_t c = mine; c < (there ? n : 0u); c += LANES) {
    const float mc = p.part_ml[(first + c * step) * 2], lc = p.part_ml[(first + c * step) * 2 + 1];
    const float4v oc = d < (uint32_t)DP ? *(const float4v*)(p.part_o + (first + c * step) * DP + d) : float4v{0.f, 0.f, 0.f, 0.f};
    const float down = mc == -kInf ? 0.f : __builtin_amdgcn_exp2f(mc - m);  // a chunk of which the query sees no key: its l and o are 0 (or NaN, which stays)
    l += lc * down;
    o += oc * down;
  }
  if (LANES > 1) {
    sum_o[part][threadIdx.x & 31u] = o;
    if (d == 0u) sum_l[part] = l;
    __syncthreads();
    if (mine != 0u) return;
#pragma unroll
    for (int i = 1; i < LANES; ++i) {
      l += sum_l[part + i];
      o += sum_o[part + i][threadIdx.x & 31u];
    }
  }
  if (!there) return;
  if (d == 0u && p.lse) p.lse[(int64_t)head * p.q_rows + row] = log_sum(m, l);
  if (d >= p.dim) return;
  const float factor = l > 0.f ? 1.f / l : l;
  *(half4*)(p.O + row * p.o_row + (int64_t)head * p.o_head + d) =
      half4{(_Float16)(o[0] * factor), (_Float16)(o[1] * factor), (_Float16)(o[2] * factor), (_Float16)(o[3] * factor)};
}

// --- host -----------------------------------------------------------------------------------------------------------------------

static uint32_t padded_dim(uint32_t dim) { return dim <= 64 ? 64 : dim <= 96 ? 96 : 128; }

// Chunks for many queries, by an estimate (us) that takes all sequences to have max_k keys.  `busy` workgroups of 128 queries, two to a CU: on 256 CUs a tile of 64 keys takes
// 1.15 us where half of the CUs have one, 1.6 one on each, 2.2 two on each (of 96 values 0.86 of that, of 64 0.73); sums are written and read, and a second kernel is
// started.  Fewer CUs take their share of it.  512 queries, 64 heads of 128, in front of 512, 2512 and 8512 keys, one chunk and two: 21 and 29, 72 and 66, 216 and 163 us; 32 heads and 8512 keys
// in one, two, four and eight: 153, 129, 91, 105.
static uint32_t chunks_of_many(uint64_t busy, uint64_t part_rows_heads, uint32_t DP, uint64_t max_k, uint64_t most, uint32_t cus) {
  uint32_t best = 1;
  float least = 3e38f;
  const float share = 256.f / (float)cus;
  for (uint32_t c = 1; c == 1 || (c <= most && c * busy <= 4u * cus); c += 1 + c / 8) {
    const float units = (float)(c * busy) * share, tiles = (float)((max_k + 64 * c - 1) / (64 * c));
    const float tile = (0.45f + 0.0043f * DP) * (units <= 128.f ? 1.15f : units <= 256.f ? 1.15f + (units - 128.f) * 0.0036f : units <= 512.f ? 1.6f + (units - 256.f) * 0.0023f : units * 0.0043f);
    const float us = tiles * tile + (c == 1 ? 0.f : 3.f + (float)part_rows_heads * c * DP * (8.f / 4.5e6f) * share);
    if (us < least) {
      least = us;
      best = c;
    }
  }
  return best;
}

AttentionPlan attention_plan(int64_t q_rows, uint32_t sequences, uint32_t heads, uint32_t kv_heads, uint32_t dim, int64_t max_q, int64_t max_k, uint32_t cus) {
  AttentionPlan plan = {};
  const uint32_t rep = heads / kv_heads;
  const uint64_t packed = (uint64_t)max_q * rep, row_blocks = (packed + 31) / 32;  // rows of queries that share keys
  // Few or many queries: the kernel for few has a workgroup for 32 rows, the other one for 128 queries of a head, filled or not.  8 sequences in front of 4000 keys, few and many: 32
  // heads on 4, 8 queries 33 and 96 us, 16: 54 and 91; 4 sequences, 64 heads on 1, 16 queries 39 and 74, 40: 80 and 72; 16 heads of 64 on 16 in front of 1000 keys, 32 queries 17 and 22, 64: 19
  // and 18; 8 sequences in front of 300 keys, 32 heads on 4, 8 queries 14.5 and 12.2, 16: 17.4 and 13.3.
  plan.few = row_blocks <= (rep < 4u || max_k <= 512 ? 1u : rep / 2u) ? 1u : 0u;
  plan.row_blocks = plan.few ? (uint32_t)row_blocks : 0u;
  // workgroups with work if the keys are not split: about.  With few queries one to a CU is enough (4 sequences of 8000 keys, 8 key heads: 256 of them 30 us, 512 34, 1024 38).
  // A chunk has 256 keys at least (1 token behind 1000 keys, 8 key heads: 12.1 us in a graph, 14.6 with 512, 11.6 with 128; behind 4000: 14.3, 15.9, 15.3).
  const uint64_t busy = plan.few ? (uint64_t)sequences * kv_heads * plan.row_blocks : ((uint64_t)q_rows + kTileQ - 1) / kTileQ * heads;
  const uint64_t most = ((uint64_t)max_k + 255) / 256, wanted = plan.few ? cus / (busy ? busy : 1) : chunks_of_many(busy, q_rows * heads, padded_dim(dim), max_k, most, cus);
  uint64_t chunks = wanted < most ? wanted : most;
  if (chunks < 1) chunks = 1;
  plan.chunk = (uint32_t)((((uint64_t)max_k + chunks - 1) / chunks + 127) / 128 * 128);
  if (plan.chunk == 0) plan.chunk = 128;
  plan.chunks = (uint32_t)(((uint64_t)max_k + plan.chunk - 1) / plan.chunk);
  if (plan.chunks == 0) plan.chunks = 1;
  plan.part_rows = plan.few ? (uint64_t)sequences * max_q : (uint64_t)q_rows;
  plan.parts_bytes = plan.chunks > 1 ? plan.part_rows * heads * plan.chunks * (padded_dim(dim) + 2) * sizeof(float) : 0;
  plan.slots = (uint32_t)(q_rows / kTileQ) + sequences;
  plan.units = (plan.few ? busy : (uint64_t)plan.slots * heads) * plan.chunks;
  // Four waves to a workgroup where every CU has one at most (8 key heads, 1000 keys: 11.9 us, 13.1 with two), else two (16 such sequences: 19.9 us, 26.4 with four)
  plan.waves = !plan.few || plan.units <= cus ? 4u : 2u;
  // Tiles of 32 keys where heads have 128 values and there are more than four workgroups to a CU, none of them long: 8 prompts of 1024, 56 heads, 181 us, 196 with 64; 16 of 512 123 and 129; 4 of
  // 2048 303 and 308; 2 of 4096 553 and 549; one of 8192 1050 and 1035; 512 queries behind 2000 keys, 64 heads (512 workgroups) 77 and 63; heads of 96 lose by it (3 chunks of 100 - 700 queries, 32 heads of 80: 75 and 69).
  plan.tile = plan.few || (padded_dim(dim) == 128u && plan.units > 4u * cus && max_k <= 2048) ? 32u : 64u;
  return plan;
}

template <int DP>
static hipError_t run(AttentionParams& p, const AttentionPlan& plan, hipStream_t stream) {
  if (plan.few && plan.waves == 4u) attention_few_kernel<DP, 4><<<p.units, 256, 0, stream>>>(p);
  else if (plan.few) attention_few_kernel<DP, 2><<<dim3(min(p.units, kGridRow), (p.units + kGridRow - 1u) / kGridRow), 128, 0, stream>>>(p);
  else if (DP == 128 && plan.tile == 32u) attention_kernel<DP, DP == 128 ? 32 : 64><<<(p.units + 7u) / 8u * 8u, 256, 0, stream>>>(p);
  else attention_kernel<DP, 64><<<(p.units + 7u) / 8u * 8u, 256, 0, stream>>>(p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.chunks == 1u) return e;
  const uint64_t pairs = p.part_rows * p.heads;
  // 8 lanes of threads side by side where there are many chunks (390 of 100000 keys: the call 25 us, 31 with two), one where there are many rows (16384 of 9 chunks:
  // 59 us, 73 with eight)
  if (pairs >= 8192u) attention_join_kernel<DP, 1><<<(uint32_t)((pairs + 7u) / 8u), 256, 0, stream>>>(p);
  else if (p.chunks <= 32u) attention_join_kernel<DP, 2><<<(uint32_t)((pairs + 3u) / 4u), 256, 0, stream>>>(p);
  else attention_join_kernel<DP, 8><<<(uint32_t)pairs, 256, 0, stream>>>(p);
  return hipGetLastError();
}

hipError_t launch_attention(const AttentionLaunch& a, const AttentionPlan& plan, hipStream_t stream) {
  const uint32_t DP = padded_dim(a.dim);
  AttentionParams p = {};
  p.Q = a.Q, p.K = a.K, p.V = a.V, p.O = a.O, p.lse = a.lse;
  p.q_start = a.q_start, p.k_start = a.k_start, p.k_len = a.k_len;
  p.q_rows = a.q_rows, p.k_rows = a.k_rows;
  p.q_row = a.q_row, p.q_head = a.q_head, p.k_row = a.k_row, p.k_head = a.k_head, p.v_row = a.v_row, p.v_head = a.v_head, p.o_row = a.o_row, p.o_head = a.o_head;
  p.sequences = a.sequences, p.heads = a.heads, p.rep = a.heads / a.kv_heads, p.dim = a.dim, p.max_q = (uint32_t)a.max_q, p.max_k = (uint32_t)a.max_k;
  p.chunk = plan.chunk, p.chunks = plan.chunks;
  p.scale_log2 = a.scale * 1.44269504088896341f;
  p.part_o = a.parts;
  p.part_ml = a.parts + plan.chunks * plan.part_rows * a.heads * DP;
  p.part_rows = plan.part_rows;
  p.few = plan.few;
  p.by_heads = divisor(a.heads), p.by_max_q = divisor((uint32_t)a.max_q);
  p.by_chunk = divisor(p.chunk / 128u);
  p.by_rep = divisor(p.rep), p.by_chunks = divisor(p.chunks), p.by_kv_heads = divisor(a.kv_heads);
  p.row_blocks = plan.row_blocks, p.slots = plan.slots, p.units = (uint32_t)plan.units;
  p.by_row_blocks = divisor(plan.few ? p.row_blocks : 1u), p.by_slots = divisor(p.slots);
  return DP == 64 ? run<64>(p, plan, stream) : DP == 96 ? run<96>(p, plan, stream) : run<128>(p, plan, stream);
}

}  // namespace fls
