// fls_quantize and fls_fp8_gemm: C = W . X with both operands in e4m3 and a power-of-two scale for each 128 consecutive k of a
// row of W and of a token of X.
//
// A power of two is the scale that the matrix instruction takes (v_mfma_scale_f32_16x16x128_f8f6f4: a byte of exponent for every
// lane's 32 values), so scaling costs no instruction: sums run over the whole K in the accumulators, in fp32.  It costs no
// precision either: e4m3 is floating point, so a scale only decides which values become subnormal (under 2^-6 of a block whose
// largest value is over 224).  Inside one instruction products are cut to about 17 bits below the largest of them: 1.5e-5 of C (2-norm,
// normal operands, K 128 - 49152), a fourteenth of what the rounding to fp16 costs.
#include "fls_device.h"
#include "fls_launch.h"

namespace fls {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kBlock = 128;             // k that share a scale = K of one MFMA
constexpr uint32_t kPanel = 4;               // tile columns of a panel
constexpr uint32_t kNowhere = 0x80000000u;   // an offset past every buffer descriptor here: a load from it gives 0

// --- quantising a block -----------------------------------------------------------------------------------------------------

// Largest magnitude of 16 fp16 values, as bits; magnitudes of fp16 are ordered as their bits are.
__device__ __forceinline__ uint32_t largest_bits(const u32x4& a, const u32x4& b) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) m = max_u16(m, max_u16(a[i] & 0x7fff7fffu, b[i] & 0x7fff7fffu));
  return max(m & 0xffffu, m >> 16);
}

// The same over finite values only.
__device__ __forceinline__ uint32_t largest_finite_bits(const u32x4& a, const u32x4& b) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t w = (i < 4 ? a[i & 3] : b[i & 3]) & 0x7fff7fffu;
    const uint32_t lo = w & 0xffffu, hi = w >> 16;
    m = max(m, max(lo < 0x7c00u ? lo : 0u, hi < 0x7c00u ? hi : 0u));
  }
  return m;
}

// Smallest e with a * 2^-e <= 448 = 1.75 * 2^8, plus 127; 127 for a = 0.  a = f * 2^x with f in [1, 2): e = x - 8, one more for f > 1.75.
__device__ __forceinline__ uint32_t scale_byte(uint32_t fp16_bits) {
  const uint32_t f = __builtin_bit_cast(uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)fp16_bits));
  return fp16_bits == 0u ? 127u : (f >> 23) - 8u + ((f & 0x7fffffu) > 0x600000u ? 1u : 0u);
}

// 16 values times 2^(127 - byte), rounded to nearest even; inf and NaN become NaN (the product is exact: a power of two, and fp32
// holds fp16's values over 2^-32 exactly).
__device__ __forceinline__ u32x4 to_e4m3(const u32x4& a, const u32x4& b, uint32_t byte) {
  const float down = __builtin_bit_cast(float, (254u - byte) << 23);
  u32x4 q;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const half4 h = __builtin_bit_cast(half4, i < 2 ? uint2{a[2 * i], a[2 * i + 1]} : uint2{b[2 * i - 4], b[2 * i - 3]});
    int w = __builtin_amdgcn_cvt_pk_fp8_f32((float)h[0] * down, (float)h[1] * down, 0, false);
    q[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32((float)h[2] * down, (float)h[3] * down, w, true);
  }
  return q;
}

// Rows of fp16 -> e4m3 [rows][K] and scales [rows][stride].  Bound by memory: 2 bytes in, 1 out.  A lane takes 16 values (32 B in,
// 16 B out), the eight lanes of a block agree on its largest.  Blocks from K on, up to the stride, have a scale of one.  The caches need not keep what
// is read; what is written they keep where a product follows (KEEP: 12288 x 12288, N = 4096 1 % less), not where a matrix is quantised once (28672 x 7168 102 us, 6.1 TB/s; kept 106).
// FRAGMENTS: the values as the stream kernel reads them, [step][16 rows][half][lane][16] with `columns` groups of 16 rows, whole steps.
template <bool FRAGMENTS, bool KEEP>
__global__ __launch_bounds__(256) void quantize_kernel(const _Float16* W, uint8_t* q, uint8_t* s, uint32_t K, uint32_t stride, Divisor by_slots, uint64_t rows, uint32_t columns) {
  // blocks of a grid row cover kQuantizeRows rows, so that the division is one of small numbers
  const uint64_t row0 = (uint64_t)blockIdx.y * kQuantizeRows;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, r = divide(i, by_slots), slot = i - r * (stride * 8u);
  const uint64_t row = row0 + r;
  const uint32_t k = slot * 16u;
  const bool here = r < kQuantizeRows && row < rows;
  const bool in = here && k < K;
  u32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
  if (in) {
    const u32x4* src = (const u32x4*)(W + row * K + k);
    a = __builtin_nontemporal_load(src);
    b = __builtin_nontemporal_load(src + 1);
  }
  uint32_t m = largest_bits(a, b);
#pragma unroll
  for (int d = 1; d < 8; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  if (m >= 0x7c00u) {  // the eight lanes of a block come here together
    m = largest_finite_bits(a, b);
#pragma unroll
    for (int d = 1; d < 8; d *= 2) m = max(m, (uint32_t)__shfl_xor((int)m, d));
  }
  const uint32_t byte = scale_byte(m);
  if (FRAGMENTS) {
    const uint32_t piece = slot & 7u, step = slot >> 3;
    if (here && step * kBlock < K)
      *(u32x4*)(q + (((uint64_t)step * columns + row / 16u) * 2u + piece % 2u) * 1024u + (piece / 2u * 16u + row % 16u) * 16u) = to_e4m3(a, b, byte);
  } else if (in) {
    const u32x4 v = to_e4m3(a, b, byte);
    if (KEEP) *(u32x4*)(q + row * K + k) = v;
    else __builtin_nontemporal_store(v, (u32x4*)(q + row * K + k));
  }
  if (here && (slot & 7u) == 0u) s[row * stride + slot / 8u] = (uint8_t)byte;
}

// --- products -----------------------------------------------------------------------------------------------------------------

struct Fp8Params {
  const uint8_t *W, *Ws;    // e4m3 [M][K], scales [M][stride]
  const uint8_t *Xq, *Xs;   // e4m3 [N][K], scales [N][stride]
  const _Float16* X;        // [N][K], where the kernel quantises it itself
  _Float16* C;              // [N][M]
  float* parts;             // [slices][N][M] where a K slice is not the whole of K
  uint32_t M, K, N, stride;
  uint32_t steps;           // of 128 k
  uint32_t slices;
  uint32_t units;           // workgroups with work
  uint32_t tiles, tiles_m, tiles_n;
  Divisor by_slices, by_tiles, by_panel;
};

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void* p, uint64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)p, 0, (int)(bytes < 0x7fffffffull ? bytes : 0x7fffffffull), kBufferFlags);
}

__device__ __forceinline__ i32x8 join(const u32x4& a, const u32x4& b) {
  i32x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = (int)a[i], r[4 + i] = (int)b[i];
  return r;
}

__device__ __forceinline__ float4v mfma(const i32x8& a, const i32x8& b, const float4v& c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, (int)sa, 0, (int)sb);
}

// Up to 64 columns: bound by the stream of W.  A workgroup has 16 RB rows and a K slice; its waves take the slice's steps of 128 k in turn, so that they
// read neighbouring 128 B lines of the same rows, a step ahead.  A load takes whole lines, 8 rows of them, which the caches need not keep (lane l: row l & 7,
// piece l >> 3 of 16 B); neighbours at a distance of 8 lanes then exchange a piece each, which leaves MFMA fragments: lane l has bytes 32 (l >> 4) .. + 31
// of row l & 15.  (Loaded as fragments, two loads share every line: it has to stay in the caches for the second: 50257 x 7168, N = 13, 72 us, 65.5 so.)  The waves' sums meet in LDS.
// What counts beside W's own loads is how many lines they ask for: the slice's scales of W are copied to LDS row by row (a byte of each row for every step,
// as many lines again as half of W, cost 8 - 20 %), and X lies in fragment order (from fp16 rows: 10 - 30 % more).
// QUANT: a wave quantises the X that it multiplies itself, in registers, for calls where another kernel in front would cost more.
// One step ahead and eight waves, four for 64 columns: a deeper ring or other numbers of waves were up to 5 % slower (the kernel at 28672 x 7168, N = 64: 53 us in
// four, 56 in eight).
constexpr int stream_waves(int NB) { return NB == 4 ? 4 : 8; }
constexpr uint32_t kStreamSteps = 256, kScalePitch = kStreamSteps + 4;  // steps of a slice at most; bytes from one row's scales to the next's in LDS

template <int RB, int NB, bool QUANT>
__global__ __launch_bounds__(stream_waves(NB) * 64) void fp8_stream_kernel(Fp8Params p) {
  constexpr int WAVES = stream_waves(NB);
  constexpr int kRows = 16 * RB, kPitch = kRows + 4, kScaleRows = kRows + (QUANT ? 0 : 16 * NB);
  constexpr int kSums = WAVES * 16 * kPitch * 4, kScales = kScaleRows * kScalePitch;
  __shared__ __align__(16) uint8_t lds[kSums > kScales ? kSums : kScales];
  float* red = (float*)lds;  // [wave][16][kPitch], once the scales are no longer needed
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t group = divide(blockIdx.x, p.by_slices), slice = blockIdx.x - group * p.slices;
  const uint32_t row0 = group * kRows;
  const uint32_t quads = (p.steps + 3u) / 4u, step0 = divide(slice * quads, p.by_slices) * 4u, step1 = min(p.steps, divide((slice + 1u) * quads, p.by_slices) * 4u);
  const uint32_t rows = min((uint32_t)kRows, p.M - row0);
  const __amdgpu_buffer_rsrc_t wbuf = buffer(p.W + (uint64_t)row0 * p.K, (uint64_t)rows * p.K);
  const __amdgpu_buffer_rsrc_t xbuf = QUANT ? buffer(p.X, (uint64_t)p.N * p.K * 2u) : buffer(p.Xq, (uint64_t)p.steps * (NB * 2048u));
  const uint32_t r = lane & 15u, w_off = (lane & 7u) * p.K + (lane >> 3) * 16u;

  float4v acc[RB][NB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[rb][nb] = float4v{0.f, 0.f, 0.f, 0.f};

  constexpr int XL = QUANT ? 4 : 2;  // loads of X for 16 columns
  struct Stage {
    u32x4 w[RB][2], x[NB][XL];
  } ahead;

  // a step past the slice loads nothing (every offset is nowhere); of a K that is no multiple of 128 the last step has the lanes before K
  auto issue = [&](Stage& s, uint32_t step) {
    const uint32_t k_end = step < step1 ? p.K : 0u;
    const bool in = step * kBlock + (lane >> 3) * 16u < k_end;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        s.w[rb][h] = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(wbuf, in ? w_off + (rb * 16u + h * 8u) * p.K + step * kBlock : kNowhere, 0, kAuxNonTemporal));
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < XL; ++j) {
        uint32_t off;
        const uint32_t k = step * kBlock + (lane >> 4) * 32u + j * 8u;
        if (QUANT) off = k < k_end ? ((nb * 16u + r) * p.K + k) * 2u : kNowhere;
        else off = step < step1 ? ((step * NB + nb) * 2u + j) * 1024u + lane * 16u : kNowhere;
        s.x[nb][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xbuf, off, 0, 0));
      }
  };
  const bool upper = (lane & 8u) != 0u;
  auto fragment = [&](const u32x4& a, const u32x4& b) {  // a: rows 0 - 7, b: rows 8 - 15
    u32x4 first, second;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(upper ? a[i] : b[i]), 0x128, 0xf, 0xf, true);  // from the lane 8 further, in rows of 16
      first[i] = upper ? other : a[i];
      second[i] = upper ? b[i] : other;
    }
    return join(first, second);
  };
  auto consume = [&](Stage& s, uint32_t step) {
    const uint8_t* scale = lds + step - step0;
    i32x8 w[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) w[rb] = fragment(s.w[rb][0], s.w[rb][1]);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      i32x8 x;
      uint32_t xs;
      if (QUANT) {
        uint32_t m = max(largest_bits(s.x[nb][0], s.x[nb][1]), largest_bits(s.x[nb][XL - 2], s.x[nb][XL - 1]));
        m = max(m, (uint32_t)__shfl_xor((int)m, 16));
        m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        if (__any(m >= 0x7c00u)) {
          m = max(largest_finite_bits(s.x[nb][0], s.x[nb][1]), largest_finite_bits(s.x[nb][XL - 2], s.x[nb][XL - 1]));
          m = max(m, (uint32_t)__shfl_xor((int)m, 16));
          m = max(m, (uint32_t)__shfl_xor((int)m, 32));
        }
        xs = scale_byte(m);
        x = join(to_e4m3(s.x[nb][0], s.x[nb][1], xs), to_e4m3(s.x[nb][XL - 2], s.x[nb][XL - 1], xs));
      } else {
        x = join(s.x[nb][0], s.x[nb][1]);
        xs = scale[(kRows + nb * 16u + r) * kScalePitch];
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) acc[rb][nb] = mfma(w[rb], x, acc[rb][nb], scale[(rb * 16u + r) * kScalePitch], xs);
    }
  };

  issue(ahead, step0 + wave);
  const uint32_t words = (step1 - step0 + 3u) / 4u;  // of scales to a row
  for (uint32_t row = threadIdx.x / 16u; row < (uint32_t)kScaleRows; row += WAVES * 4u) {
    const bool of_w = row < (uint32_t)kRows;
    const uint32_t from = of_w ? row : row - kRows;
    const uint32_t* src = (const uint32_t*)((of_w ? p.Ws + (uint64_t)row0 * p.stride : p.Xs) + (uint64_t)from * p.stride + step0);
    const bool there = of_w ? from < rows : from < p.N;
    for (uint32_t j = threadIdx.x % 16u; j < words; j += 16u) *(uint32_t*)(lds + row * kScalePitch + j * 4u) = there ? src[j] : 0x7f7f7f7fu;
  }
  __syncthreads();
  for (uint32_t step = step0 + wave; step < step1; step += WAVES) {
    consume(ahead, step);
    issue(ahead, step + WAVES);
  }

  // 16 columns after the other; lane l has column l & 15, rows 4 (l >> 4) .. + 3 of each 16 x 16
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    __syncthreads();
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) *(float4v*)(red + (wave * 16u + r) * kPitch + rb * 16u + (lane >> 4) * 4u) = acc[rb][nb];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kRows * 16; i += WAVES * 64) {
      const uint32_t c = i / kRows, n = nb * 16u + c, m = i % kRows;
      if (n >= p.N || m >= rows) continue;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) sum += red[(w * 16 + c) * kPitch + m];
      if (p.slices == 1u) p.C[(uint64_t)n * p.M + row0 + m] = (_Float16)sum;
      else p.parts[((uint64_t)slice * p.N + n) * p.M + row0 + m] = sum;
    }
  }
}

// More columns: bound by power and by the loads (12288 x 12288, N = 4096: all inputs zero 464 us at 2.3 GHz), if LDS is read while the matrix cores multiply.  A workgroup of eight waves has TM x TN of C, a wave TM/WM x TN/WN.
// Steps of 128 k of both operands go to LDS without passing through registers, into two stages.  The two waves of a SIMD take turns: while one takes
// its fragments of a step into registers (phase 2 t for the first four waves, 2 t + 1 for the others), the other multiplies; barriers keep them
// in step.  From phase 2 t + 2 on nobody reads step t in LDS, and step t + 2 is loaded in its place, two phases before it is read.  16-byte
// piece c of a row lies at place c ^ (row & 7): eight lanes that read the same piece of eight rows read eight different places.
// Scales come 16 steps at a time, 16 bytes to a row: a row's scales lie apart from its neighbours', so a load for every step asked the L2 for
// half as many lines as the operands do.  12288 x 12288, N = 4096: 485 - 498 us, 2.5 PFLOP/s, matrix cores 61 % busy at 1.9 - 2.0 GHz.
template <int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(512, 2) void fp8_tile_kernel(Fp8Params p) {
  constexpr int kThreads = 512, MT = TM / WM / 16, NT = TN / WN / 16, kRows = TM + TN;
  static_assert(WM * WN == 8, "eight waves");
  constexpr int kStage = kRows * kBlock, kLoads = kRows * 8 / kThreads, kLoadsW = TM * 8 / kThreads;
  static_assert(kLoadsW * kThreads == TM * 8 && kLoads * kThreads == kRows * 8 && TM % 64 == 0 && kRows <= kThreads, "whole loads");
  __shared__ __align__(16) uint8_t stages[2 * kStage];      // TM rows of W, TN of X
  __shared__ __align__(16) uint8_t scales[2 * kRows * 16];  // of 16 steps each
  uint32_t unit;
  if (!xcd_unit(p.units, unit)) return;
  // slice by slice, panels of up to kPanel tile columns, and a panel row by row: the 32 workgroups that run on an XCD at one time have some 8 x 4
  // tiles, whose rows and columns they share through its L2
  const uint32_t slice = divide(unit, p.by_tiles), tile = unit - slice * p.tiles;
  const uint32_t panel = divide(tile, p.by_panel), in_panel = tile - panel * (p.tiles_m * kPanel);
  const uint32_t width = min(kPanel, p.tiles_n - panel * kPanel), tm = in_panel / width, tn = panel * kPanel + in_panel - tm * width;
  const uint32_t step0 = divide(slice * p.steps, p.by_slices), step1 = divide((slice + 1u) * p.steps, p.by_slices);
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t row0 = tm * TM, col0 = tn * TN;
  const uint32_t rows = min((uint32_t)TM, p.M - row0), cols = min((uint32_t)TN, p.N - col0);
  const u32x4 wbuf = descriptor(p.W + (uint64_t)row0 * p.K, (uint64_t)rows * p.K), xbuf = descriptor(p.Xq + (uint64_t)col0 * p.K, (uint64_t)cols * p.K);
  const u32x4 sbuf = descriptor(p.Ws + (uint64_t)row0 * p.stride, (uint64_t)rows * p.stride);
  const u32x4 tbuf = descriptor(p.Xs + (uint64_t)col0 * p.stride, (uint64_t)cols * p.stride);
  const uint32_t stages_at = lds_at(stages) + wave * 1024u, scales_at = lds_at(scales);

  // 16 scales from here on hold those of a step (the last 16 of a row if it has as many); rows of fewer are loaded four at a time
  const bool wide = p.stride >= 16u;
  auto scales_from = [&](uint32_t step) { return wide ? min(step & ~15u, p.stride - 16u) : 0u; };
  const uint32_t load_row = threadIdx.x >> 3, load_k = ((threadIdx.x & 7u) ^ (load_row & 7u)) * 16u;
  auto issue = [&](uint32_t step) {
    if ((step == step0 || ((step & 15u) == 0u && step < step1)) && wave * 64u < (uint32_t)kRows) {  // this wave's 64 rows: all of W or all of X
      const bool of_w = wave * 64u < (uint32_t)TM;
      const uint32_t at = (wave * 64u + lane - (of_w ? 0u : (uint32_t)TM)) * p.stride + scales_from(step);
      if (wide) load_lds<16>(of_w ? sbuf : tbuf, scales_at + (step >> 4 & 1u) * (kRows * 16u) + wave * 1024u, at);
      else
        for (uint32_t j = 0; j < p.stride; j += 4u) load_lds<4>(of_w ? sbuf : tbuf, scales_at + (j / 4u * kRows + wave * 64u) * 4u, at + j);
    }
    const uint32_t k = step * kBlock + load_k;
    const bool in = step < step1 && k < p.K;
    const uint32_t to = stages_at + (step & 1u) * kStage;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool of_w = i < kLoadsW;
      const uint32_t row = (of_w ? i : i - kLoadsW) * (kThreads / 8) + load_row;
      load_lds<16>(of_w ? wbuf : xbuf, to + i * kThreads * 16, in ? row * p.K + k : kNowhere);
    }
  };

  float4v acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
  const uint32_t r = lane & 15u, g = lane >> 4, wm = (wave % WM) * (TM / WM), wn = (wave / WM) * (TN / WN);
  const uint32_t at0 = r * kBlock + ((g ^ (r & 7u)) * 16u), at1 = r * kBlock + (((g + 4u) ^ (r & 7u)) * 16u);
  const uint32_t scale_row = wide ? 16u : 4u;  // bytes from one row's scales to the next's

  i32x8 w[MT], x[NT];
  uint32_t ws[MT], xs[NT];
  auto take = [&](uint32_t step) {
    const uint32_t in_row = step - scales_from(step);
    const uint8_t* stage = stages + (step & 1u) * kStage;
    const uint8_t* scale = scales + (wide ? (step >> 4 & 1u) * kRows * 16u + in_row : in_row / 4u * kRows * 4u + in_row % 4u);
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      xs[j] = scale[(TM + wn + j * 16u + r) * scale_row];
      x[j] = join(*(const u32x4*)(stage + (TM + wn + j * 16u) * kBlock + at0), *(const u32x4*)(stage + (TM + wn + j * 16u) * kBlock + at1));
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      ws[i] = scale[(wm + i * 16u + r) * scale_row];
      w[i] = join(*(const u32x4*)(stage + (wm + i * 16u) * kBlock + at0), *(const u32x4*)(stage + (wm + i * 16u) * kBlock + at1));
    }
  };
  auto multiply = [&]() {
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = mfma(w[i], x[j], acc[i][j], ws[i], xs[j]);
  };
  auto phase_ends = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  issue(step0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  phase_ends();
  if (wave < 4u) {
    for (uint32_t step = step0; step < step1; ++step) {
      issue(step + 1u);
      take(step);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wave has taken the step,
      phase_ends();
      multiply();
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");    // and its pieces of the next one are in LDS
      phase_ends();
    }
    phase_ends();
  } else {
    issue(step0 + 1u);
    phase_ends();
    for (uint32_t step = step0; step < step1; ++step) {
      take(step);
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      phase_ends();
      issue(step + 2u);
      multiply();
      phase_ends();
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no load into LDS outlives the workgroup

  // lane l has column l & 15, rows 4 (l >> 4) .. + 3 of each 16 x 16
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const uint32_t n = wn + j * 16u + r;
    if (n >= cols) continue;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint32_t m = wm + i * 16u + g * 4u;
      const uint64_t at = (uint64_t)(col0 + n) * p.M + row0 + m;
      const bool whole = m + 4u <= rows && (p.M & 3u) == 0u;
      if (p.slices != 1u) {
        float* out = p.parts + (uint64_t)slice * p.N * p.M + at;
        if (whole) *(float4v*)out = acc[i][j];
        else
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (m + e < rows) out[e] = acc[i][j][e];
      } else if (whole) {
        *(half4*)(p.C + at) = half4{(_Float16)acc[i][j][0], (_Float16)acc[i][j][1], (_Float16)acc[i][j][2], (_Float16)acc[i][j][3]};
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (m + e < rows) p.C[at + e] = (_Float16)acc[i][j][e];
      }
    }
  }
}

// C = the slices' sums, in slice order.
__global__ __launch_bounds__(256) void fp8_sum_kernel(const float* parts, _Float16* C, uint64_t values, uint32_t slices) {
  const uint64_t i = ((uint64_t)blockIdx.x * 256u + threadIdx.x) * 4u;
  if (i >= values) return;
  if (i + 4u <= values && (values & 3u) == 0u) {
    float4v sum = *(const float4v*)(parts + i);
    for (uint32_t s = 1; s < slices; ++s) sum += *(const float4v*)(parts + s * values + i);
    *(half4*)(C + i) = half4{(_Float16)sum[0], (_Float16)sum[1], (_Float16)sum[2], (_Float16)sum[3]};
    return;
  }
  for (uint64_t e = i; e < i + 4u && e < values; ++e) {
    float sum = parts[e];
    for (uint32_t s = 1; s < slices; ++s) sum += parts[s * values + e];
    C[e] = (_Float16)sum;
  }
}

// --- host ---------------------------------------------------------------------------------------------------------------------

template <bool FRAGMENTS, bool KEEP>
static hipError_t run_quantize(const _Float16* W, uint8_t* q, uint8_t* s, uint64_t rows, uint32_t K, uint32_t columns, hipStream_t stream) {
  const uint32_t stride = scale_stride(K), slots = stride * 8u;
  const uint64_t a_row = rows < kQuantizeRows ? rows : kQuantizeRows;
  const dim3 grid((uint32_t)((a_row * slots + 255u) / 256u), (uint32_t)((rows + kQuantizeRows - 1) / kQuantizeRows));
  quantize_kernel<FRAGMENTS, KEEP><<<grid, 256, 0, stream>>>(W, q, s, K, stride, divisor(slots), rows, columns);
  return hipGetLastError();
}

hipError_t launch_quantize(const _Float16* W, uint8_t* q, uint8_t* s, uint64_t rows, uint32_t K, hipStream_t stream) {
  return run_quantize<false, false>(W, q, s, rows, K, 0, stream);
}

template <int RB, int NB, bool QUANT>
static hipError_t run_stream(const Fp8Params& p, hipStream_t stream) {
  fp8_stream_kernel<RB, NB, QUANT><<<(p.M + 16 * RB - 1) / (16 * RB) * p.slices, stream_waves(NB) * 64, 0, stream>>>(p);
  return hipGetLastError();
}

template <int TM, int TN, int WM, int WN>
static hipError_t run_tile(Fp8Params& p, hipStream_t stream) {
  p.tiles_m = (p.M + TM - 1) / TM, p.tiles_n = (p.N + TN - 1) / TN;
  p.tiles = p.tiles_m * p.tiles_n;
  p.units = p.tiles * p.slices;
  p.by_tiles = divisor(p.tiles);
  p.by_panel = divisor(p.tiles_m * kPanel);
  fp8_tile_kernel<TM, TN, WM, WN><<<(p.units + 7u) / 8u * 8u, 512, 0, stream>>>(p);
  return hipGetLastError();
}

// Microseconds that sums of S slices cost: a second kernel, and fp32 written and read.
static float sums_us(uint32_t slices, uint32_t M, uint32_t N) { return slices == 1u ? 0.f : 2.5f + (float)slices * M * N * (8.f / 4.5e6f); }

// What a call runs, by an estimate of its time (us) from measured rates on 256 CUs.  Times in the comments below are those of whole calls in a graph.
Fp8Plan fp8_plan(uint32_t M, uint32_t K, uint32_t N, int cus) {
  Fp8Plan best = {};
  float least = 3e38f;
  const uint32_t steps = (K + kBlock - 1) / kBlock;
  const uint64_t room = fp8_parts_bytes() / sizeof(float) / ((uint64_t)M * N);  // slices whose sums there is room for (0: one, with no sums)
  const uint32_t least_slices = (steps + kStreamSteps - 1) / kStreamSteps;
  if (N <= 64 && (least_slices == 1u || least_slices <= room)) {
    // Streams run at 5.6 TB/s.  c workgroups to a CU: up to two, some CUs have one more than others; more even out.  16 and 32 rows to a workgroup read X more
    // often than 64 do - 28672 x 7168, N = 13: 47, 42, 39 us, N = 32: 50 and 45 us in 32 and 64 rows, N = 64: 67 and 55 - and where there is one to a CU they have
    // fewer loads under way: 7168 x 28672, N = 13: 47 us in 32 rows, 42 in 64 and two slices.  12288 x 12288, N = 13: 34 us in four slices of 64 rows (c = 3), 40 in one (c = 3/4).
    const uint32_t nb = fp8_column_groups(N);
    const float extra[3][3] = {{1.f, 1.02f, 1.15f}, {1.f, 1.12f, 1.3f}, {1.f, 1.22f, 1.5f}};
    for (int i = 0; i < 3; ++i)
      for (uint32_t slices = least_slices; slices <= least_slices + 7u; ++slices) {
        if (slices > least_slices && (slices > room || slices * 16u > steps)) break;
        const uint32_t rows = 64u >> i;
        const float c = (float)((M + rows - 1) / rows) * slices / cus, uneven = 0.88f * ceilf(c) / c;
        const float us = (float)M * K / 5.6e6f * (c > 2.f ? 1.03f : uneven > 1.f ? uneven : 1.f) * extra[nb / 2][i] * (c <= 1.f ? 1.f + 0.12f * i : 1.f) +
                         sums_us(slices, M, N);
        if (us < least) {
          least = us;
          best.tile_m = rows;
          best.slices = slices;
        }
      }
    // Up to 16 columns of a small matrix: quantising X on the way (16 rows to a workgroup) costs less than a kernel in front of it.  N = 1: 1024 x 1024 3.9 us
    // against 5.1, 4096 x 4096 8.3 against 9.0, 12288 x 12288 37 against 32; N = 13: 4.0 and 5.4, 9.3 and 9.3, 54 and 34.
    const bool small = N <= 16 && K <= 8192 && (uint64_t)M * K <= (1u << 24);
    best.pass = small ? kFp8StreamQuant : kFp8Stream;
    if (small) best.tile_m = 16, best.slices = 1;
    return best;
  }
  // Tiles: a step of 256 x 256 takes 1.62 us, of 256 x 128 1.1, of 128 x 128 0.62 alone on a CU and 0.56 of two; beside them a workgroup starts and stores.
  // 12288 x 12288, N = 4096: 517, 783, 680 us; 4096 x 4096, N = 2048: 58, 45, 50; 1024 x 1024, N = 256: 22, 16, 12.
  best.pass = kFp8Tile;
  const struct {
    uint32_t m, n;
    float step, start;
  } tiles[3] = {{256, 256, 1.62f, 4.f}, {256, 128, 1.1f, 5.f}, {128, 128, 0.56f, 5.f}};
  for (int i = 0; i < 3; ++i)
    for (uint32_t slices = 1; slices <= 16u; ++slices) {
      if (slices > 1u && (slices > room || slices * 4u > steps)) break;
      const uint64_t units = (uint64_t)((M + tiles[i].m - 1) / tiles[i].m) * ((N + tiles[i].n - 1) / tiles[i].n) * slices;
      const float rounds = (float)((units + cus - 1) / cus), deep = (float)((steps + slices - 1) / slices);
      const float us = (i == 2 ? (rounds == 1.f ? deep * 0.62f : rounds * deep * tiles[i].step) + tiles[i].start * ceilf(rounds / 2.f) : rounds * (deep * tiles[i].step + tiles[i].start)) +
                       sums_us(slices, M, N);
      if (us < least) {
        least = us;
        best.tile_m = tiles[i].m;
        best.tile_n = tiles[i].n;
        best.slices = slices;
      }
    }
  return best;
}

template <int NB>
static hipError_t run_stream_of(const Fp8Params& p, uint32_t rows, hipStream_t stream) {
  return rows == 64u ? run_stream<4, NB, false>(p, stream) : rows == 32u ? run_stream<2, NB, false>(p, stream) : run_stream<1, NB, false>(p, stream);
}

hipError_t launch_fp8(const Fp8Launch& a, hipStream_t stream) {
  const Fp8Plan plan = fp8_plan(a.M, a.K, a.N, a.num_cus);
  Fp8Params p = {};
  p.W = a.W, p.Ws = a.Ws, p.Xq = a.Xq, p.Xs = a.Xs, p.X = a.X, p.C = a.C, p.parts = a.parts;
  p.M = a.M, p.K = a.K, p.N = a.N, p.stride = scale_stride(a.K);
  p.steps = (a.K + kBlock - 1) / kBlock;
  p.slices = plan.slices;
  p.by_slices = divisor(plan.slices);
  hipError_t e = hipSuccess;
  if (plan.pass == kFp8Stream) e = run_quantize<true, true>(a.X, a.Xq, a.Xs, a.N, a.K, fp8_column_groups(a.N), stream);
  else if (plan.pass == kFp8Tile) e = run_quantize<false, true>(a.X, a.Xq, a.Xs, a.N, a.K, 0, stream);
  if (e != hipSuccess) return e;
  if (plan.pass == kFp8StreamQuant) e = run_stream<1, 1, true>(p, stream);
  else if (plan.pass == kFp8Stream)
    e = a.N <= 16 ? run_stream_of<1>(p, plan.tile_m, stream) : a.N <= 32 ? run_stream_of<2>(p, plan.tile_m, stream) : run_stream_of<4>(p, plan.tile_m, stream);
  else if (plan.tile_m == 128u) e = run_tile<128, 128, 4, 2>(p, stream);
  else e = plan.tile_n == 128u ? run_tile<256, 128, 4, 2>(p, stream) : run_tile<256, 256, 2, 4>(p, stream);
  if (e != hipSuccess || plan.slices == 1u) return e;
  const uint64_t values = (uint64_t)a.M * a.N;
  fp8_sum_kernel<<<(uint32_t)((values + 1023u) / 1024u), 256, 0, stream>>>(a.parts, a.C, values, plan.slices);
  return hipGetLastError();
}

}  // namespace fls
