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
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));

constexpr uint32_t kBlock = 128;             // k that share a scale = K of one MFMA
constexpr uint32_t kNowhere = 0x80000000u;   // an offset past every buffer descriptor here: a load from it gives 0

// --- quantising a block -----------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t max_u16(uint32_t a, uint32_t b) {
  const u16x2 x = __builtin_bit_cast(u16x2, a), y = __builtin_bit_cast(u16x2, b);
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

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
// 16 B out), the eight lanes of a block agree on its largest.  Blocks from K on, up to the stride, have a scale of one.
__global__ __launch_bounds__(256) void quantize_kernel(const _Float16* W, uint8_t* q, uint8_t* s, uint32_t K, uint32_t stride, Divisor by_slots, uint64_t rows) {
  const uint32_t slots = stride * 8u;  // lanes to a row
  // blocks of a grid row cover kQuantizeRows rows, so that the division is one of small numbers
  const uint64_t row0 = (uint64_t)blockIdx.y * kQuantizeRows;
  const uint32_t i = blockIdx.x * 256u + threadIdx.x, r = divide(i, by_slots), slot = i - r * slots;
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
  if (in) __builtin_nontemporal_store(to_e4m3(a, b, byte), (u32x4*)(q + row * K + k));
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
  Divisor by_slices, by_tiles_m;
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

// Up to 64 columns: bound by the stream of W.  A workgroup has 16 RB rows; its waves take its steps of 128 k in turn, so that they
// read neighbouring 128 B lines of the same rows, straight into MFMA fragments (lane l: row l & 15, bytes 16 (l >> 4) .. + 15 and
// the same 64 further: which k a lane contributes is free as long as X uses the same), NS steps ahead.  The waves' sums meet in
// LDS.  With up to 16 columns (QUANT) a wave quantises the X that it multiplies itself, in registers; wider calls find it quantised.
template <int RB, int NB, bool QUANT, int NS, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void fp8_stream_kernel(Fp8Params p) {
  constexpr int kRows = 16 * RB, kPitch = kRows + 4;
  extern __shared__ __align__(16) float red[];  // [WAVES][16 NB][kPitch]
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t group = divide(blockIdx.x, p.by_slices), slice = blockIdx.x - group * p.slices;
  const uint32_t row0 = group * kRows;
  const uint32_t step0 = divide(slice * p.steps, p.by_slices), step1 = divide((slice + 1u) * p.steps, p.by_slices);
  const uint32_t rows = min((uint32_t)kRows, p.M - row0);
  const __amdgpu_buffer_rsrc_t wbuf = buffer(p.W + (uint64_t)row0 * p.K, (uint64_t)rows * p.K);
  const __amdgpu_buffer_rsrc_t sbuf = buffer(p.Ws + (uint64_t)row0 * p.stride, (uint64_t)rows * p.stride);
  const __amdgpu_buffer_rsrc_t xbuf = QUANT ? buffer(p.X, (uint64_t)p.N * p.K * 2u) : buffer(p.Xq, (uint64_t)p.N * p.K);
  const __amdgpu_buffer_rsrc_t tbuf = buffer(QUANT ? p.Ws : p.Xs, (uint64_t)p.N * p.stride);
  const uint32_t r = lane & 15u, k_lane = (lane >> 4) * 16u;
  const uint32_t w_off = r * p.K + k_lane, s_off = r * p.stride;

  float4v acc[RB][NB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) acc[rb][nb] = float4v{0.f, 0.f, 0.f, 0.f};

  constexpr int XL = QUANT ? 4 : 2;  // loads of X for 16 columns
  struct Stage {
    u32x4 w[RB][2], x[NB][XL];
    uint32_t ws[RB], xs[NB];
  } st[NS];

  // a step past the slice loads nothing (every offset is nowhere); of a K that is no multiple of 128 the last step has the lanes before K
  auto issue = [&](Stage& s, uint32_t step) {
    const uint32_t k = step * kBlock + k_lane, k_end = step < step1 ? p.K : 0u;
    const bool in0 = k < k_end, in1 = k + 64u < k_end;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const uint32_t at = w_off + rb * 16u * p.K + step * kBlock;
      s.w[rb][0] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wbuf, in0 ? at : kNowhere, 0, kAuxNonTemporal));
      s.w[rb][1] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wbuf, in1 ? at + 64u : kNowhere, 0, kAuxNonTemporal));
      s.ws[rb] = __builtin_amdgcn_raw_buffer_load_b8(sbuf, step < step1 ? s_off + rb * 16u * p.stride + step : kNowhere, 0, 0);
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const uint32_t at = (nb * 16u + r) * p.K + step * kBlock + k_lane;
#pragma unroll
      for (int j = 0; j < XL; ++j) {
        const bool in = j < XL / 2 ? in0 : in1;
        const uint32_t off = QUANT ? (at + (j / 2) * 64u + (j % 2) * 8u) * 2u : at + j * 64u;
        s.x[nb][j] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(xbuf, in ? off : kNowhere, 0, 0));
      }
      if (!QUANT) s.xs[nb] = __builtin_amdgcn_raw_buffer_load_b8(tbuf, step < step1 ? (nb * 16u + r) * p.stride + step : kNowhere, 0, 0);
    }
  };
  auto consume = [&](Stage& s) {
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
        xs = s.xs[nb];
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) acc[rb][nb] = mfma(join(s.w[rb][0], s.w[rb][1]), x, acc[rb][nb], s.ws[rb], xs);
    }
  };

  uint32_t step = step0 + wave;
#pragma unroll
  for (int i = 0; i < NS; ++i) issue(st[i], step + i * WAVES);
  while (step < step1) {
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      consume(st[i]);  // a step past the slice adds zeros
      issue(st[i], step + (NS + i) * WAVES);
    }
    step += NS * WAVES;
  }

  // lane l has column l & 15, rows 4 (l >> 4) .. + 3 of each 16 x 16
  float* mine = red + wave * (16 * NB * kPitch);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) *(float4v*)(mine + (nb * 16u + r) * kPitch + rb * 16u + (lane >> 4) * 4u) = acc[rb][nb];
  __syncthreads();
  for (uint32_t i = threadIdx.x; i < kRows * 16 * NB; i += WAVES * 64) {
    const uint32_t n = i / kRows, m = i % kRows;
    if (n >= p.N || m >= rows) continue;
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += red[(w * 16 * NB + n) * kPitch + m];
    if (p.slices == 1u) p.C[(uint64_t)n * p.M + row0 + m] = (_Float16)sum;
    else p.parts[((uint64_t)slice * p.N + n) * p.M + row0 + m] = sum;
  }
}

// More columns: bound by the matrix cores (and by power).  A workgroup has TM x TN of C; steps of 128 k of both operands go to LDS
// without passing through registers, one step ahead, and every wave multiplies TM/WM x TN/WN of it.  16-byte piece c of a row lies at
// place c ^ (row & 7), so that eight lanes that read the same piece of eight rows read eight different places.  The two stages are two
// arrays: of one, the compiler would wait for the loads into the next stage before it reads the present one.
template <int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(WM * WN * 64) void fp8_tile_kernel(Fp8Params p) {
  constexpr int kThreads = WM * WN * 64, MT = TM / WM / 16, NT = TN / WN / 16;
  constexpr int kLoads = (TM + TN) * 8 / kThreads, kLoadsW = TM * 8 / kThreads;
  static_assert((TM + TN) % kThreads == 0 && TM % 64 == 0 && kLoadsW * kThreads == TM * 8 && kLoads * kThreads == (TM + TN) * 8, "whole loads");
  __shared__ __align__(16) uint8_t stage0[(TM + TN) * kBlock], stage1[(TM + TN) * kBlock];  // TM rows of W, TN of X
  __shared__ __align__(16) uint8_t scale0[(TM + TN) * 4], scale1[(TM + TN) * 4];            // their scales of four steps
  uint32_t unit;
  if (!xcd_unit(p.units, unit)) return;
  const uint32_t tile = divide(unit, p.by_slices), slice = unit - tile * p.slices;
  const uint32_t tn = divide(tile, p.by_tiles_m), tm = tile - tn * ((p.M + TM - 1) / TM);
  const uint32_t step0 = divide(slice * p.steps, p.by_slices), step1 = divide((slice + 1u) * p.steps, p.by_slices);
  const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t row0 = tm * TM, col0 = tn * TN;
  const uint32_t rows = min((uint32_t)TM, p.M - row0), cols = min((uint32_t)TN, p.N - col0);
  const __amdgpu_buffer_rsrc_t wbuf = buffer(p.W + (uint64_t)row0 * p.K, (uint64_t)rows * p.K);
  const __amdgpu_buffer_rsrc_t xbuf = buffer(p.Xq + (uint64_t)col0 * p.K, (uint64_t)cols * p.K);
  const __amdgpu_buffer_rsrc_t sbuf = buffer(p.Ws + (uint64_t)row0 * p.stride, (uint64_t)rows * p.stride);
  const __amdgpu_buffer_rsrc_t tbuf = buffer(p.Xs + (uint64_t)col0 * p.stride, (uint64_t)cols * p.stride);

  const uint32_t load_row = threadIdx.x >> 3, load_k = ((threadIdx.x & 7u) ^ (load_row & 7u)) * 16u;
  auto issue = [&](uint32_t step, uint8_t* stage, uint8_t* scale) {
    const uint32_t k = step * kBlock + load_k;
    const bool in = step < step1 && k < p.K;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const bool of_w = i < kLoadsW;
      const uint32_t row = (of_w ? i : i - kLoadsW) * (kThreads / 8) + load_row;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(of_w ? wbuf : xbuf, (__attribute__((address_space(3))) void*)(stage + i * kThreads * 16 + wave * 1024u), 16,
                                               in ? row * p.K + k : kNowhere, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < (TM + TN) / kThreads; ++i) {
      const uint32_t first = i * kThreads + wave * 64u;  // this wave's 64 rows: all of W or all of X
      const bool of_w = first < TM;
      const uint32_t row = (of_w ? first : first - TM) + lane;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(of_w ? sbuf : tbuf, (__attribute__((address_space(3))) void*)(scale + first * 4u), 4,
                                               step < step1 ? row * p.stride + (step & ~3u) : kNowhere, 0, 0, 0);
    }
  };

  float4v acc[MT][NT];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = float4v{0.f, 0.f, 0.f, 0.f};
  const uint32_t r = lane & 15u, g = lane >> 4, wm = (wave % WM) * (TM / WM), wn = (wave / WM) * (TN / WN);
  const uint32_t at0 = r * kBlock + ((g ^ (r & 7u)) * 16u), at1 = r * kBlock + (((g + 4u) ^ (r & 7u)) * 16u);

  auto multiply = [&](uint32_t step, const uint8_t* stage, const uint8_t* scale, uint8_t* next, uint8_t* next_scale) {
    __builtin_amdgcn_s_waitcnt(0);  // this wave's pieces of the step are in LDS
    __syncthreads();                // everybody's are, and nobody reads the other stage any more
    issue(step + 1u, next, next_scale);
    const uint8_t* tw = stage + wm * kBlock;
    const uint8_t* tx = stage + (TM + wn) * kBlock;
    const uint8_t* sw = scale + wm * 4u + r * 4u + (step & 3u);
    const uint8_t* sx = scale + (TM + wn) * 4u + r * 4u + (step & 3u);
    i32x8 x[NT];
    uint32_t xs[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) xs[j] = sx[j * 64];
#pragma unroll
    for (int j = 0; j < NT; ++j) x[j] = join(*(const u32x4*)(tx + j * 16 * kBlock + at0), *(const u32x4*)(tx + j * 16 * kBlock + at1));
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const i32x8 w = join(*(const u32x4*)(tw + i * 16 * kBlock + at0), *(const u32x4*)(tw + i * 16 * kBlock + at1));
#pragma unroll
      for (int j = 0; j < NT; ++j) acc[i][j] = mfma(w, x[j], acc[i][j], sw[i * 64], xs[j]);
    }
  };
  issue(step0, stage0, scale0);
  for (uint32_t step = step0; step < step1; step += 2u) {  // a step past the slice is zeros: no way out in the middle, which made the compiler keep the sums twice
    multiply(step, stage0, scale0, stage1, scale1);
    multiply(step + 1u, stage1, scale1, stage0, scale0);
  }
  __builtin_amdgcn_s_waitcnt(0);  // no load into LDS outlives the workgroup

#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const uint32_t n = wn + j * 16u + r;
    if (n >= cols) continue;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const uint32_t m = wm + i * 16u + g * 4u;
      const uint64_t at = (uint64_t)(col0 + n) * p.M + row0 + m;
      if (p.slices != 1u) {
        float* out = p.parts + (uint64_t)slice * p.N * p.M + at;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (m + e < rows) out[e] = acc[i][j][e];
      } else if (m + 4u <= rows && (p.M & 3u) == 0u) {
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

hipError_t launch_quantize(const _Float16* W, uint8_t* q, uint8_t* s, uint64_t rows, uint32_t K, hipStream_t stream) {
  const uint32_t stride = scale_stride(K), slots = stride * 8u;
  const uint64_t a_row = rows < kQuantizeRows ? rows : kQuantizeRows;
  const dim3 grid((uint32_t)((a_row * slots + 255u) / 256u), (uint32_t)((rows + kQuantizeRows - 1) / kQuantizeRows));
  quantize_kernel<<<grid, 256, 0, stream>>>(W, q, s, K, stride, divisor(slots), rows);
  return hipGetLastError();
}

template <int RB, int NB, bool QUANT, int NS, int WAVES>
static hipError_t run_stream(const Fp8Params& p, hipStream_t stream) {
  const size_t lds = (size_t)WAVES * 16 * NB * (16 * RB + 4) * sizeof(float);
  static const hipError_t allowed = hipFuncSetAttribute((const void*)fp8_stream_kernel<RB, NB, QUANT, NS, WAVES>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (allowed != hipSuccess) return allowed;
  fp8_stream_kernel<RB, NB, QUANT, NS, WAVES><<<(p.M + 16 * RB - 1) / (16 * RB) * p.slices, WAVES * 64, lds, stream>>>(p);
  return hipGetLastError();
}

template <int TM, int TN, int WM, int WN>
static hipError_t run_tile(Fp8Params& p, hipStream_t stream) {
  const uint32_t tiles_m = (p.M + TM - 1) / TM, tiles_n = (p.N + TN - 1) / TN;
  p.by_tiles_m = divisor(tiles_m);
  p.units = tiles_m * tiles_n * p.slices;
  fp8_tile_kernel<TM, TN, WM, WN><<<(p.units + 7u) / 8u * 8u, WM * WN * 64, 0, stream>>>(p);
  return hipGetLastError();
}

Fp8Plan fp8_plan(uint32_t M, uint32_t K, uint32_t N, int cus) {
  Fp8Plan plan = {};
  const uint32_t steps = (K + kBlock - 1) / kBlock;
  plan.pass = N <= 16 ? kFp8StreamQuant : N <= 64 ? kFp8Stream : kFp8Tile;
  uint32_t groups;
  if (plan.pass == kFp8Tile) groups = ((M + 255) / 256) * ((N + 255) / 256);
  else groups = (M + 63) / 64;
  uint32_t most = (uint32_t)(fp8_parts_bytes() / sizeof(float) / ((uint64_t)M * N));
  uint32_t slices = (uint32_t)cus / groups;
  if (slices > steps / 8u) slices = steps / 8u;
  if (slices > most) slices = most;
  plan.slices = slices < 1u ? 1u : slices;
  return plan;
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
  if (plan.pass != kFp8StreamQuant) e = launch_quantize(a.X, a.Xq, a.Xs, a.N, a.K, stream);
  if (e != hipSuccess) return e;
  if (plan.pass == kFp8StreamQuant) e = run_stream<4, 1, true, 2, 8>(p, stream);
  else if (plan.pass == kFp8Stream) e = a.N <= 32 ? run_stream<4, 2, false, 2, 8>(p, stream) : run_stream<4, 4, false, 2, 8>(p, stream);
  else e = run_tile<256, 256, 2, 4>(p, stream);
  if (e != hipSuccess || plan.slices == 1u) return e;
  const uint64_t values = (uint64_t)a.M * a.N;
  fp8_sum_kernel<<<(uint32_t)((values + 1023u) / 1024u), 256, 0, stream>>>(a.parts, a.C, values, plan.slices);
  return hipGetLastError();
}

}  // namespace fls
