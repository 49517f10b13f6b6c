// Append of keys and values to a paged cache of E4M3 codes: blocks of 64 tokens, a power-of-two scale for each (block, head,
// keys | values).  The layout is the one cache_attn.cu reads: codes [block][head][2][4096], keys as [token][dim], values as
// [dim][token]; scales [block][head][2].
//
//   fresh = least 2^e, e >= -126, with max |finite new value of the block| <= 448 * 2^e
//   scale = fresh where the call begins the block, else max(scale held, fresh)
//   code  = RN_e4m3(x / scale), saturating;  older codes of the block: RN_e4m3(code * scale held / scale)
//
// A scale that is a power of two costs a format with an exponent of its own nothing but part of its subnormal range, and makes every division
// exact: the codes do not depend on the precision they are computed in, and a block whose scale grows keeps its older
// tokens' values as they are, but for those that leave the normal range.
//
// One CTA per head, walking a sequence's blocks.  A thread holds four tokens of eight dims, of the keys and of the values, so that it
// writes keys as 8 bytes per token and values, whose layout is turned, as whole words of four tokens, with no pass through shared memory.
// Reads every element once (2 or 4 bytes) and writes a byte: 32 x 16 heads x 2048 bf16 tokens 64.4 us, 6.2 TB/s, 95 % of the copy rate; sequences
// of 0 to 2048 tokens 38.6 us (82 %: the longest ones' CTAs end last); one token for each of 64 sequences 4.6 us, a chain of
// counts, table, scale and store.  It took eight 16-byte loads under way per thread and packed arithmetic: with four, and
// element by element, instruction issue bound it (55 us where the bytes take 31.6).
#include <cuda_fp16.h>

#include <algorithm>

#include "op_launch.cuh"
#include "pd_internal.h"

using namespace pd;

namespace {

constexpr int kBlk = PD_CACHE_BLOCK;
constexpr int kPart = kBlk * kDh;                 // codes of a block's keys (values) of one head
constexpr long long kAppendCtas = 64 * kSms;      // about nine waves: with 24 per SM the ends of unequal sequences cost 5 %, with 400 the starts of CTAs

struct AppendArgs {
  int heads, n_blocks, max_blocks, rows, max_new;
  const void *k, *v;
  long long k_stride, v_stride;
  const int32_t *row_start, *n_new, *pos_start, *table;
  uint8_t *codes; float *scales; int32_t *status;
};

// Four codes in a word: round to nearest even, saturating; NaN stays NaN.
__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tcvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\tmov.b32 %0, {lo, hi};\n\t}"
      : "=r"(r) : "f"(a), "f"(b), "f"(c), "f"(d));
  return r;
}

// The codes of four tokens (or dims) at another scale: times f, rounded again.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((unsigned short)w));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((unsigned short)(w >> 16)));
  const float2 a = __half22float2(*reinterpret_cast<__half2 *>(&lo)), b = __half22float2(*reinterpret_cast<__half2 *>(&hi));
  return e4m3x4(a.x * f, a.y * f, b.x * f, b.y * f);
}

// Least e >= -126 with amax <= 448 * 2^e, 448 = 1.75 * 2^8; amax given by its bits.
__device__ __forceinline__ int scale_exponent(uint32_t amax_bits) {
  const int k = (int)(amax_bits >> 23) - 127;
  return max(k - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0), -126);
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }      // -126 <= e <= 127

// Eight dims of a token as they lie in memory (zeros where there is no new token), and as numbers.
template <typename T> struct Raw8 { uint4 v[sizeof(T) / 2]; };
__device__ __forceinline__ void unpack8(const Raw8<float> &r, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f[4 * i] = __uint_as_float(r.v[i].x); f[4 * i + 1] = __uint_as_float(r.v[i].y);
    f[4 * i + 2] = __uint_as_float(r.v[i].z); f[4 * i + 3] = __uint_as_float(r.v[i].w);
  }
}
__device__ __forceinline__ void unpack8(const Raw8<__nv_bfloat16> &r, float (&f)[8]) {
  const uint32_t u[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(u[i] << 16);
    f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}

// Eight dims times a power of two, exact (bf16: two at a time; what gets too small for bf16 is far below the smallest code).
__device__ __forceinline__ void scaled8(const Raw8<float> &r, float inv, float (&f)[8]) {
  unpack8(r, f);
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] *= inv;
}
__device__ __forceinline__ void scaled8(const Raw8<__nv_bfloat16> &r, float inv, float (&f)[8]) {
  const __nv_bfloat162 by = __float2bfloat162_rn(inv);
  const uint32_t u[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
  Raw8<__nv_bfloat16> s;
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 x = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&u[i]), by);
    w[i] = *reinterpret_cast<const uint32_t *>(&x);
  }
  s.v[0] = make_uint4(w[0], w[1], w[2], w[3]);
  unpack8(s, f);
}

// Largest magnitude so far, by its bits, NaN left out: two at a time in bf16.
struct AbsMax32 {
  float m = 0.f;
  __device__ __forceinline__ void add(const Raw8<float> &r) {
    float f[8];
    unpack8(r, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(f[i]));
  }
  __device__ __forceinline__ uint32_t bits() const { return __float_as_uint(m); }
};
struct AbsMax16 {
  __nv_bfloat162 m = __floats2bfloat162_rn(0.f, 0.f);
  __device__ __forceinline__ void add(const Raw8<__nv_bfloat16> &r) {
    const uint32_t u[4] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __hmax2(m, __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&u[i])));
  }
  __device__ __forceinline__ uint32_t bits() const {
    const uint32_t w = *reinterpret_cast<const uint32_t *>(&m);
    return max(w << 16, w & 0xffff0000u);
  }
};
template <typename T> struct AbsMaxOf { using type = AbsMax32; };
template <> struct AbsMaxOf<__nv_bfloat16> { using type = AbsMax16; };

template <typename T>
__global__ void __launch_bounds__(128, sizeof(T) == 2 ? 7 : 4) cache_append_kernel(AppendArgs a) {
  __shared__ uint32_t warp_max[2][2][4];
  op_begin();
  const int b = blockIdx.z, h = blockIdx.x, warp = threadIdx.x >> 5, t = threadIdx.x;
  const int n = a.n_new[b], p0 = a.pos_start[b], row0 = a.row_start[b];
  if (n <= 0) return;
  if (n > a.max_new || p0 < 0 || row0 < 0 || (long long)row0 + n > a.rows) {
    if (threadIdx.x == 0 && a.status) *a.status = PD_ERR_ARG;
    return;
  }
  // four tokens of eight dims, of the keys and of the values; keys: neighbouring lanes share a token, values: they share dims
  const int dg[2] = {t & 7, t >> 4}, tg[2] = {t >> 3, t & 15};
  const long long stride[2] = {a.k_stride, a.v_stride}, end = (long long)p0 + n;
  const T *src[2];                                                                // the thread's first token in block 0
#pragma unroll
  for (int w = 0; w < 2; ++w)
    src[w] = static_cast<const T *>(w ? a.v : a.k) + h * kDh + dg[w] * 8 + (row0 - (long long)p0 + tg[w] * 4) * stride[w];
  const int32_t *table = a.table + (size_t)b * a.max_blocks;
  const int j1 = (int)((end - 1) / kBlk);
  int turn = 0;
  for (int j = p0 / kBlk + blockIdx.y; j <= j1; j += gridDim.y, turn ^= 1) {      // blocks of the sequence
    const int lo = max(p0 - j * kBlk, 0), hi = (int)min(end - (long long)j * kBlk, (long long)kBlk);
    const int id = j < a.max_blocks ? table[j] : -1;
    auto is_new = [&](int w, int k) { return tg[w] * 4 + k >= lo && tg[w] * 4 + k < hi; };
    Raw8<T> raw[2][4];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const T *row = src[w] + (long long)j * kBlk * stride[w];
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i)
          raw[w][k].v[i] = is_new(w, k) ? reinterpret_cast<const uint4 *>(row + k * stride[w])[i] : make_uint4(0u, 0u, 0u, 0u);
    }
    if (id < 0 || id >= a.n_blocks) {                                             // the same in all threads
      if (threadIdx.x == 0 && a.status) *a.status = PD_ERR_ARG;
      __syncthreads();                                                            // a half of warp_max is written again behind the barrier of the block between only
      continue;
    }
    const size_t block = (size_t)id * a.heads + h;
    const float2 had = lo > 0 ? reinterpret_cast<const float2 *>(a.scales)[block] : make_float2(0.f, 0.f);
    uint32_t amax[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      typename AbsMaxOf<T>::type most;
#pragma unroll
      for (int k = 0; k < 4; ++k) most.add(raw[w][k]);
      amax[w] = __reduce_max_sync(0xffffffffu, most.bits());
      if ((t & 31) == 0) warp_max[turn][w][warp] = amax[w];
    }
    if (__syncthreads_or(max(amax[0], amax[1]) >= 0x7f800000u)) {                 // infinities set no scale: once more without them
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        amax[w] = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float f[8];
          unpack8(raw[w][k], f);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const uint32_t m = __float_as_uint(f[i]) & 0x7fffffffu;
            amax[w] = max(amax[w], m < 0x7f800000u ? m : 0u);
          }
        }
        amax[w] = __reduce_max_sync(0xffffffffu, amax[w]);
        if ((t & 31) == 0) warp_max[turn][w][warp] = amax[w];
      }
      __syncthreads();
    }
    float scale[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      const uint32_t m = max(max(warp_max[turn][w][0], warp_max[turn][w][1]), max(warp_max[turn][w][2], warp_max[turn][w][3]));
      const float held = w ? had.y : had.x;
      scale[w] = fmaxf(pow2(scale_exponent(m)), held);
      const float inv = 1.f / scale[w];                                           // exact: a power of two
      uint8_t *dst = a.codes + (block * 2 + w) * kPart;
      if (lo > 0 && scale[w] > held) {                                            // older tokens of the block move to the new scale
        const float g = held * inv;
        if (w == 0) {
          for (int i = t; i < lo * (kDh / 4); i += 128) {
            uint32_t *p = reinterpret_cast<uint32_t *>(dst) + i;
            *p = rescale4(*p, g);
          }
        } else {
          for (int i = t; i < kDh * kBlk / 4; i += 128) {
            const int tok = (i & 15) * 4;
            if (tok >= lo) continue;
            uint32_t *p = reinterpret_cast<uint32_t *>(dst) + i;
            const uint32_t r = rescale4(*p, g);
            if (tok + 4 <= lo) *p = r;
            else                                                                  // the word's other bytes are new tokens'
              for (int k = 0; k < lo - tok; ++k) reinterpret_cast<uint8_t *>(p)[k] = (uint8_t)(r >> (8 * k));
          }
        }
      }
      if (tg[w] * 4 + 4 <= lo || tg[w] * 4 >= hi) continue;
      float f[4][8];
#pragma unroll
      for (int k = 0; k < 4; ++k) scaled8(raw[w][k], inv, f[k]);
      if (w == 0) {
        uint8_t *p = dst + tg[w] * 4 * kDh + dg[w] * 8;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (is_new(w, k))
            *reinterpret_cast<uint2 *>(p + k * kDh) = make_uint2(e4m3x4(f[k][0], f[k][1], f[k][2], f[k][3]), e4m3x4(f[k][4], f[k][5], f[k][6], f[k][7]));
      } else {
        const bool whole = is_new(w, 0) && is_new(w, 3);
        uint8_t *p = dst + dg[w] * 8 * kBlk + tg[w] * 4;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t c = e4m3x4(f[0][i], f[1][i], f[2][i], f[3][i]);
          if (whole) *reinterpret_cast<uint32_t *>(p + i * kBlk) = c;
          else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (is_new(w, k)) p[i * kBlk + k] = (uint8_t)(c >> (8 * k));
          }
        }
      }
    }
    if (t == 0) reinterpret_cast<float2 *>(a.scales)[block] = make_float2(scale[0], scale[1]);
  }
}

}  // namespace

extern "C" pd_status pd_cache_append(int32_t dtype, int32_t batch, int32_t n_kv_heads, int32_t n_blocks, int32_t max_blocks, int32_t rows,
                                     int32_t max_new, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                                     const int32_t *row_start, const int32_t *n_new, const int32_t *pos_start, const int32_t *table,
                                     void *codes, float *scales, int32_t *status, void *cuda_stream) {
  if (dtype != PD_DTYPE_FP32 && dtype != PD_DTYPE_BF16) return PD_ERR_ARG;
  if (batch < 1 || batch > 65535 || n_kv_heads < 1 || n_kv_heads > 65535 || n_blocks < 1 || max_blocks < 1 || rows < 0 || max_new < 0) return PD_ERR_ARG;
  const int e = dtype == PD_DTYPE_BF16 ? 2 : 4;
  if (max_new == 0 || rows == 0) {                                                 // nothing to write; a sequence with new tokens all the same is reported
    if (!status || !row_start || !n_new || !pos_start) return PD_OK;
  } else {
    if (!k || !v || !row_start || !n_new || !pos_start || !table || !codes || !scales) return PD_ERR_ARG;
    if (k_stride < (int64_t)n_kv_heads * kDh || v_stride < (int64_t)n_kv_heads * kDh || (k_stride * e) % 16 != 0 || (v_stride * e) % 16 != 0) return PD_ERR_ARG;
    if (!aligned_to(16, k, v, codes) || !aligned_to(8, scales) || !aligned_to(4, table)) return PD_ERR_ARG;
  }
  if (!aligned_to(4, row_start, n_new, pos_start, status)) return PD_ERR_ARG;
  AppendArgs a;
  a.heads = n_kv_heads; a.n_blocks = n_blocks; a.max_blocks = max_blocks; a.rows = rows; a.max_new = max_new;
  a.k = k; a.v = v; a.k_stride = k_stride; a.v_stride = v_stride;
  a.row_start = row_start; a.n_new = n_new; a.pos_start = pos_start; a.table = table;
  a.codes = static_cast<uint8_t *>(codes); a.scales = scales; a.status = status;
  // blocks that max_new tokens touch at most, wherever they begin; a CTA walks several where there are more than keep the GPU busy
  const long long blocks = ((long long)max_new + kBlk - 2) / kBlk + 1, pairs = (long long)n_kv_heads * batch;
  const dim3 grid(n_kv_heads, (unsigned)std::min(65535ll, std::max(1ll, std::min(blocks, kAppendCtas / pairs))), batch);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  const cudaError_t st = op_launch(dtype == PD_DTYPE_BF16 ? cache_append_kernel<__nv_bfloat16> : cache_append_kernel<float>, grid, 128, 0, 1, s, a);
  return op_status(st);
}
