// Rotary positions on caller-supplied heads, without a decoder handle: neighbouring dims or the two halves paired, the whole
// head or its first rot_dim dims, frequencies of the caller's choice (pd_rotary_turns has the usual ones), either direction.
//
//   t = 2 pi frac(pos * turns[i]),   y_a = A (x_a cos t - x_b sin t),   y_b = A (x_a sin t + x_b cos t)
//
// A frequency is held as turns per position in 64 bits: the product with the position keeps its fraction of a turn to 2^-52 of
// the product, so that position 10^6 is as exact as position 1, and sincospif gets an argument in [-1, 1].  Sine and cosine
// belong to a (token, pair), not to a head: a CTA computes those of its tokens once into shared memory and then streams all
// heads through it, 16 bytes per load.  One read and one write of every element: HBM-bound for prompts (65536 x 32 bf16 heads 83.8 us in a graph,
// 6.4 TB/s, 98 % of the copy rate; calls on changing buffers up to 94 us, 5.7 TB/s, 87 %; with loads of one token at a time 99.5), one launch latency for a decode
// step (2.2 us).  The bf16 form by halves spills 24 bytes per thread at its 64 registers.
#include <math.h>

#include "op_launch.cuh"
#include "pd_internal.h"

using namespace pd;

namespace {

constexpr int kRotThreads = 256;
constexpr int kRotMaxTokens = 8;         // tokens per CTA
constexpr int kBatch = 4;                // tokens whose loads a thread has under way together
constexpr int kRotMaxHead = 256;

struct RotaryArgs {
  const void *x; void *out;
  long long x_tok, x_head, o_tok, o_head;     // strides in elements
  const int32_t *pos; const double *turns;
  float amplitude;
  int tokens, heads, dh, rot, inverse, copy_rest, tok_per_cta;
};

// What one access moves, as it lies in memory and as numbers.
template <typename T, int VEC> struct Piece;
template <> struct Piece<float, 4> {
  float4 v;
  __device__ __forceinline__ void unpack(float (&f)[4]) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
  __device__ __forceinline__ void pack(const float (&f)[4]) { v = make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct Piece<__nv_bfloat16, 8> {
  uint4 v;
  __device__ __forceinline__ void unpack(float (&f)[8]) const {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(u[i] << 16); f[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u); }
  }
  __device__ __forceinline__ void pack(const float (&f)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    v = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <> struct Piece<float, 2> {
  float2 v;
  __device__ __forceinline__ void unpack(float (&f)[2]) const { f[0] = v.x; f[1] = v.y; }
  __device__ __forceinline__ void pack(const float (&f)[2]) { v = make_float2(f[0], f[1]); }
};
template <> struct Piece<__nv_bfloat16, 4> {
  uint2 v;
  __device__ __forceinline__ void unpack(float (&f)[4]) const {
    f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
    f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
  }
  __device__ __forceinline__ void pack(const float (&f)[4]) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
    v = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
  }
};
template <> struct Piece<float, 1> {
  float v;
  __device__ __forceinline__ void unpack(float (&f)[1]) const { f[0] = v; }
  __device__ __forceinline__ void pack(const float (&f)[1]) { v = f[0]; }
};
template <> struct Piece<__nv_bfloat16, 1> {
  __nv_bfloat16 v;
  __device__ __forceinline__ void unpack(float (&f)[1]) const { f[0] = __bfloat162float(v); }
  __device__ __forceinline__ void pack(const float (&f)[1]) { v = __float2bfloat16_rn(f[0]); }
};

// u c + v s, written out so that every form of the kernel gives the same bits.
__device__ __forceinline__ float turned(float u, float c, float v, float s) { return fmaf(u, c, __fmul_rn(v, s)); }

// VEC elements per access: 16 bytes, 8 where the pairs or the strides allow no more, or 1 where they allow neither.  An item is what one thread
// turns of a head at a time - VEC pairs (halves), VEC / 2 pairs (neighbours), one pair where VEC is 1 - or copies of its rest.  A thread
// keeps its item (or one every 256) and takes it of several tokens at once: loads of kBatch tokens are under way together, the first ones
// while sines and cosines are computed.
template <typename T, bool INTERLEAVED, int VEC>
__global__ void __launch_bounds__(kRotThreads, 4) rotary_kernel(RotaryArgs a) {
  __shared__ float2 cs[kRotMaxTokens * kRotMaxHead / 2];
  op_begin();
  using V = Piece<T, VEC>;
  constexpr bool TWO = !(INTERLEAVED && VEC > 1);                      // an item is two pieces of a head
  constexpr int PAIRS = VEC == 1 ? 1 : INTERLEAVED ? VEC / 2 : VEC;
  const int half = a.rot / 2, tok0 = blockIdx.x * a.tok_per_cta, nt = min(a.tok_per_cta, a.tokens - tok0);
  const int turn_items = half / PAIRS, items = turn_items + (a.copy_rest ? (a.dh - a.rot) / VEC : 0), per_tok = items * a.heads;
  const int threads = blockDim.x, groups = max(threads / per_tok, 1), grp = groups > 1 ? threadIdx.x / per_tok : 0;      // groups of threads that share the tokens
  const int step = groups > 1 ? per_tok : threads, r0 = threadIdx.x - grp * step;
  const int per_item = grp < groups ? (nt - grp + groups * kBatch - 1) / (groups * kBatch) : 0;       // batches of an item
  const int n = r0 < per_tok ? (per_tok - r0 + step - 1) / step * per_item : 0;
  V pa[kBatch], pb[kBatch];
  int at_a = 0, at_b = 0, at_cs = 0, tt0 = 0, h = 0, r = r0, batch = -1;
  bool turn = false;
  auto load = [&] {                                                     // the next batch
    if (++batch == per_item) { batch = 0; r += step; }
    if (batch == 0) {
      h = r / items;
      const int c = r - h * items;
      turn = c < turn_items;
      at_cs = c * PAIRS;
      at_a = !turn ? a.rot + (c - turn_items) * VEC : VEC > 1 ? c * VEC : INTERLEAVED ? 2 * c : c;
      at_b = INTERLEAVED ? at_a + 1 : at_a + half;
    }
    tt0 = grp + batch * groups * kBatch;
    const T *x = static_cast<const T *>(a.x) + h * a.x_head;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int tt = tt0 + k * groups;
      if (tt < nt) {
        const T *p = x + (tok0 + tt) * a.x_tok;
        pa[k] = *reinterpret_cast<const V *>(p + at_a);
        if (TWO && turn) pb[k] = *reinterpret_cast<const V *>(p + at_b);
      }
    }
  };
  if (n > 0) load();
  for (int i = threadIdx.x; i < nt * half; i += threads) {
    const double t = (double)a.pos[tok0 + i / half] * a.turns[i % half];
    float s, c;
    sincospif((float)(2.0 * (t - rint(t))), &s, &c);
    cs[i] = make_float2(c * a.amplitude, (a.inverse ? -s : s) * a.amplitude);
  }
  __syncthreads();
  for (int i = 0; i < n; ++i) {
    if (i) load();
    T *o = static_cast<T *>(a.out) + h * a.o_head;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int tt = tt0 + k * groups;
      if (tt >= nt) break;
      T *p = o + (tok0 + tt) * a.o_tok;
      const float2 *w = cs + tt * half + at_cs;
      if (turn) {
        float x[VEC], y[VEC];
        pa[k].unpack(x);
        if (TWO) {
          pb[k].unpack(y);
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float2 z = w[e];
            const float xa = x[e], xb = y[e];
            x[e] = turned(xa, z.x, -xb, z.y);
            y[e] = turned(xb, z.x, xa, z.y);
          }
          pb[k].pack(y);
          *reinterpret_cast<V *>(p + at_b) = pb[k];
        } else {
#pragma unroll
          for (int e = 0; e < VEC / 2; ++e) {
            const float2 z = w[e];
            const float xa = x[2 * e], xb = x[2 * e + 1];
            x[2 * e] = turned(xa, z.x, -xb, z.y);
            x[2 * e + 1] = turned(xb, z.x, xa, z.y);
          }
        }
        pa[k].pack(x);
      }
      *reinterpret_cast<V *>(p + at_a) = pa[k];
    }
  }
}

// Heads whose rows are 16-byte pieces but whose pairs are not (half a rotated part that is no multiple of a piece, an odd number of pairs): whole head
// rows pass through shared memory, so that loads and stores stay whole pieces, and are turned there pair by pair.
// (65536 x 32 heads, 20 of 64 dims by halves: 115 us; element by element 452, which is left for what is not aligned.)
template <typename T, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotThreads, 4) rotary_staged_kernel(RotaryArgs a) {
  constexpr int VEC = 16 / sizeof(T);
  using V = Piece<T, VEC>;
  using E = Piece<T, 1>;
  __shared__ float2 cs[kRotMaxTokens * kRotMaxHead / 2];
  __shared__ V stage[2][kBatch * kRotThreads];                          // head rows one after the other
  op_begin();
  const int half = a.rot / 2, tok0 = blockIdx.x * a.tok_per_cta, nt = min(a.tok_per_cta, a.tokens - tok0);
  const int chunks = a.dh / VEC, pass = kRotThreads / chunks, mine = threadIdx.x / chunks, c = threadIdx.x - mine * chunks, rows = nt * a.heads;
  V piece[kBatch];
  // piece c of row r of the CTA, in x or out
  auto at = [&](auto *base, long long tok, long long head, int r) {
    const int tt = r / a.heads;
    return base + (tok0 + tt) * tok + (r - tt * a.heads) * head + c * VEC;
  };
  auto load = [&](int r0) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int r = r0 + k * pass + mine;
      if (mine < pass && r < rows) piece[k] = *reinterpret_cast<const V *>(at(static_cast<const T *>(a.x), a.x_tok, a.x_head, r));
    }
  };
  load(0);
  for (int i = threadIdx.x; i < nt * half; i += kRotThreads) {
    const double t = (double)a.pos[tok0 + i / half] * a.turns[i % half];
    float s, co;
    sincospif((float)(2.0 * (t - rint(t))), &s, &co);
    cs[i] = make_float2(co * a.amplitude, (a.inverse ? -s : s) * a.amplitude);
  }
  const int rows_step = kRotThreads / half, row0 = threadIdx.x / half, pair = threadIdx.x - row0 * half;      // a thread turns one pair of every rows_step-th row
  for (int r0 = 0, buf = 0; r0 < rows; r0 += kBatch * pass, buf ^= 1) {
    if (mine < pass) {
#pragma unroll
      for (int k = 0; k < kBatch; ++k) stage[buf][k * pass * chunks + threadIdx.x] = piece[k];
    }
    __syncthreads();                                                    // of the buffer before the last all reads are done, too
    load(r0 + kBatch * pass);
    if (row0 < rows_step) {
      for (int m = row0; m < min(kBatch * pass, rows - r0); m += rows_step) {
        E *row = reinterpret_cast<E *>(&stage[buf][m * chunks]);
        E &ea = row[INTERLEAVED ? 2 * pair : pair], &eb = row[INTERLEAVED ? 2 * pair + 1 : pair + half];
        const float2 z = cs[(r0 + m) / a.heads * half + pair];
        float xa[1], xb[1];
        ea.unpack(xa); eb.unpack(xb);
        const float ya[1] = {turned(xa[0], z.x, -xb[0], z.y)}, yb[1] = {turned(xb[0], z.x, xa[0], z.y)};
        ea.pack(ya); eb.pack(yb);
      }
    }
    __syncthreads();
    if (mine >= pass || (c * VEC >= a.rot && !a.copy_rest)) continue;
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int r = r0 + k * pass + mine;
      if (r < rows) *reinterpret_cast<V *>(at(static_cast<T *>(a.out), a.o_tok, a.o_head, r)) = stage[buf][k * pass * chunks + threadIdx.x];
    }
  }
}

template <typename T>
cudaError_t launch_rotary_staged(const RotaryArgs &a, int interleaved, cudaStream_t s) {
  const int grid = (a.tokens - 1) / a.tok_per_cta + 1;
  return op_launch(interleaved ? rotary_staged_kernel<T, true> : rotary_staged_kernel<T, false>, dim3(grid), kRotThreads, 0, 1, s, a);
}

template <typename T, int VEC>
cudaError_t launch_rotary(const RotaryArgs &a, int interleaved, cudaStream_t s) {
  const int pairs = VEC == 1 ? 1 : interleaved ? VEC / 2 : VEC;
  const long long per_tok = ((long long)a.rot / 2 / pairs + (a.copy_rest ? (a.dh - a.rot) / VEC : 0)) * a.heads;
  // whole groups of a token's items, or even shares of them, so that few threads have none
  const long long shares = (per_tok + kRotThreads - 1) / kRotThreads, busy = shares > 1 ? (per_tok + shares - 1) / shares : kRotThreads / per_tok * per_tok;
  const int threads = (int)((busy + 31) / 32 * 32);
  const int grid = (a.tokens - 1) / a.tok_per_cta + 1;
  return op_launch(interleaved ? rotary_kernel<T, true, VEC> : rotary_kernel<T, false, VEC>, dim3(grid), threads, 0, 1, s, a);
}

}  // namespace

extern "C" {

pd_status pd_rotary_turns(int32_t rot_dim, double theta, int32_t scaling, double factor, int32_t original_len, double fast_turns,
                          double slow_turns, double *turns, float *amplitude) {
  if (!turns || rot_dim < 2 || rot_dim > kRotMaxHead || rot_dim % 2 || !(theta > 1.0) || !isfinite(theta)) return PD_ERR_ARG;
  if (scaling != PD_ROTARY_PLAIN && scaling != PD_ROTARY_LINEAR && scaling != PD_ROTARY_BY_PARTS) return PD_ERR_ARG;
  if (scaling != PD_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return PD_ERR_ARG;
  const double two_pi = 6.283185307179586476925;
  double lo = 0.0, hi = 0.0;
  bool all_slow = false;                               // even the first pair, which makes one turn in 2 pi positions: the ramp would leave it as it is
  if (scaling == PD_ROTARY_BY_PARTS) {
    if (original_len < 1 || !(slow_turns > 0.0) || !(fast_turns >= slow_turns) || !isfinite(fast_turns)) return PD_ERR_ARG;
    // pair index (of rot_dim / 2, as a real number) that makes `n` turns over the original context: theta^(-2 i / rot) L / (2 pi) = n
    auto pair_of = [&](double n) { return rot_dim * log(original_len / (n * two_pi)) / (2.0 * log(theta)); };
    lo = fmax(floor(pair_of(fast_turns)), 0.0);
    hi = fmin(ceil(pair_of(slow_turns)), rot_dim - 1.0);
    all_slow = original_len / two_pi <= slow_turns && original_len / two_pi < fast_turns;
  }
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = pow(theta, -2.0 * i / rot_dim);
    if (scaling == PD_ROTARY_LINEAR) f /= factor;
    if (scaling == PD_ROTARY_BY_PARTS) {
      const double ramp = all_slow ? 1.0 : fmin(fmax((i - lo) / fmax(hi - lo, 1e-3), 0.0), 1.0);
      f = f / factor * ramp + f * (1.0 - ramp);
    }
    turns[i] = f / two_pi;
  }
  if (amplitude) *amplitude = scaling == PD_ROTARY_BY_PARTS ? (float)(0.1 * log(factor) + 1.0) : 1.f;
  return PD_OK;
}

pd_status pd_rotary(int32_t dtype, int32_t tokens, int32_t n_heads, int32_t d_head, int32_t rot_dim, int32_t interleaved, int32_t inverse,
                    const void *x, int64_t x_token_stride, int64_t x_head_stride, const int32_t *positions, const double *turns,
                    float amplitude, void *out, int64_t out_token_stride, int64_t out_head_stride, void *cuda_stream) {
  if (dtype != PD_DTYPE_FP32 && dtype != PD_DTYPE_BF16) return PD_ERR_ARG;
  if (tokens < 0 || n_heads < 1 || n_heads > 65535 || d_head < 2 || d_head > kRotMaxHead) return PD_ERR_ARG;
  if (rot_dim < 2 || rot_dim > d_head || rot_dim % 2) return PD_ERR_ARG;
  if (x_token_stride < 0 || x_head_stride < 0 || out_token_stride < 0 || out_head_stride < 0) return PD_ERR_ARG;
  if (tokens == 0) return PD_OK;
  if (!x || !positions || !turns || !out) return PD_ERR_ARG;
  const size_t e = dtype == PD_DTYPE_BF16 ? 2 : 4;
  if (!aligned_to(e, x, out) || !aligned_to(4, positions) || !aligned_to(8, turns)) return PD_ERR_ARG;
  // the output's heads must not overlap: heads inside tokens, or tokens inside heads
  const bool by_token = (n_heads == 1 || out_head_stride >= d_head) && (tokens == 1 || out_token_stride >= (n_heads - 1) * out_head_stride + d_head);
  const bool by_head = (tokens == 1 || out_token_stride >= d_head) && (n_heads == 1 || out_head_stride >= (tokens - 1) * out_token_stride + d_head);
  if (!by_token && !by_head) return PD_ERR_ARG;
  const bool in_place = x == out;
  if (in_place && (x_token_stride != out_token_stride || x_head_stride != out_head_stride)) return PD_ERR_ARG;
  RotaryArgs a;
  a.x = x; a.out = out;
  a.x_tok = x_token_stride; a.x_head = x_head_stride; a.o_tok = out_token_stride; a.o_head = out_head_stride;
  a.pos = positions; a.turns = turns; a.amplitude = amplitude;
  a.tokens = tokens; a.heads = n_heads; a.dh = d_head; a.rot = rot_dim; a.inverse = inverse != 0;
  a.copy_rest = !in_place && rot_dim < d_head;
  // as many tokens per CTA as leave four CTAs per SM
  a.tok_per_cta = max(1, min(kRotMaxTokens, tokens / (4 * kSms)));
  // whether heads fall into pieces of so many bytes, and the pairs into whole pieces too
  auto pieces = [&](int bytes) {
    return aligned_to(bytes, x, out) && ((x_token_stride | x_head_stride | out_token_stride | out_head_stride) * (int64_t)e) % bytes == 0 && d_head * e % bytes == 0;
  };
  auto whole = [&](int bytes) { return pieces(bytes) && (interleaved ? rot_dim : rot_dim / 2) * e % bytes == 0; };
  // pieces of 8 bytes cost the whole head, the way through shared memory the turned pairs (65536 x 32 bf16 heads by halves, 56 of 64 dims 134 us against 162; 32768 in
  // fp32, 20 of 64 dims 170 against 95)
  const bool by_eight = whole(8) && (rot_dim * 4 > d_head * 3 || !pieces(16));
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t st;
  if (dtype == PD_DTYPE_BF16)
    st = whole(16) ? launch_rotary<__nv_bfloat16, 8>(a, interleaved, s) : by_eight ? launch_rotary<__nv_bfloat16, 4>(a, interleaved, s)
       : pieces(16) ? launch_rotary_staged<__nv_bfloat16>(a, interleaved, s) : launch_rotary<__nv_bfloat16, 1>(a, interleaved, s);
  else
    st = whole(16) ? launch_rotary<float, 4>(a, interleaved, s) : by_eight ? launch_rotary<float, 2>(a, interleaved, s)
       : pieces(16) ? launch_rotary_staged<float>(a, interleaved, s) : launch_rotary<float, 1>(a, interleaved, s);
  return op_status(st);
}

}  // extern "C"
