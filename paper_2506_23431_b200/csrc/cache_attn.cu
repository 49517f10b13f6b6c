// Attention of a decode step's rows over a paged cache of E4M3 codes (the layout of cache_append.cu: blocks of 64 tokens, a
// power-of-two scale for each block, head and keys | values).
//
//   score(row, p) = scale * q . k_p;  with a cap: cap * tanh(score / cap);  with a bias: + bias[head][min(end - 1 - p, n_bias - 1)]
//   out(row) = softmax over the visible p (begin <= p < end, p < len) of score . v;  zero where nothing is visible
//
// Bound by the cache's bytes: 128 per (token, kv head), read once for all rows that share the head.  A segment is a
// (sequence, kv head, tile of 16 or 32 rows; a row is a (query row, head of the group)); its blocks are split over CTAs, and in a CTA
// over four warps that work alone: each streams its blocks - keys and values of a (block, head) are 8 KB in one piece -
// through a ring of its own with bulk copies, and reads them with 16-byte loads straight in the order the tensor cores take them, because a contraction does not
// see the order of its terms:
//   keys    [token][dim]: lane (g, t) takes dims 16 t .. 16 t + 15 of a token, four for each of four k16 steps; the queries have the same order;
//   values  [dim][token]: lane (g, t) takes tokens 16 t .. 16 t + 15 of a dim; column c of score tile j is therefore token
//           16 (c >> 1) + 4 (j >> 1) + 2 (j & 1) + (c & 1), and the scores are the next product's operand where they stand.
// Codes are widened to f16 pairs (exact).  Every block has its own maximum: weights 2^(s - max + 15) keep 11 bits down to 2^-29 of
// the largest in f16, the block's sum of values is a fresh accumulator, and only then do the running maximum and the values' scale come in, in 32 bits - a
// block of tiny weights and large values loses nothing.  32-bit queries and weights go through two f16 parts (22 bits).
#include <cuda_fp16.h>
#include <limits.h>

#include <algorithm>

#include "pd_internal.h"

using namespace pd;

namespace {

constexpr int kBlk = PD_CACHE_BLOCK;
constexpr int kPart = kBlk * kDh;                 // codes of a block's keys (values) of one head
constexpr int kStageBytes = 2 * kPart;
constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kStages = 3;
constexpr int kRingBytes = kWarps * kStages * kStageBytes;
constexpr int kSmem = kRingBytes + kWarps * kStages * 8;
constexpr int kCtasPerSm = 2;
constexpr uint32_t kSpinLimit = 1u << 24;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLift = 15.f;                     // weights are 2^(s - max + kLift): at most 2^15 in f16

struct CacheAttnArgs {
  int R, H, HK, G, n_blocks, max_blocks, max_len, tiles, splits, n_bias;
  float scale_log2e, cap_log2e, inv_cap;          // cap_log2e = 0: no cap; inv_cap = 2 * scale / cap * log2(e) (bf16) or scale / cap (fp32)
  const void *q; long long q_row;                 // row b * R + r of the queries at (b * R + r) * q_row
  const uint8_t *codes; const float2 *scales; const int32_t *table, *n_rows, *lens; const int2 *spans; const float *bias;
  void *out; float *part; int32_t *status;
};

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {        // false when the phase did not complete within the limit
  for (uint32_t it = 0; it < kSpinLimit; ++it) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    if (ok) return true;
  }
  return false;
}
__device__ __forceinline__ void fetch(uint32_t dst, const uint8_t *src, uint32_t bar) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(kStageBytes) : "memory");
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(kStageBytes), "r"(bar) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) {    // four codes -> two f16 pairs
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((unsigned short)(w & 0xffffu)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((unsigned short)(w >> 16)));
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&v);
}
// what pack() left of its arguments, rounded in turn
__device__ __forceinline__ uint32_t pack_rest(float lo, float hi, uint32_t packed) {
  const float2 p = __half22float2(*reinterpret_cast<const __half2 *>(&packed));
  return pack(lo - p.x, hi - p.y);
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor_sync(0xffffffffu, v, 1);
  return v + __shfl_xor_sync(0xffffffffu, v, 2);
}
// bytes of a word that hold the code of "no number" (0x7f, 0xff), as 0x80 each
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

__device__ __forceinline__ void load16(const float *p, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = reinterpret_cast<const float4 *>(p)[i];
    f[4 * i] = v.x; f[4 * i + 1] = v.y; f[4 * i + 2] = v.z; f[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ void load16(const __nv_bfloat16 *p, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint4 v = reinterpret_cast<const uint4 *>(p)[i];
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[8 * i + 2 * k] = __uint_as_float(u[k] << 16);
      f[8 * i + 2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void store2(float *p, float a, float b) { *reinterpret_cast<float2 *>(p) = make_float2(a, b); }
__device__ __forceinline__ void store2(__nv_bfloat16 *p, float a, float b) { *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(a, b); }

// One row of the tile that this lane holds columns of: what it sees, and its softmax so far.
struct Row {
  int begin, end;                   // visible positions; begin == end: none
  float mul;                        // score in log2 units (or the cap's argument) per unit of q . code at a key scale of 1
  float m, l;
  const float *bias;                // the head's
};

// T: type of queries and output; MT: 16-row tiles; MOD: cap or bias.  fp32: queries and weights in two f16 parts.
template <typename T, int MT, bool MOD>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) cache_attn_kernel(CacheAttnArgs a) {
  constexpr int NP = sizeof(T) == 4 ? 2 : 1;
  constexpr int ROWS = MT * 16;
  extern __shared__ __align__(128) uint8_t ring[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x, kvh = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles, b = blockIdx.z;
  const uint32_t stage0 = smem_u32(ring) + warp * kStages * kStageBytes, bar0 = smem_u32(ring) + kRingBytes + warp * kStages * 8;
  if (lane == 0) {
    for (int s = 0; s < kStages; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar0 + s * 8) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();

  // ---- the rows and what they see
  const int n_rows = min(max(a.n_rows[b], 0), a.R);
  const int len = (int)min((long long)min(max(a.lens[b], 0), a.max_len), (long long)a.max_blocks * kBlk);
  Row row[MT][2];
  int lo = INT_MAX, hi = 0, all_lo = 0, all_hi = INT_MAX;       // seen by some row; seen by every row that sees anything
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    Row &w = row[i >> 1][i & 1];
    const int m = tile * ROWS + (i >> 1) * 16 + (i & 1) * 8 + g, r = m / a.G, h = kvh * a.G + m % a.G;
    w.begin = w.end = 0; w.mul = 0.f; w.m = -INFINITY; w.l = 0.f; w.bias = nullptr;
    if (r < n_rows) {
      const int2 sp = a.spans ? a.spans[(size_t)b * a.R + r] : make_int2(0, len);
      w.begin = max(sp.x, 0); w.end = min(sp.y, len);
      if (w.begin >= w.end) w.begin = w.end = 0;
      else {
        lo = min(lo, w.begin); hi = max(hi, w.end); all_lo = max(all_lo, w.begin); all_hi = min(all_hi, w.end);
        if (MOD && a.bias) w.bias = a.bias + (size_t)h * a.n_bias;
      }
    }
  }
  lo = __reduce_min_sync(0xffffffffu, lo); hi = __reduce_max_sync(0xffffffffu, hi);
  all_lo = __reduce_max_sync(0xffffffffu, all_lo); all_hi = __reduce_min_sync(0xffffffffu, all_hi);
  const int blk0 = hi > 0 ? lo / kBlk : 0, n_blk = hi > 0 ? (hi + kBlk - 1) / kBlk - blk0 : 0;
  const int c0 = blk0 + (int)((long long)n_blk * split / a.splits), c1 = blk0 + (int)((long long)n_blk * (split + 1) / a.splits);
  const int n = c1 - c0 > warp ? (c1 - c0 - warp + kWarps - 1) / kWarps : 0;       // this warp's blocks: c0 + warp + i * kWarps

  // ---- first copies
  const int32_t *table = a.table + (size_t)b * a.max_blocks + c0 + warp;
  auto block_id = [&](int i) {                                                     // lane's block of a run of 32
    int id = -1;
    if (i < n) {
      id = table[(size_t)i * kWarps];
      if (id < 0 || id >= a.n_blocks) { id = -1; if (a.status) *a.status = PD_ERR_ARG; }
    }
    return id;
  };
  auto block_scale = [&](int id) { return id >= 0 ? a.scales[(size_t)id * a.HK + kvh] : make_float2(0.f, 0.f); };
  auto block_ptr = [&](int id) { return a.codes + ((size_t)max(id, 0) * a.HK + kvh) * kStageBytes; };     // an id out of range is fetched from block 0 and not used
  int ids = block_id(lane), next_ids = -1;
  float2 sc = block_scale(ids), next_sc = make_float2(0.f, 0.f);
#pragma unroll
  for (int s = 0; s < kStages; ++s) {
    const int id = __shfl_sync(0xffffffffu, ids, s);
    if (s < n && lane == 0) fetch(stage0 + s * kStageBytes, block_ptr(id), bar0 + s * 8);
  }

  // ---- queries: dims 16 t + 4 s + {0, 1} | {2, 3} of k16 step s; a row is brought to a largest value in [1, 2) so that f16 holds it
  uint32_t qf[NP][MT][4][4];
#pragma unroll
  for (int i = 0; i < 2 * MT; ++i) {
    Row &w = row[i >> 1][i & 1];
    const int m = tile * ROWS + (i >> 1) * 16 + (i & 1) * 8 + g, r = m / a.G, h = kvh * a.G + m % a.G;
    float f[16];
#pragma unroll
    for (int k = 0; k < 16; ++k) f[k] = 0.f;
    if (w.begin < w.end) load16(static_cast<const T *>(a.q) + ((size_t)b * a.R + r) * a.q_row + h * kDh + 16 * t, f);
    float mx = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) mx = fmaxf(mx, fabsf(f[k]));
    mx = quad_max(mx);
    const int e = min(max((int)(__float_as_uint(mx) >> 23) - 127, -100), 100);
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    w.mul = __uint_as_float((uint32_t)(127 + e) << 23) * (MOD && a.cap_log2e > 0.f ? a.inv_cap : a.scale_log2e);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float x = f[4 * s + 2 * k] * down, y = f[4 * s + 2 * k + 1] * down;
        const uint32_t p = pack(x, y);
        qf[0][i >> 1][s][2 * k + (i & 1)] = p;
        if (NP == 2) qf[NP - 1][i >> 1][s][2 * k + (i & 1)] = pack_rest(x, y, p);
      }
  }

  float o[MT][8][4];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int dn = 0; dn < 8; ++dn) o[mt][dn][0] = o[mt][dn][1] = o[mt][dn][2] = o[mt][dn][3] = 0.f;

  // ---- the blocks
  bool ok = true;
  int st = 0; uint32_t phase = 0;
  for (int i = 0; i < n && ok; ++i) {
    if ((i & 31) == 0) {
      if (i) { ids = next_ids; sc = next_sc; }
      next_ids = block_id(i + 32 + lane);
    }
    if ((i & 31) == 16) next_sc = block_scale(next_ids);
    const int id = __shfl_sync(0xffffffffu, ids, i & 31);
    const float ks = __shfl_sync(0xffffffffu, sc.x, i & 31), vs = __shfl_sync(0xffffffffu, sc.y, i & 31);
    const uint32_t kbase = stage0 + st * kStageBytes, vbase = kbase + kPart;
    ok = __all_sync(0xffffffffu, mbar_wait(bar0 + st * 8, phase));
    const int p0 = (c0 + warp + i * kWarps) * kBlk;
    if (ok && id >= 0) {
      const bool edge = p0 < all_lo || p0 + kBlk > all_hi;                         // some row does not see all of it
      // ---- scores
      float s[MT][8][4];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int token = 16 * (g >> 1) + 4 * (j >> 1) + 2 * (j & 1) + (g & 1);
        const uint4 w = lds128(kbase + token * kDh + t * 16);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) s[mt][j][0] = s[mt][j][1] = s[mt][j][2] = s[mt][j][3] = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t b0, b1;
          widen(u[k], b0, b1);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int p = 0; p < NP; ++p) mma_f16(s[mt][j], qf[p][mt][k], b0, b1);
        }
      }
      // ---- the block's softmax
      uint32_t pf[NP][MT][4][4];
      float keep[MT][2], take[MT][2];                                              // factors of the values so far and of this block's
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          Row &w = row[mt][x];
          const float mul = w.mul * ks;
          float mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float v = s[mt][j][2 * x + e] * mul;
              const int pos = p0 + 16 * t + 4 * (j >> 1) + 2 * (j & 1) + e;
              if (MOD) {
                if (a.cap_log2e > 0.f) v = a.cap_log2e * (NP == 2 ? tanhf(v) : 1.f - __fdividef(2.f, 1.f + ex2(v)));
                if (w.bias) v += w.bias[min(max(w.end - 1 - pos, 0), a.n_bias - 1)] * kLog2e;
              }
              if (edge && (pos < w.begin || pos >= w.end)) v = -INFINITY;
              s[mt][j][2 * x + e] = v;
              mx = fmaxf(mx, v);
            }
          mx = quad_max(mx);
          const float ref = (mx == -INFINITY ? 0.f : mx) - kLift;
          float sum = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float w0 = ex2(s[mt][j][2 * x] - ref), w1 = ex2(s[mt][j][2 * x + 1] - ref);
            sum += w0 + w1;
            const uint32_t p = pack(w0, w1);
            pf[0][mt][j >> 1][2 * (j & 1) + x] = p;
            if (NP == 2) pf[NP - 1][mt][j >> 1][2 * (j & 1) + x] = pack_rest(w0, w1, p);
          }
          const float m_new = fmaxf(w.m, mx), mref = m_new == -INFINITY ? 0.f : m_new;
          keep[mt][x] = ex2(w.m - mref);
          const float tk = ex2(mx - mref);
          w.l = w.l * keep[mt][x] + sum * tk;
          take[mt][x] = tk * vs;
          w.m = m_new;
        }
      // ---- values
      bool nan_seen = false;                                                       // a value that is no number, at a position that some row sees
#pragma unroll
      for (int dn = 0; dn < 8; ++dn) {
        const uint4 w = lds128(vbase + (dn * 8 + g) * kBlk + t * 16);
        uint32_t u[4] = {w.x, w.y, w.z, w.w};
        float tv[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) tv[mt][0] = tv[mt][1] = tv[mt][2] = tv[mt][3] = 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (edge) {                                                              // 0 must not meet what is no number
            const uint32_t nb = nan_bytes(u[k]);
            if (nb) {
#pragma unroll
              for (int y = 0; y < 4; ++y)
                if (nb >> (8 * y) & 0x80u) {
                  const int pos = p0 + 16 * t + 4 * k + y;
                  nan_seen |= pos >= lo && pos < hi;
                  u[k] &= ~(0xffu << (8 * y));
                }
            }
          }
          uint32_t b0, b1;
          widen(u[k], b0, b1);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int p = 0; p < NP; ++p) mma_f16(tv[mt], pf[p][mt][k], b0, b1);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[mt][dn][x] = o[mt][dn][x] * keep[mt][x >> 1] + tv[mt][x] * take[mt][x >> 1];
      }
      if (edge && __any_sync(0xffffffffu, nan_seen)) {
        // rows that see such a value get it after all (values of 0x7f and 0xff at visible positions; not a path of speed)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
          for (int dn = 0; dn < 8; ++dn)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const Row &w = row[mt][x >> 1];
              const uint8_t *v = ring + (vbase - smem_u32(ring)) + (dn * 8 + 2 * t + (x & 1)) * kBlk;
              for (int y = 0; y < kBlk; ++y)
                if ((v[y] & 0x7f) == 0x7f && p0 + y >= w.begin && p0 + y < w.end) o[mt][dn][x] = __int_as_float(0x7fffffff);
            }
      }
    }
    // ---- the stage is free: the copy must not overtake the warp's reads
    __syncwarp();
    const int nx = i + kStages;
    const int nid = __shfl_sync(0xffffffffu, (nx ^ i) & ~31 ? next_ids : ids, nx & 31);
    if (ok && nx < n && lane == 0) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      fetch(stage0 + st * kStageBytes, block_ptr(nid), bar0 + st * 8);
    }
    if (++st == kStages) { st = 0; phase ^= 1; }
  }
  if (!ok) {                                                                       // the other copies in flight must land before the CTA ends
    if (lane == 0 && a.status) *a.status = PD_ERR_TIMEOUT;
    for (int s = 0; s < kStages - 1; ++s) { mbar_wait(bar0 + st * 8, phase); if (++st == kStages) { st = 0; phase ^= 1; } }
  }

  // ---- join the warps: sums of every row, then 64 columns of every row
  __syncthreads();                                                                 // the rings are free
  float *rec = reinterpret_cast<float *>(ring), *ml = rec + kWarps * ROWS * kDh;   // [warp][row][64], [warp][row][2]
#pragma unroll
  for (int mt = 0; mt < MT; ++mt)
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int m = warp * ROWS + mt * 16 + x * 8 + g;
      const bool any = row[mt][x].begin < row[mt][x].end;                          // rows that see nothing went along unmasked
      const float l = quad_sum(row[mt][x].l);
      if (t == 0) { ml[2 * m] = any ? row[mt][x].m : -INFINITY; ml[2 * m + 1] = any ? l : 0.f; }
#pragma unroll
      for (int dn = 0; dn < 8; ++dn)
        store2(rec + m * kDh + ((dn * 8 + 2 * t) ^ ((g & 3) << 3)), any ? o[mt][dn][2 * x] : 0.f, any ? o[mt][dn][2 * x + 1] : 0.f);
    }
  __syncthreads();
  for (int i = threadIdx.x; i < ROWS * (kDh / 2); i += kThreads) {
    const int m = i / (kDh / 2), c = 2 * (i % (kDh / 2)), at = c ^ ((m & 3) << 3);
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) mx = fmaxf(mx, ml[2 * (w * ROWS + m)]);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float l = 0.f, x = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = ex2(ml[2 * (w * ROWS + m)] - ref);
      const float2 v = *reinterpret_cast<const float2 *>(rec + (w * ROWS + m) * kDh + at);
      l += ml[2 * (w * ROWS + m) + 1] * f; x += v.x * f; y += v.y * f;
    }
    const int gm = tile * ROWS + m, r = gm / a.G, h = kvh * a.G + gm % a.G;
    if (a.splits > 1) {
      float *p = a.part + (((size_t)b * gridDim.y + blockIdx.y) * a.splits + split) * ROWS * (kDh + 2) + (size_t)m * (kDh + 2);
      store2(p + c, x, y);
      if (c == 0) store2(p + kDh, mx, l);
    } else if (r < a.R) {
      const float inv = l == 0.f ? 0.f : 1.f / l;                                  // nothing seen: zero
      store2(static_cast<T *>(a.out) + (((size_t)b * a.R + r) * a.H + h) * kDh + c, x * inv, y * inv);
    }
  }
}

// Joins the splits of a row in their order: one warp per (sequence, row, head), two columns per lane.
template <typename T>
__global__ void __launch_bounds__(128) cache_attn_merge_kernel(CacheAttnArgs a, int rows_tile, long long n_out) {
  const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (i >= n_out) return;
  const int h = (int)(i % a.H), r = (int)(i / a.H % a.R), b = (int)(i / a.H / a.R);
  const int kvh = h / a.G, m = r * a.G + h % a.G, tile = m / rows_tile;
  const float *p = a.part + (((size_t)b * a.HK + kvh) * a.tiles + tile) * a.splits * rows_tile * (kDh + 2) + (size_t)(m % rows_tile) * (kDh + 2);
  const size_t step = (size_t)rows_tile * (kDh + 2);
  float mx = -INFINITY;
  for (int s = lane; s < a.splits; s += 32) mx = fmaxf(mx, p[s * step + kDh]);
  for (int x = 16; x; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, x));
  const float ref = mx == -INFINITY ? 0.f : mx;
  float l = 0.f, x = 0.f, y = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const float2 ml = *reinterpret_cast<const float2 *>(p + s * step + kDh), v = *reinterpret_cast<const float2 *>(p + s * step + 2 * lane);
    const float f = ex2(ml.x - ref);
    l += ml.y * f; x += v.x * f; y += v.y * f;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store2(static_cast<T *>(a.out) + i * kDh + 2 * lane, x * inv, y * inv);
}

// Shape of a launch: rows per tile, tiles, splits.  A function of sizes the scratch is asked for with.
struct Plan { int mt, tiles, splits; };

Plan plan_of(int dtype, int batch, int rows, int heads, int kv_heads, int max_len) {
  Plan p;
  const int m = rows * (heads / kv_heads);
  p.mt = dtype == PD_DTYPE_BF16 && m > 16 ? 2 : 1;
  p.tiles = (m + 16 * p.mt - 1) / (16 * p.mt);
  const long long segs = (long long)batch * kv_heads * p.tiles, blocks = ((long long)max_len + kBlk - 1) / kBlk;
  const long long most = std::max(1ll, blocks / kWarps);                           // a block for each warp
  p.splits = (int)std::max(1ll, std::min(most, kSms * kCtasPerSm / segs));
  return p;
}

bool cache_attn_sizes_ok(int dtype, int batch, int rows, int heads, int kv_heads, int max_len) {
  if (dtype != PD_DTYPE_FP32 && dtype != PD_DTYPE_BF16) return false;
  if (batch < 1 || batch > 65535 || rows < 1 || rows > kMaxRows || kv_heads < 1 || heads < kv_heads || heads % kv_heads || heads > 1024) return false;
  return max_len >= 0 && max_len <= INT_MAX - kBlk;
}

size_t scratch_bytes_of(const Plan &p, int batch, int kv_heads) {
  return p.splits > 1 ? (size_t)batch * kv_heads * p.tiles * p.splits * p.mt * 16 * (kDh + 2) * sizeof(float) : 0;
}

template <typename T, int MT>
cudaError_t launch_cache_attn(const CacheAttnArgs &a, int batch, bool mod, cudaStream_t s) {
  auto kernel = mod ? cache_attn_kernel<T, MT, true> : cache_attn_kernel<T, MT, false>;
  cudaError_t st = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (st != cudaSuccess) return st;
  kernel<<<dim3(a.splits, a.HK * a.tiles, batch), kThreads, kSmem, s>>>(a);
  if ((st = cudaGetLastError()) != cudaSuccess || a.splits == 1) return st;
  const long long n_out = (long long)batch * a.R * a.H;
  cache_attn_merge_kernel<T><<<(unsigned)((n_out + 3) / 4), 128, 0, s>>>(a, MT * 16, n_out);
  return cudaGetLastError();
}

}  // namespace

extern "C" {

size_t pd_cache_attention_scratch_bytes(int32_t dtype, int32_t batch, int32_t rows_per_seq, int32_t n_heads, int32_t n_kv_heads, int32_t max_len) {
  if (!cache_attn_sizes_ok(dtype, batch, rows_per_seq, n_heads, n_kv_heads, max_len)) return 0;
  return std::max<size_t>(256, scratch_bytes_of(plan_of(dtype, batch, rows_per_seq, n_heads, n_kv_heads, max_len), batch, n_kv_heads));
}

pd_status pd_cache_attention(int32_t dtype, int32_t batch, int32_t rows_per_seq, int32_t n_heads, int32_t n_kv_heads, int32_t n_blocks,
                             int32_t max_blocks, int32_t max_len, float attn_scale, float softcap, const void *q, int64_t q_stride,
                             const void *codes, const float *scales, const int32_t *table, const int32_t *n_rows, const int32_t *lens,
                             const int32_t *spans, const float *bias, int32_t n_bias, void *out, void *scratch, size_t scratch_bytes,
                             int32_t *status, void *cuda_stream) {
  if (!cache_attn_sizes_ok(dtype, batch, rows_per_seq, n_heads, n_kv_heads, max_len) || n_blocks < 1 || max_blocks < 1) return PD_ERR_ARG;
  if (!q || !codes || !scales || !table || !n_rows || !lens || !out) return PD_ERR_ARG;
  if (!(attn_scale > 0.f) || !(attn_scale < 1e30f) || !(softcap >= 0.f) || !(softcap < 1e30f) || (bias && (n_bias < 1 || n_bias > (1 << 20)))) return PD_ERR_ARG;
  const int e = dtype == PD_DTYPE_BF16 ? 2 : 4;
  if (q_stride < (int64_t)n_heads * kDh || (q_stride * e) % 16 != 0) return PD_ERR_ARG;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(codes) | reinterpret_cast<uintptr_t>(out)) % 16 != 0 ||
      (reinterpret_cast<uintptr_t>(scales) | reinterpret_cast<uintptr_t>(spans)) % 8 != 0 || reinterpret_cast<uintptr_t>(scratch) % 16 != 0) return PD_ERR_ARG;
  const Plan p = plan_of(dtype, batch, rows_per_seq, n_heads, n_kv_heads, max_len);
  if ((long long)n_kv_heads * p.tiles > 65535) return PD_ERR_ARG;
  const size_t need = scratch_bytes_of(p, batch, n_kv_heads);
  if (need && !scratch) return PD_ERR_ARG;
  if (scratch_bytes < need) return PD_ERR_WORKSPACE;
  CacheAttnArgs a;
  a.R = rows_per_seq; a.H = n_heads; a.HK = n_kv_heads; a.G = n_heads / n_kv_heads; a.n_blocks = n_blocks; a.max_blocks = max_blocks; a.max_len = max_len;
  a.tiles = p.tiles; a.splits = p.splits; a.n_bias = bias ? n_bias : 0;
  a.scale_log2e = attn_scale * kLog2e; a.cap_log2e = softcap * kLog2e;
  // tanh(x) = 1 - 2 / (1 + e^2x): the bf16 kernel wants 2 x in log2 units
  a.inv_cap = softcap > 0.f ? (dtype == PD_DTYPE_BF16 ? 2.f * kLog2e : 1.f) * attn_scale / softcap : 0.f;
  a.q = q; a.q_row = q_stride; a.codes = static_cast<const uint8_t *>(codes); a.scales = reinterpret_cast<const float2 *>(scales);
  a.table = table; a.n_rows = n_rows; a.lens = lens; a.spans = reinterpret_cast<const int2 *>(spans); a.bias = bias;
  a.out = out; a.part = static_cast<float *>(scratch); a.status = status;
  const bool mod = softcap > 0.f || bias;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t st;
  if (dtype == PD_DTYPE_FP32) st = launch_cache_attn<float, 1>(a, batch, mod, s);
  else if (p.mt == 1) st = launch_cache_attn<__nv_bfloat16, 1>(a, batch, mod, s);
  else st = launch_cache_attn<__nv_bfloat16, 2>(a, batch, mod, s);
  return st == cudaSuccess ? PD_OK : PD_ERR_CUDA;
}

}  // extern "C"
