// Attention of a decode step's rows over a paged cache of E4M3 codes (the layout of cache_append.cu: blocks of 64 tokens, a
// power-of-two scale for each block, head and keys | values).
//
//   score(row, p) = scale * q . k_p;  with a cap: cap * tanh(score / cap);  with a bias: + bias[head][min(end - 1 - p, n_bias - 1)]
//   out(row) = softmax over the visible p (begin <= p < end, p < len) of score . v;  zero where nothing is visible
//
// Bound by the cache's bytes: 128 per (token, kv head), read once for the rows of a tile.  A segment is a (sequence, kv head, tile of 16 rows; a row is a
// (query row, head of the group)); its blocks are split over the CTAs of a cluster and, where segments are few and long, over several clusters, and in a CTA
// over four warps that work alone: each streams its blocks - keys and values of a (block, head) are 4 KB each, in one
// piece - through a ring of its own with bulk copies, and reads them with 16-byte loads straight in the order the tensor
// cores take them, because a contraction does not see the order of its terms:
//   keys    [token][dim]: lane (g, t) takes dims 16 t .. 16 t + 15 of a token, four for each of four k16 steps; the queries have the same order;
//   values  [dim][token]: lane (g, t) takes tokens 16 t .. 16 t + 15 of a dim; column c of score tile j is therefore token
//           16 (c >> 1) + 4 (j >> 1) + 2 (j & 1) + (c & 1), and the scores are the next product's operand where they stand.
// Codes are widened to f16 pairs (exact).  Every block has its own maximum: weights 2^(s - max + 15) keep 11 bits down to 2^-29 of
// the largest in f16, the block's sum of values is a fresh accumulator, and only then do the running maximum and the values' scale come in, in 32 bits - a
// block of tiny weights and large values loses nothing.  32-bit queries and weights go through two f16 parts (22 bits), each with its own sums.
//
// Sixteen warps per SM with four independent products each: with eight warps and products in chains a launch of 32 sequences x 16 heads x 2048 tokens, 12
// rows, took 56 us, now 28.3 (134 MB, 4.8 TB/s; every further 2048 tokens 21.3 us, 6.3 TB/s: what is left is the launch, one round of loads, and the last
// blocks' work and join).  Loads alone take 25.  1 x 12 heads x 777 tokens 5.7 us, 2 x 4 key heads x 131072 tokens 31.1, of which 2.3 the merge of eight clusters.
// A cap costs 2 us in 14, a bias over the table's distances 2.5 in 13.  At 128 registers the bf16 forms spill 24 bytes per thread (fp32 8, with cap or bias 4).
#include <cuda_fp16.h>
#include <float.h>
#include <limits.h>

#include <algorithm>
#include <atomic>

#include "op_launch.cuh"
#include "pd_internal.h"

using namespace pd;

namespace {

constexpr int kBlk = PD_CACHE_BLOCK;
constexpr int kPart = kBlk * kDh;                 // codes of a block's keys (values) of one head
constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kMaxCluster = 8, kClusterSms = 128;
// Fewest blocks for each warp where a segment is split beyond a cluster: what a merge costs (12 heads x 16384 tokens 10.3 us, with four 12.7; 1 x 32768 8.6
// and 11.1; 12 x 4096 would go from 6.8 to about 9 with one).
constexpr int kOuterBlocks = 2;
constexpr int kRows = 16;                         // rows of a tile
// CTAs per SM as the registers allow (128 a thread; two f16 parts 168), and slots of 4 KB (a block's keys, or its values) in a warp's ring: what then
// fits the shared memory (one CTA fewer per SM: 28 -> 37 us).
__host__ __device__ constexpr int ctas_per_sm(bool f32) { return f32 ? 3 : 4; }
__host__ __device__ constexpr int slots(bool f32) { return f32 ? 4 : 3; }
constexpr int kRec = kDh + 4;                     // a row's partial result: 64 sums, maximum, sum of weights, alignment
constexpr int kInboxBytes = kRows * kRec * (int)sizeof(float);
// What a warp looks up rather than holds in registers: scales and ids of two runs of 16 blocks, spans of its rows, its ring's barriers.
constexpr int kRun = 16;
struct WarpNotes { float2 scale[2 * kRun]; int id[2 * kRun]; int2 span[kRows]; uint64_t bar[4]; };
__host__ __device__ constexpr int ring_bytes(bool f32) { return kWarps * slots(f32) * kPart; }
__host__ __device__ constexpr int smem_bytes(bool f32) { return ring_bytes(f32) + kInboxBytes + kWarps * (int)sizeof(WarpNotes); }
constexpr bool all_resident(bool f32) { return (smem_bytes(f32) + 1024) * ctas_per_sm(f32) <= 228 * 1024; }      // of 228 KB per SM each CTA takes 1 KB besides
static_assert(all_resident(false) && all_resident(true), "shared memory for ctas_per_sm CTAs");
constexpr uint32_t kSpinLimit = 1u << 24;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLift = 15.f, kDrop = 0x1p-15f;   // weights are 2^(s - max + kLift): at most 2^15 in f16; kDrop takes the lift out again
// Scores from this size on have a last place of half a weight's step and more; kMostSum bounds 64 products of a query below 4 and a code up to 448.
// (The vote on it: 32 x 16 heads x 2048 tokens, 12 rows, bf16 28.3 us instead of 27.9; differences everywhere 29.0.  fp32, whose products leave room: differences 50.1, vote 52.0,
// neither 49.7.)
constexpr float kCoarse = 0x1p22f, kMostSum = 0x1p17f;
// A score whose bias is below -2e38 counts as minus infinity (scores without a bias are lost in its last place).
constexpr float kGone = -2e38f * kLog2e;
// Sums of values keep the lift (the factor of a block of the smallest scales stays a normal number) until a warp meets a block of this scale: its lifted sums could overflow
// where sums of the values do not.  Of smaller blocks 2^31 tokens cannot.  (Taking the lift out with every block's factor, and with its sums where the factor gets too
// small: 32 x 16 heads x 2048 tokens 28.8 us instead of 28.0.)
constexpr float kLarge = 0x1p64f;
// Largest cap whose tanh is taken as a quotient where weights are f16: the quotient is a difference of numbers near the cap, and a score is off by up to 2^-21 of the cap,
// whatever its own size - 2^-15 at this one, an eighth of the weights' rounding.  tanhf is off by its own last place (32 x 16 heads x 2048 tokens, 12 rows: no cap 28.3 us,
// quotient 35.2, tanhf 41.7).
constexpr float kQuotientCap = 64.f;

struct CacheAttnArgs {
  int R, H, HK, G, n_blocks, max_blocks, max_len, tiles, cluster, outer, n_bias;
  int cap;                                        // 0: none; tanh(x) as 1: 1 - 2 / (1 + e^2x), 2: tanhf(x)
  float factor, cap_log2e, inv_cap;               // of q . k: scale * log2(e), by quotient 2 * scale / cap * log2(e); 1 / cap_log2e, a step of its own in tanhf's argument, since
                                                  // scale / cap may be too small for a number where the scores are not
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
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(kPart) : "memory");
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(kPart), "r"(bar) : "memory");
}
template <typename V>
__device__ __forceinline__ void async_copy(V *dst, const V *src) {                 // 4 or 8 bytes into shared memory, through no register
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(dst)), "l"(src), "n"(sizeof(V)) : "memory");
}
__device__ __forceinline__ void async_copies_land() {                              // the warp's copies are visible to all its lanes
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncwarp();
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
__device__ __forceinline__ void mma_f16_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {      // onto zero
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) {    // four codes -> two f16 pairs
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(w));
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
__device__ __forceinline__ float rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
  return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, int rank) {           // the same place of another CTA of the cluster
  uint32_t at;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
  return at;
}
__device__ __forceinline__ void peer_st4(uint32_t at, float4 v) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// bytes of a word that hold the code of "no number" (0x7f, 0xff), as 0x80 each
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// the first n bytes of a word
__device__ __forceinline__ uint32_t below(int n) { return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1; }

// Sixteen dims of a row as they lie in memory, and as numbers.
template <typename T> struct Raw16 { uint4 v[sizeof(T)]; };
__device__ __forceinline__ void unpack16(const Raw16<float> &r, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[4 * i] = __uint_as_float(r.v[i].x); f[4 * i + 1] = __uint_as_float(r.v[i].y);
    f[4 * i + 2] = __uint_as_float(r.v[i].z); f[4 * i + 3] = __uint_as_float(r.v[i].w);
  }
}
__device__ __forceinline__ void unpack16(const Raw16<__nv_bfloat16> &r, float (&f)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t u[4] = {r.v[i].x, r.v[i].y, r.v[i].z, r.v[i].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      f[8 * i + 2 * k] = __uint_as_float(u[k] << 16);
      f[8 * i + 2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
    }
  }
}
__device__ __forceinline__ void store4(float *p, float4 v) { *reinterpret_cast<float4 *>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float4 v) {
  const __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
  *reinterpret_cast<uint2 *>(p) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}
__device__ __forceinline__ void store2(float *p, float a, float b) { *reinterpret_cast<float2 *>(p) = make_float2(a, b); }
__device__ __forceinline__ void store2(__nv_bfloat16 *p, float a, float b) { *reinterpret_cast<__nv_bfloat162 *>(p) = __floats2bfloat162_rn(a, b); }

// One row of the tile that this lane holds columns of: its softmax so far.
struct Row {
  float unit;                       // of the queries as the tensor cores hold them: a power of two
  float m, l;
};

// T: type of queries and output; MOD: cap or bias.  fp32: queries and weights in two f16 parts.
template <typename T, bool MOD>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(sizeof(T) == 4)) cache_attn_kernel(CacheAttnArgs a) {
  constexpr int NP = sizeof(T) == 4 ? 2 : 1, NS = slots(NP == 2), RING = ring_bytes(NP == 2);
  extern __shared__ __align__(128) uint8_t ring[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x, splits = gridDim.x, kvh = blockIdx.y / a.tiles, tile = blockIdx.y % a.tiles, b = blockIdx.z;
  WarpNotes &notes = reinterpret_cast<WarpNotes *>(ring + RING + kInboxBytes)[warp];
  const uint32_t slot0 = smem_u32(ring) + warp * NS * kPart, bar0 = smem_u32(notes.bar);
  if (lane == 0) {
    for (int s = 0; s < NS; ++s) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(bar0 + s * 8) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  if (a.cluster > 1) cluster_arrive();             // waited for where the first CTA writes into another
  op_begin();

  // ---- one round of independent loads: counts, the table where the blocks are if the sequence has its full length, spans, queries
  const int blocks_most = (int)min(((long long)a.max_len + kBlk - 1) / kBlk, (long long)a.max_blocks);
  const int32_t *table = a.table + (size_t)b * a.max_blocks;
  // this CTA's share of n blocks: the first n % splits CTAs have one more
  auto share = [&](int n, int k) { const int q = n / splits; return q * k + min(k, n - q * splits); };
  const int guess = share(blocks_most, split), guess_at = guess + warp + lane * kWarps;
  const int rows_here = a.n_rows[b], len_here = a.lens[b], guess_id = guess_at < a.max_blocks ? table[guess_at] : -1;
  int2 span[2];
  Raw16<T> qv[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int m = tile * kRows + i * 8 + g, r = m / a.G, h = kvh * a.G + m % a.G;
    span[i] = make_int2(0, INT_MAX);
#pragma unroll
    for (int k = 0; k < (int)sizeof(T); ++k) qv[i].v[k] = make_uint4(0u, 0u, 0u, 0u);
    if (r < a.R) {
      if (a.spans) span[i] = a.spans[(size_t)b * a.R + r];
      const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const T *>(a.q) + ((size_t)b * a.R + r) * a.q_row + h * kDh + 16 * t);
#pragma unroll
      for (int k = 0; k < (int)sizeof(T); ++k) qv[i].v[k] = src[k];
    }
  }

  // ---- the rows and what they see
  const int n_rows = min(max(rows_here, 0), a.R);
  const int len = (int)min((long long)min(max(len_here, 0), a.max_len), (long long)a.max_blocks * kBlk);
  Row row[2];
  int lo = INT_MAX, hi = 0, all_lo = 0, all_hi = INT_MAX;       // seen by some row; seen by every row that sees anything
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    Row &w = row[i];
    const int r = (tile * kRows + i * 8 + g) / a.G;
    int2 sp = make_int2(0, 0);                                  // begin == end: the row sees nothing
    w.m = -INFINITY; w.l = 0.f;
    if (r < n_rows) {
      sp = make_int2(max(span[i].x, 0), min(span[i].y, len));
      if (sp.x >= sp.y) sp.x = sp.y = 0;
      else { lo = min(lo, sp.x); hi = max(hi, sp.y); all_lo = max(all_lo, sp.x); all_hi = min(all_hi, sp.y); }
    }
    span[i] = sp;
    if (t == 0) notes.span[i * 8 + g] = sp;
  }
  lo = __reduce_min_sync(0xffffffffu, lo); hi = __reduce_max_sync(0xffffffffu, hi);
  all_lo = __reduce_max_sync(0xffffffffu, all_lo); all_hi = __reduce_min_sync(0xffffffffu, all_hi);
  const int blk0 = hi > 0 ? lo / kBlk : 0, n_blk = hi > 0 ? (hi + kBlk - 1) / kBlk - blk0 : 0;
  const int c0 = blk0 + share(n_blk, split), c1 = blk0 + share(n_blk, split + 1);
  const int n = c1 - c0 > warp ? (c1 - c0 - warp + kWarps - 1) / kWarps : 0;       // this warp's blocks: c0 + warp + i * kWarps

  // ---- first copies: block i's keys are copy 2 i, its values copy 2 i + 1; copy c goes to slot c % NS
  // an id out of range is fetched from block 0 and not used
  auto in_range = [&](int id) { return id >= 0 && id < a.n_blocks; };
  auto copy_src = [&](int id, int c) { return a.codes + ((size_t)(in_range(id) ? id : 0) * a.HK + kvh) * (2 * kPart) + (c & 1) * kPart; };
  auto scale_src = [&](int id) { return a.scales + (size_t)(in_range(id) ? id : 0) * a.HK + kvh; };
  const int id0 = c0 == guess ? guess_id : lane < min(n, kRun) ? table[c0 + warp + lane * kWarps] : -1;
#pragma unroll
  for (int c = 0; c < NS; ++c) {
    const int id = __shfl_sync(0xffffffffu, id0, c >> 1);
    if (c < 2 * n && lane == 0) fetch(slot0 + c * kPart, copy_src(id, c), bar0 + c * 8);
  }
  if (lane < min(n, kRun)) {
    notes.id[lane] = id0;
    async_copy(&notes.scale[lane], scale_src(id0));
  }

  // ---- queries: dims 16 t + 4 s + {0, 1} | {2, 3} of k16 step s; a row is brought to a largest value in [1, 2) so that f16 holds it
  uint32_t qf[NP][4][4];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    Row &w = row[i];
    float f[16];
    unpack16(qv[i], f);
    if (span[i].x == span[i].y) {
#pragma unroll
      for (int k = 0; k < 16; ++k) f[k] = 0.f;
    }
    float mx = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) mx = fmaxf(mx, fabsf(f[k]));
    mx = quad_max(mx);
    const int e = min(max((int)(__float_as_uint(mx) >> 23) - 127, -126), 126);
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
    w.unit = __uint_as_float((uint32_t)(127 + e) << 23);
#pragma unroll
    for (int s = 0; s < 4; ++s)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float x = f[4 * s + 2 * k] * down, y = f[4 * s + 2 * k + 1] * down;
        const uint32_t p = pack(x, y);
        qf[0][s][2 * k + i] = p;
        if (NP == 2) qf[NP - 1][s][2 * k + i] = pack_rest(x, y, p);
      }
  }

  async_copies_land();
  float o[8][4];
#pragma unroll
  for (int dn = 0; dn < 8; ++dn) o[dn][0] = o[dn][1] = o[dn][2] = o[dn][3] = 0.f;

  // ---- the blocks
  bool ok = true;
  float unit = 1.f;                                                                // of the sums of values: kDrop once there were large ones
  int st = 0; uint32_t phase = 0;                                                  // slot and phase of the copy that is waited for next
  auto arrived = [&] { return __all_sync(0xffffffffu, mbar_wait(bar0 + st * 8, phase)); };
  // The warp is through with copy c: its slot takes copy c + NS, which must not overtake the warp's reads.
  auto refill = [&](int i, int c) {
    __syncwarp();
    const int nc = c + NS, ni = nc >> 1;
    if (ni < n && lane == 0) {
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      fetch(slot0 + st * kPart, copy_src(notes.id[ni & (2 * kRun - 1)], nc), bar0 + st * 8);
    }
    if (++st == NS) { st = 0; phase ^= 1; }
  };
  for (int i = 0; i < n; ++i) {
    // the run of blocks after this one: ids while its first block is worked on, scales from its ninth
    if ((i & (kRun / 2 - 1)) == 0) {
      async_copies_land();
      const int at = (i & ~(kRun - 1)) + kRun + lane, to = at & (2 * kRun - 1);
      if (lane < kRun && at < n) {
        if ((i & (kRun / 2)) == 0) async_copy(&notes.id[to], table + c0 + warp + at * kWarps);
        else async_copy(&notes.scale[to], scale_src(notes.id[to]));
      }
    }
    const bool here = in_range(notes.id[i & (2 * kRun - 1)]);
    if (!here && lane == 0 && a.status) *a.status = PD_ERR_ARG;
    const float2 sc = notes.scale[i & (2 * kRun - 1)];
    const int p0 = (c0 + warp + i * kWarps) * kBlk;
    const bool edge = p0 < all_lo || p0 + kBlk > all_hi;                           // some row does not see all of it
    if (!(ok = arrived())) break;
    // ---- scores, four tiles of eight tokens at a time: products in a row are independent
    float s[8][4];
    const uint32_t kbase = slot0 + st * kPart;
#pragma unroll
    for (int jh = 0; jh < 8; jh += 4) {
      uint32_t u[4][4];
      float rest[4][4];                                                            // the second parts' sums: the tensor cores drop what lies below a sum's last place
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int token = 16 * (g >> 1) + 4 * ((jh + j) >> 1) + 2 * (j & 1) + (g & 1);
        const uint4 w = lds128(kbase + token * kDh + t * 16);
        u[j][0] = w.x; u[j][1] = w.y; u[j][2] = w.z; u[j][3] = w.w;
      }
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t b0, b1;
          widen(u[j][k], b0, b1);
#pragma unroll
          for (int p = 0; p < NP; ++p) {
            float (&c)[4] = p ? rest[j] : s[jh + j];
            if (k == 0) mma_f16_first(c, qf[p][k], b0, b1);
            else mma_f16(c, qf[p][k], b0, b1);
          }
        }
      if (NP == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int x = 0; x < 4; ++x) s[jh + j][x] += rest[j][x];
      }
    }
    refill(i, 2 * i);
    // ---- the block's softmax; without cap and bias the scale (positive) comes in with the exponent
    uint32_t pf[NP][4][4];
    float keep[2], take[2];                                                // factors of the values so far and of this block's
    float mref[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      Row &w = row[x];
      // Score in log2 units (or the cap's argument) per unit of q . code.  The units of queries and keys first: one may be near the end of the range where the other is near its other
      // end.  Neither a zero (times a masked score) nor an infinity (times a zero) may come of it
      const float per = w.unit * sc.x * a.factor, mul = MOD ? fminf(per, FLT_MAX) : fmaxf(per, FLT_MIN);
      if (MOD && a.cap) {
        if (NP == 1 && a.cap == 1) {
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) s[j][2 * x + e] = fmaf(-2.f * a.cap_log2e, rcp(1.f + ex2(s[j][2 * x + e] * mul)), a.cap_log2e);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) s[j][2 * x + e] = a.cap_log2e * tanhf(s[j][2 * x + e] * mul * a.inv_cap);
        }
      } else if (MOD) {
#pragma unroll
        for (int j = 0; j < 8; ++j) { s[j][2 * x] *= mul; s[j][2 * x + 1] *= mul; }
      }
      if (MOD && a.bias) {
        // sixteen neighbouring distances, the largest first: near (in the table), far (its last value) or across an end of the table
        const float *bias = a.bias + (size_t)(kvh * a.G + (tile * kRows + x * 8 + g) % a.G) * a.n_bias;
        const int most = notes.span[x * 8 + g].y - 1 - p0 - 16 * t;
        if (__all_sync(0xffffffffu, most - 15 >= a.n_bias - 1)) {
          const float far = bias[a.n_bias - 1] * kLog2e;
#pragma unroll
          for (int j = 0; j < 8; ++j) { s[j][2 * x] += far; s[j][2 * x + 1] += far; }
        } else if (__all_sync(0xffffffffu, most >= 15 && most < a.n_bias)) {
          const float *near = bias + most;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) s[j][2 * x + e] = fmaf(near[-(4 * (j >> 1) + 2 * (j & 1) + e)], kLog2e, s[j][2 * x + e]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              s[j][2 * x + e] = fmaf(bias[min(max(most - (4 * (j >> 1) + 2 * (j & 1) + e), 0), a.n_bias - 1)], kLog2e, s[j][2 * x + e]);
        }
      }
      if (edge) {
        const int2 sp = notes.span[x * 8 + g];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int pos = p0 + 16 * t + 4 * (j >> 1) + 2 * (j & 1) + e;
            if (pos < sp.x || pos >= sp.y) s[j][2 * x + e] = -INFINITY;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) mx = fmaxf(mx, fmaxf(s[j][2 * x], s[j][2 * x + 1]));
      mx = quad_max(mx);
      if (!here) mx = -INFINITY;
      if (MOD && a.bias && mx < kGone) mx = -INFINITY;                             // where others have more, such positions weigh nothing anyway
      // Weights are 2^(score - top + lift).  Without cap and bias the scale and both terms come in with one fused step; where a score's last place is a weight's step and more
      // that would round past f16's end, and the difference is taken first, exact where it matters.
      float f = MOD ? 1.f : mul;
      mx *= f;
      const float top = mx == -INFINITY ? 0.f : mx;
      float ref = kLift - top;
      constexpr bool DIFF = MOD || NP == 2;
      if (!DIFF && __any_sync(0xffffffffu, mul >= kCoarse / kMostSum)) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) s[j][2 * x + e] = __fsub_rn(__fmul_rn(s[j][2 * x + e], f), top);
        f = 1.f; ref = kLift;
      }
      auto exponent = [&](float v) { return MOD ? (v - top) + kLift : DIFF ? __fsub_rn(__fmul_rn(v, f), top) + kLift : fmaf(v, f, ref); };
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float w0 = ex2(exponent(s[j][2 * x])), w1 = ex2(exponent(s[j][2 * x + 1]));
        const uint32_t p = pack(w0, w1);
        pf[0][j >> 1][2 * (j & 1) + x] = p;
        if (NP == 2) pf[NP - 1][j >> 1][2 * (j & 1) + x] = pack_rest(w0, w1, p);
      }
      const float m_new = fmaxf(w.m, mx);
      mref[x] = m_new == -INFINITY ? 0.f : m_new;
      keep[x] = ex2(w.m - mref[x]);
      take[x] = ex2(mx - mref[x]);
      w.m = m_new;
    }
    // ---- values, four tiles of eight dims at a time
    if (!(ok = arrived())) break;
    const uint32_t vbase = slot0 + st * kPart;
    const bool large = sc.y >= kLarge && unit == 1.f;                              // lifted sums of such values could overflow where the values' own do not
    if (large || __any_sync(0xffffffffu, keep[0] != 1.f || keep[1] != 1.f)) {      // some row's running maximum moved
      const float f = large ? kDrop : 1.f;
#pragma unroll
      for (int dn = 0; dn < 8; ++dn)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[dn][x] *= keep[x >> 1] * f;
      unit *= f;
    }
    const float vscale = sc.y * unit;
    uint32_t nan_seen = 0;                                                         // values that are no numbers, at positions that some row sees
    if (here) {
#pragma unroll
      for (int dh = 0; dh < 8; dh += 4) {
        uint32_t u[4][4];
        float tv[4][4], rest[4][4];
#pragma unroll
        for (int dn = 0; dn < 4; ++dn) {
          const uint4 w = lds128(vbase + ((dh + dn) * 8 + g) * kBlk + t * 16);
          u[dn][0] = w.x; u[dn][1] = w.y; u[dn][2] = w.z; u[dn][3] = w.w;
        }
        if (edge) {                                                                // 0 must not meet what is no number
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int p = p0 + 16 * t + 4 * k;
            const uint32_t seen = below(hi - p) & ~below(lo - p);
#pragma unroll
            for (int dn = 0; dn < 4; ++dn) {
              const uint32_t nb = nan_bytes(u[dn][k]);
              nan_seen |= nb & seen;
              u[dn][k] &= ~(nb | (nb - (nb >> 7)));
            }
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
          for (int dn = 0; dn < 4; ++dn) {
            uint32_t b0, b1;
            widen(u[dn][k], b0, b1);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
              float (&c)[4] = p ? rest[dn] : tv[dn];
              if (k == 0) mma_f16_first(c, pf[p][k], b0, b1);
              else mma_f16(c, pf[p][k], b0, b1);
            }
          }
        if (NP == 2) {
#pragma unroll
          for (int dn = 0; dn < 4; ++dn)
#pragma unroll
            for (int x = 0; x < 4; ++x) tv[dn][x] += rest[dn][x];
        }
#pragma unroll
        for (int dn = 0; dn < 4; ++dn)
#pragma unroll
          for (int x = 0; x < 4; ++x) o[dh + dn][x] = fmaf(tv[dn][x], take[x >> 1] * vscale, o[dh + dn][x]);
      }
      if (edge && __any_sync(0xffffffffu, nan_seen != 0)) {
        // rows that see such a value get it after all: a product of who sees which position with where they stand
        uint32_t sees[4][4];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int2 sp = notes.span[x * 8 + g];
#pragma unroll
          for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int p = p0 + 16 * t + 4 * k + 2 * y;
              sees[k][2 * y + x] = (p >= sp.x && p < sp.y ? 0x3c00u : 0u) | (p + 1 >= sp.x && p + 1 < sp.y ? 0x3c000000u : 0u);
            }
        }
#pragma unroll
        for (int dn = 0; dn < 8; ++dn) {
          const uint4 w = lds128(vbase + (dn * 8 + g) * kBlk + t * 16);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
          float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t nb = nan_bytes(u[k]);
            mma_f16(c, sees[k], (nb & 0x80u ? 0x3c00u : 0u) | (nb & 0x8000u ? 0x3c000000u : 0u),
                    (nb & 0x800000u ? 0x3c00u : 0u) | (nb & 0x80000000u ? 0x3c000000u : 0u));
          }
#pragma unroll
          for (int x = 0; x < 4; ++x)
            if (c[x] > 0.f) o[dn][x] = __int_as_float(0x7fffffff);
        }
      }
    }
    // the weights' sum is a product with ones: every lane of a row gets it, and numerator and denominator see the same roundings
    float sum[4];
    mma_f16_first(sum, pf[0][0], 0x3c003c00u, 0x3c003c00u);
#pragma unroll
    for (int k = 1; k < 4 * NP; ++k) mma_f16(sum, pf[k >> 2][k & 3], 0x3c003c00u, 0x3c003c00u);
#pragma unroll
    for (int x = 0; x < 2; ++x)
      if (here) row[x].l = row[x].l * keep[x] + sum[2 * x] * take[x];
    refill(i, 2 * i + 1);
  }
  if (!ok) {                                                                       // the copies in flight must land before the CTA ends
    if (lane == 0 && a.status) *a.status = PD_ERR_TIMEOUT;
    for (int s = 0; s < NS; ++s) { mbar_wait(bar0 + st * 8, phase); if (++st == NS) { st = 0; phase ^= 1; } }
  }

  // ---- join the warps, then the cluster's CTAs, both in their order: a thread takes columns 4 k .. 4 k + 3 and 32 + 4 k .. of a row
  __syncthreads();                                                                 // the rings are free
  const float drop = unit == 1.f ? kDrop : 1.f;                                    // the lift leaves here at the latest
  float *rec = reinterpret_cast<float *>(ring), *ml = rec + kWarps * kRows * kDh;   // [warp][row][64], [warp][row][2]
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int m = warp * kRows + x * 8 + g;
    const int2 sp = notes.span[x * 8 + g];
    const bool any = sp.x < sp.y;                          // rows that see nothing went along unmasked
    if (t == 0) store2(ml + 2 * m, any ? row[x].m : -INFINITY, any ? row[x].l * kDrop : 0.f);
#pragma unroll
    for (int dn = 0; dn < 8; ++dn)
      store2(rec + m * kDh + ((dn * 8 + 2 * t) ^ ((g & 3) << 3)), any ? o[dn][2 * x] * drop : 0.f, any ? o[dn][2 * x + 1] * drop : 0.f);
  }
  __syncthreads();
  const int cluster = a.cluster, rank = split % cluster, own = kRows / cluster;     // rank k sums rows k * own .. of the cluster's CTAs
  float *inbox = reinterpret_cast<float *>(ring + RING);                           // [CTA][row of this rank][kRec]
  // Sum of n partial results of a row; `ml_of` and `o_of` give the addresses of one's (maximum, sum) and first columns.
  auto join = [&](int n, auto ml_of, auto o_of, float2 &h, float4 &x, float4 &y) {
    float mx = -INFINITY;
    for (int k = 0; k < n; ++k) mx = fmaxf(mx, ml_of(k)->x);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float l = 0.f;
    x = y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int k = 0; k < n; ++k) {
      const float2 s = *ml_of(k);
      const float f = ex2(s.x - ref);
      const float4 u = *reinterpret_cast<const float4 *>(o_of(k, 0)), v = *reinterpret_cast<const float4 *>(o_of(k, 32));
      l += s.y * f;
      x.x += u.x * f; x.y += u.y * f; x.z += u.z * f; x.w += u.w * f;
      y.x += v.x * f; y.y += v.y * f; y.z += v.z * f; y.w += v.w * f;
    }
    h = make_float2(mx, l);
  };
  auto finish = [&](int m, int c, float2 h, float4 x, float4 y) {
    if (a.outer > 1) {
      float *p = a.part + ((((size_t)b * gridDim.y + blockIdx.y) * a.outer + split / cluster) * kRows + m) * kRec;
      store4(p + c, x); store4(p + c + 32, y);
      if (c == 0) store2(p + kDh, h.x, h.y);
      return;
    }
    const int gm = tile * kRows + m, r = gm / a.G, head = kvh * a.G + gm % a.G;
    if (r >= a.R) return;
    const float inv = h.y == 0.f ? 0.f : 1.f / h.y;                                // nothing seen: zero
    T *p = static_cast<T *>(a.out) + (((size_t)b * a.R + r) * a.H + head) * kDh + c;
    store4(p, make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv));
    store4(p + 32, make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv));
  };
  if (cluster > 1) cluster_wait();                                                 // all CTAs of the cluster have begun
#pragma unroll
  for (int i = threadIdx.x; i < kRows * 8; i += kThreads) {
    const int m = i >> 3, c = (i & 7) * 4;
    float2 h;
    float4 x, y;
    join(kWarps, [&](int k) { return reinterpret_cast<const float2 *>(ml + 2 * (k * kRows + m)); },
         [&](int k, int at) { return rec + (k * kRows + m) * kDh + ((c + at) ^ ((m & 3) << 3)); }, h, x, y);
    if (cluster == 1) { finish(m, c, h, x, y); continue; }
    const uint32_t to = peer_addr(smem_u32(inbox + ((size_t)rank * own + m % own) * kRec), m / own);
    peer_st4(to + c * 4, x); peer_st4(to + (c + 32) * 4, y);
    if (c == 0) peer_st4(to + kDh * 4, make_float4(h.x, h.y, 0.f, 0.f));
  }
  if (cluster == 1) return;
  cluster_arrive();
  cluster_wait();
  for (int i = threadIdx.x; i < own * 8; i += kThreads) {
    const int m = i >> 3, c = (i & 7) * 4;
    float2 h;
    float4 x, y;
    join(cluster, [&](int k) { return reinterpret_cast<const float2 *>(inbox + (k * own + m) * kRec + kDh); },
         [&](int k, int at) { return inbox + (k * own + m) * kRec + c + at; }, h, x, y);
    finish(rank * own + m, c, h, x, y);
  }
}

// Joins the splits of a row in their order: one warp per (sequence, row, head), two columns per lane.
template <typename T>
__global__ void __launch_bounds__(128) cache_attn_merge_kernel(CacheAttnArgs a, long long n_out) {
  op_begin();
  const long long i = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
  const int lane = threadIdx.x & 31;
  if (i >= n_out) return;
  const int h = (int)(i % a.H), r = (int)(i / a.H % a.R), b = (int)(i / a.H / a.R);
  const int kvh = h / a.G, m = r * a.G + h % a.G, tile = m / kRows;
  const float *p = a.part + (((size_t)b * a.HK + kvh) * a.tiles + tile) * a.outer * kRows * kRec + (size_t)(m % kRows) * kRec;
  const size_t step = (size_t)kRows * kRec;
  float mx = -INFINITY, l = 0.f, x = 0.f, y = 0.f;
  for (int s0 = 0; s0 < a.outer; s0 += 8) {                                        // eight splits' loads under way together
    float2 ml[8], v[8];
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const bool in = s0 + s < a.outer;
      ml[s] = in ? *reinterpret_cast<const float2 *>(p + (s0 + s) * step + kDh) : make_float2(-INFINITY, 0.f);
      v[s] = in ? *reinterpret_cast<const float2 *>(p + (s0 + s) * step + 2 * lane) : make_float2(0.f, 0.f);
    }
    float top = mx;
#pragma unroll
    for (int s = 0; s < 8; ++s) top = fmaxf(top, ml[s].x);
    const float ref = top == -INFINITY ? 0.f : top, f0 = ex2(mx - ref);
    l *= f0; x *= f0; y *= f0; mx = top;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const float f = ex2(ml[s].x - ref);
      l += ml[s].y * f; x += v[s].x * f; y += v[s].y * f;
    }
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store2(static_cast<T *>(a.out) + i * kDh + 2 * lane, x * inv, y * inv);
}

// Shape of a launch: row tiles, CTAs of a cluster, clusters per segment.  A function of sizes the scratch is asked for with.
struct Plan { int tiles, cluster, outer; };

Plan plan_of(int dtype, int batch, int rows, int heads, int kv_heads, int max_len) {
  Plan p;
  const int m = rows * (heads / kv_heads);
  // 32 rows per tile would read the cache half as often, at half the warps: 32 x 16 heads x 2048 tokens, 30 rows 58 us against 45, 1 x 12 x 777, 20 rows 7.8 against 5.8
  p.tiles = (m + kRows - 1) / kRows;
  const long long segs = (long long)batch * kv_heads * p.tiles, blocks = ((long long)max_len + kBlk - 1) / kBlk;
  // places for CTAs in clusters: a GPC's SMs are not a multiple of a cluster's CTAs (512 of 592 places taken 35 us, 576 in two rounds 47 us, at 2 x 4
  // key heads x 131072 tokens)
  const long long room = std::max(1ll, kClusterSms * ctas_per_sm(dtype == PD_DTYPE_FP32) / segs);
  p.cluster = 1;
  while (p.cluster < kMaxCluster && p.cluster * 2 <= room && p.cluster * kWarps < blocks) p.cluster *= 2;
  p.outer = p.cluster == kMaxCluster ? (int)std::max(1ll, std::min(room / kMaxCluster, blocks / (kMaxCluster * kWarps * kOuterBlocks))) : 1;
  return p;
}

bool cache_attn_sizes_ok(int dtype, int batch, int rows, int heads, int kv_heads, int max_len) {
  if (dtype != PD_DTYPE_FP32 && dtype != PD_DTYPE_BF16) return false;
  if (batch < 1 || batch > 65535 || rows < 1 || rows > kMaxRows || kv_heads < 1 || heads < kv_heads || heads % kv_heads || heads > 1024) return false;
  return max_len >= 0 && max_len <= INT_MAX - kBlk;
}

size_t scratch_bytes_of(const Plan &p, int batch, int kv_heads) {
  return p.outer > 1 ? (size_t)batch * kv_heads * p.tiles * p.outer * kRows * kRec * sizeof(float) : 0;
}

template <typename T>
cudaError_t launch_cache_attn(const CacheAttnArgs &a, int batch, bool mod, cudaStream_t s) {
  constexpr int smem = smem_bytes(sizeof(T) == 4);
  auto kernel = mod ? cache_attn_kernel<T, true> : cache_attn_kernel<T, false>;
  // once per kernel and device: setting it costs as much host time as a third of the launch
  static std::atomic<uint64_t> ready[2];
  int dev = 0;
  cudaError_t st = cudaGetDevice(&dev);
  if (st != cudaSuccess) return st;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready[mod].load(std::memory_order_relaxed) & bit)) {
    if ((st = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem)) != cudaSuccess) return st;
    ready[mod].fetch_or(bit, std::memory_order_relaxed);
  }
  st = op_launch(kernel, dim3(a.cluster * a.outer, a.HK * a.tiles, batch), kThreads, smem, a.cluster, s, a);
  if (st != cudaSuccess || a.outer == 1) return st;
  const long long n_out = (long long)batch * a.R * a.H;
  return op_launch(cache_attn_merge_kernel<T>, dim3((unsigned)((n_out + 3) / 4)), 128, 0, 1, s, a, n_out);
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
  if (!aligned_to(16, q, codes, out, scratch) || !aligned_to(8, scales, spans) || !aligned_to(4, table, n_rows, lens, bias, status)) return PD_ERR_ARG;
  const Plan p = plan_of(dtype, batch, rows_per_seq, n_heads, n_kv_heads, max_len);
  const size_t need = scratch_bytes_of(p, batch, n_kv_heads);
  if (need && !scratch) return PD_ERR_ARG;
  if (scratch_bytes < need) return PD_ERR_WORKSPACE;
  CacheAttnArgs a;
  a.R = rows_per_seq; a.H = n_heads; a.HK = n_kv_heads; a.G = n_heads / n_kv_heads; a.n_blocks = n_blocks; a.max_blocks = max_blocks; a.max_len = max_len;
  a.tiles = p.tiles; a.cluster = p.cluster; a.outer = p.outer; a.n_bias = bias ? n_bias : 0;
  a.cap = softcap > 0.f ? (dtype == PD_DTYPE_BF16 && softcap <= kQuotientCap ? 1 : 2) : 0;
  a.factor = a.cap == 1 ? std::min(2.f * kLog2e * attn_scale / softcap, FLT_MAX) : attn_scale * kLog2e;
  a.cap_log2e = softcap * kLog2e;
  a.inv_cap = a.cap ? std::min(1.f / a.cap_log2e, FLT_MAX) : 0.f;
  a.q = q; a.q_row = q_stride; a.codes = static_cast<const uint8_t *>(codes); a.scales = reinterpret_cast<const float2 *>(scales);
  a.table = table; a.n_rows = n_rows; a.lens = lens; a.spans = reinterpret_cast<const int2 *>(spans); a.bias = bias;
  a.out = out; a.part = static_cast<float *>(scratch); a.status = status;
  const bool mod = softcap > 0.f || bias;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(cuda_stream);
  cudaError_t st;
  if (dtype == PD_DTYPE_FP32) st = launch_cache_attn<float>(a, batch, mod, s);
  else st = launch_cache_attn<__nv_bfloat16>(a, batch, mod, s);
  return op_status(st);
}

}  // extern "C"
