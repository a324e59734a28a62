// k_c8_many.cu -- many rows of one document over an 8-bit cache (c8.cuh), on the tcgen05 tensor cores:
// attention straight from the codes, for more rows a layer's blocks widened to pages of halves for the
// kernels that read such pages, and the weights of the entries by a second product.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "c8.cuh"
#include "tc_ptx.cuh"

namespace kvr {
namespace {
using namespace ptx;

// The largest powers of a head's pages: a page's halves are its codes times its power over that,
// lifted by 2^7 (448 * 2^7 is a half).  Codes are exact down to powers 2^-22 of the largest; below, a
// value is off by at most 2^-32 of it.
constexpr float LIFT = 128.f, LIFT_INV = 1.f / 128.f;

// That factor of a page's codes as halves.  From 2^-24 on (powers 2^-31 of the largest) it is one, and a
// product rounds once.  Below it is `low`: codes are first taken 2^-15 down, which is exact, then
// multiplied by the factor 2^15 up, which rounds once, too (where that is none either, below 2^-39,
// all products round to zero).
struct HalfFactor {
  __half2 down, f;
  bool low;
  __device__ __forceinline__ explicit HalfFactor(float x) : low(x < 5.9604644775390625e-8f) {
    down = __float2half2_rn(low ? 1.f / 32768.f : 1.f);
    f = __float2half2_rn(low ? x * 32768.f : x);
  }
};
// LOW: some factor of a warp's codes may be low.
template <bool LOW>
__device__ __forceinline__ uint32_t times(uint32_t codes, const HalfFactor &h) {
  __half2 x = *(const __half2 *)&codes;
  if (LOW) x = __hmul2(x, h.down);
  x = __hmul2(x, h.f);
  return *(const uint32_t *)&x;
}

// The largest powers of the first n pages of a head, by all NT threads of a CTA; s: shared, 0 before.
template <int N>
__device__ __forceinline__ float2 largest_powers(const float2 *powers, int n, uint32_t *s) {
  float2 most = make_float2(0.f, 0.f);
  for (int i = threadIdx.x; i < n; i += N) {
    const float2 p = powers[i];
    most.x = fmaxf(most.x, p.x);
    most.y = fmaxf(most.y, p.y);
  }
  const uint32_t x = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most.x)),
                 y = __reduce_max_sync(0xFFFFFFFFu, __float_as_uint(most.y));
  if (threadIdx.x % 32 == 0) {
    atomicMax(&s[0], x);
    atomicMax(&s[1], y);
  }
  __syncthreads();
  return make_float2(__uint_as_float(s[0]), __uint_as_float(s[1]));
}

// A CTA for each page and KV head, K and V.  page_power [G]: what the halves are to be multiplied
// by.  Bound by L2: a layer of 12345 positions of 4 KV heads reads 12.6 MB and writes 25.3, in
// whole sectors 7.5 us (by stores of 16 bytes 10.6).
template <int DH>
__global__ void __launch_bounds__(256)
    k_c8_unpack(const C8View v, int layer, int n_pages, __half *pages, float2 *page_power) {
  constexpr int PIECES = DH / 16;
  __shared__ uint32_t s_max[2];
  const int tid = threadIdx.x, g = blockIdx.x, page = blockIdx.y;
  if (tid < 2) s_max[tid] = 0;
  pdl_trigger();
  pdl_wait();
  const float2 *powers = v.power + v.index(layer, g, 0);
  __syncthreads();
  const float2 most = largest_powers<256>(powers, n_pages, s_max);
  if (page == 0 && tid == 0) page_power[g] = make_float2(most.x * LIFT_INV, most.y * LIFT_INV);
  const float2 own = powers[page];
  const uint8_t *block = v.blocks + v.index(layer, g, page) * c8_block_bytes(DH);
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const float f = (kv ? own.y * c8_inverse(most.y) : own.x * c8_inverse(most.x)) * LIFT;
    const uint8_t *src = block + kv * c8_half_bytes(DH);
    __half *dst = pages + (((size_t)page * 2 + kv) * v.G + g) * KVR_PAGE * DH;
    for (int i = tid; i < KVR_PAGE * PIECES; i += 256) {
      const int r = i / PIECES, c = i % PIECES;
      const uint4 u = *(const uint4 *)(src + r * DH + 16 * c8_piece<DH>(r, c));
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      uint32_t o[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float4 x = c8_values(w[k], f);
        const __half2 a = __floats2half2_rn(x.x, x.y), b = __floats2half2_rn(x.z, x.w);
        o[2 * k] = *(const uint32_t *)&a;
        o[2 * k + 1] = *(const uint32_t *)&b;
      }
      // a whole sector at once
      asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst + r * DH + 16 * c),
                   "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]),
                   "r"(o[7])
                   : "memory");
    }
  }
}

// Two blocks' K or V (128 rows) into a shared-memory tile of halves as the products take it: rows of
// 128 bytes in column blocks of 64 entries, 16-byte pieces XORed by the row.  By N threads, of
// which each has EACH pieces of 16 entries, the first half of them of the first block.  Eight lanes
// take four pieces of each of two rows, which lie in all banks on both sides; a thread's rows are
// whole eights apart, so that its offsets differ by constants.
template <int DH, int N>
struct Widen {
  static constexpr int PIECES = DH / 16, STEP = N / PIECES, EACH = 2 * KVR_PAGE / STEP;
  uint32_t from, to0, to1;  // offsets of its first piece in the codes and of its halves in the tile
  __device__ __forceinline__ explicit Widen(uint32_t t) {
    const uint32_t c = DH == 128 ? (t & 3) | (t >> 1 & 4) : t & 3,
                   r = DH == 128 ? (t >> 2 & 1) | (t >> 4 << 1) : t >> 2;
    from = r * DH + 16 * c8_piece<DH>(r, c);
    const uint32_t row = (c >> 2) * (2 * KVR_PAGE * 128) + r * 128, at = (c & 3) * 2;
    to0 = row + ((at ^ (r & 7)) << 4);
    to1 = row + (((at + 1) ^ (r & 7)) << 4);
  }
  // piece j: of the block at a, or of b
  __device__ __forceinline__ uint4 load(const uint8_t *a, const uint8_t *b, int j) const {
    return *(const uint4 *)((j < EACH / 2 ? a : b) + from + j % (EACH / 2) * (STEP * DH));
  }
  template <bool LOW>
  __device__ __forceinline__ void store(uint32_t tile, uint4 u, const HalfFactor &f, int j) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t o[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      c8_halves(w[k], o[2 * k], o[2 * k + 1]);
      o[2 * k] = times<LOW>(o[2 * k], f);
      o[2 * k + 1] = times<LOW>(o[2 * k + 1], f);
    }
    *(uint4 *)__cvta_shared_to_generic(tile + to0 + j * (STEP * 128)) =
        make_uint4(o[0], o[1], o[2], o[3]);
    *(uint4 *)__cvta_shared_to_generic(tile + to1 + j * (STEP * 128)) =
        make_uint4(o[4], o[5], o[6], o[7]);
  }
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// (x0, x1) * s + c and a + b on pairs of fp32 (one instruction each)
__device__ __forceinline__ void fma2(float &y0, float &y1, uint32_t x0, uint32_t x1, float s,
                                     float c) {
  asm("{\n\t.reg .b64 x, s, c, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 s, {%4, %4};\n\t"
      "mov.b64 c, {%5, %5};\n\tfma.rn.f32x2 y, x, s, c;\n\tmov.b64 {%0, %1}, y;\n\t}"
      : "=f"(y0), "=f"(y1)
      : "r"(x0), "r"(x1), "f"(s), "f"(c));
}
__device__ __forceinline__ void fma2(float &y0, float &y1, uint32_t x0, uint32_t x1, float s0,
                                     float s1, float c0, float c1) {
  asm("{\n\t.reg .b64 x, s, c, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 s, {%4, %5};\n\t"
      "mov.b64 c, {%6, %7};\n\tfma.rn.f32x2 y, x, s, c;\n\tmov.b64 {%0, %1}, y;\n\t}"
      : "=f"(y0), "=f"(y1)
      : "r"(x0), "r"(x1), "f"(s0), "f"(s1), "f"(c0), "f"(c1));
}
// a += b * c
__device__ __forceinline__ void fma2_add(float &a0, float &a1, float b0, float b1, float c0,
                                         float c1) {
  asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\t"
      "mov.b64 c, {%4, %5};\n\tfma.rn.f32x2 a, b, c, a;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "+f"(a0), "+f"(a1)
      : "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}
__device__ __forceinline__ void add2(float &a0, float &a1, float b0, float b1) {
  asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%0, %1};\n\tmov.b64 b, {%2, %3};\n\t"
      "add.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
      : "+f"(a0), "+f"(a1)
      : "f"(b0), "f"(b1));
}

// ---- attention straight from the codes ----

constexpr int QV = 128;              // query vectors of a tile
constexpr int CH = 2 * KVR_PAGE;     // keys of a step
constexpr int KP = 2;                // softmax: threads a vector, each with a part of a step's keys
constexpr int SM_WARPS = 4 * KP;
constexpr int CV_WARPS = 8;          // widening
constexpr int NTR = 32 * (2 + SM_WARPS + CV_WARPS);
constexpr int RAW = 4;               // K's or V's codes of a step, in flight or being widened
constexpr int NS = 3;                // scores of steps in TMEM
constexpr uint32_t TMEM_ROWS = 512;  // NS scores (P over parts of them), O
constexpr float RESCALE_LOG2 = 8.f;
constexpr int WS_MAXQ = 192;         // query slots of the split workspace

__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc,
                                       uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st8_nowait(uint32_t taddr, const uint32_t *r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
      : "memory");
}

// 32 consecutive TMEM columns of 16 lanes, without the wait: r[4 i + ..] are columns 8 i + 2 (lane % 4)
// and the next of TMEM lane lane / 4, then those of the one eight further.
__device__ __forceinline__ void tmem_ld_16x256_nowait(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
      "%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]),
        "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
// 8 consecutive 32-bit TMEM columns, without the wait.
__device__ __forceinline__ void tmem_ld8_nowait(uint32_t taddr, uint32_t *r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7])
      : "r"(taddr));
}

// A CTA owns a tile of up to 128 query vectors of a KV head and a run of pages, two at a time:
//   widening    four warps each turn K's and V's codes, which bulk copies bring, into halves over the
//               head's largest power, into two tiles each;
//   S = Q K^T   M 128 vectors x N 128 keys, S in TMEM, three times: two steps' products run
//               ahead of the softmax;
//   softmax     two threads a vector, as in the kernel of pages (integer reference, raised by powers of two
//               when a score exceeds it by 8), P in halves over S's columns;
//   O += P V    P from TMEM.
// What it saves beside the way by pages of halves are those pages: written once and read by every
// tile, three times the codes' bytes and a launch.  What bounds it is shared memory, 224 KB a step
// (codes in and out, halves in, the products' operands), beside the chain from scores to weights: a
// step takes 1.05 us (512 rows of 32 heads over 5000 entries, 128 CTAs of 40 steps, 46.6; 64 over
// 16384, 9 parts of 15 steps and their sum, 26.6; with a step's weights under the old reference taken
// beside its maximum, and again where that is not enough, 48.8 and 27.8).  Parts that a cluster adds
// in its shared memory save the other launch (128 rows over 5000, clusters of 4: 20.7 for 23.6), but
// 16 clusters of 8 do not run at once, and smaller ones have longer parts (64 rows over 16384: 32.3):
// left out.  For weights of the entries it leaves its queries as halves, with what makes weights of
// their products (by a kernel of their own 45.2 us for 64 rows over 16384, 44.3 so).
template <int DH>
__global__ void __launch_bounds__(NTR, 1) k_c8_rows(const __grid_constant__ C8RowsArgs p) {
  constexpr int HALVES = DH / 64;
  constexpr uint32_t HB = CH * 128, TBYTES = HB * HALVES;  // a column block, a tile
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t q_full, raw_full[RAW], raw_empty[RAW], k_full[2], k_empty[2],
      v_full[2], v_empty[2], s_full[NS], p_full[NS], o_done[NS], drain_bar;
  __shared__ uint32_t tmem_slot, s_max[2];
  __shared__ int abort_f;
  __shared__ float sx[KP - 1][QV];  // (what is left beside the tiles)
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int split = blockIdx.x, g = blockIdx.y;
  const int4 bd = p.blocks[blockIdx.z];
  const int n_pages = bd.z / KVR_PAGE + 1, cps = (n_pages + p.n_splits - 1) / p.n_splits;
  const int c0 = split * cps, c1 = min(n_pages, c0 + cps);
  if (c0 >= c1) {  // the combine skips it
    pdl_trigger();
    return;
  }
  const int n = (c1 - c0 + 1) / 2;
  const uint32_t base = (su32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sQ = base, sK = base + TBYTES, sV = sK + 2 * TBYTES;
  uint8_t *raw = (uint8_t *)__cvta_shared_to_generic(sV + 2 * TBYTES);  // [RAW][2 blocks' half]
  volatile int *abort_v = &abort_f;
  if (tid == 0) {
    mbar_init(&q_full, SM_WARPS);
    for (int i = 0; i < NS; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&p_full[i], SM_WARPS);
      mbar_init(&o_done[i], 1);
    }
    for (int i = 0; i < RAW; ++i) {
      mbar_init(&raw_full[i], 1);
      mbar_init(&raw_empty[i], CV_WARPS / 2);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&k_full[i], CV_WARPS / 2);
      mbar_init(&k_empty[i], 1);
      mbar_init(&v_full[i], CV_WARPS / 2);
      mbar_init(&v_empty[i], 1);
    }
    mbar_init(&drain_bar, 1);
    abort_f = 0;
    s_max[0] = s_max[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // codes of step i, K's or V's (a second page past the last one is the last again: its keys are
  // masked)
  constexpr uint32_t BB = c8_block_bytes(DH);
  auto second = [&](int i) { return min(c0 + 2 * i + 1, c1 - 1); };
  auto fetch = [&](int i, int kv) {
    const int st = 2 * (i & 1) + kv;
    const uint8_t *from =
        p.cache.blocks + p.cache.index(p.layer, g, 0) * BB + kv * c8_half_bytes(DH);
    mbar_expect_tx(&raw_full[st], BB);
    bulk_load(raw + st * BB, from + (size_t)(c0 + 2 * i) * BB, BB / 2, &raw_full[st]);
    bulk_load(raw + st * BB + BB / 2, from + (size_t)second(i) * BB, BB / 2, &raw_full[st]);
  };
  pdl_wait();
  if (tid == 0)  // the first two steps' are on their way while all else is made ready
    for (int i = 0; i < min(n, 2); ++i) {
      fetch(i, 0);
      fetch(i, 1);
    }
  // and a softmax thread's part of a row of Q
  const int part = (warp - 1) >> 2, quarter = warp & 3;
  const int vi = quarter * 32 + lane;
  const bool real = vi < bd.y * p.grp;
  const int row = bd.x + (real ? vi / p.grp : 0), hh = g * p.grp + (real ? vi % p.grp : 0);
  constexpr int QP = DH / 8 / KP;  // 16-byte pieces of it
  uint4 qx[QP];
  if (warp >= 1 && warp <= SM_WARPS) {
    const uint4 *src = (const uint4 *)(p.q + (size_t)row * p.ldq + (size_t)hh * DH) + part * QP;
#pragma unroll
    for (int k = 0; k < QP; ++k) qx[k] = real ? src[k] : make_uint4(0u, 0u, 0u, 0u);
  }
  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     su32(&tmem_slot)),
                 "r"(TMEM_ROWS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  // dependents may launch once this CTA holds its tensor memory: one of theirs that waits for
  // this grid with columns of its own cannot keep it from them
  pdl_trigger();
  const float2 *powers = p.cache.power + p.cache.index(p.layer, g, 0);
  const float2 most = largest_powers<NTR>(powers, p.n_pages, s_max);
  if (split == 0 && blockIdx.z == 0 && tid == 0) {
    p.page_power[g] = make_float2(most.x * LIFT_INV, most.y * LIFT_INV);
    if (p.vectors) p.key_power[g] = most.x * LIFT_INV;
  }

  if (warp == 0) {
    // ------------------------------------------------------------ MMA
    const uint32_t id_s = idesc_16(true, QV, CH), id_o = idesc_16(true, QV, DH, 1);
    const uint64_t dq = sw128_desc(sQ), dk0 = sw128_desc(sK), dv0 = sw128_desc_mn(sV, HB, 1024);
    const uint32_t tO = tmem + NS * CH;
    auto wait = [&](uint64_t *bar, int parity, int code) -> bool {
      return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_v, p.dev_flag, code));
    };
    bool ok = wait(&q_full, 0, 80);
    tc_fence_after();
    // a step's scores are asked for ahead of the product of the step two before it, so that the
    // softmax finds them when it is done with the last
#pragma unroll 1
    for (int i = 0; i < n + 2 && ok; ++i) {
      if (i < n) {
        ok = wait(&k_full[i & 1], (i >> 1) & 1, 81);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t dk = dk0 + (uint64_t)(((i & 1) * TBYTES) >> 4);
          const uint32_t tS = tmem + i % NS * CH;
#pragma unroll
          for (int kk = 0; kk < DH / 16; ++kk) {
            const uint64_t o = (uint64_t)(((kk >> 2) * HB + (kk & 3) * 32) >> 4);
            mma_bf16(tS, dq + o, dk + o, id_s, kk > 0 ? 1u : 0u);
          }
          mma_commit(&s_full[i % NS]);
          mma_commit(&k_empty[i & 1]);
        }
        __syncwarp();
      }
      const int j = i - 2;
      if (j >= 0) {
        ok = wait(&v_full[j & 1], (j >> 1) & 1, 83) && wait(&p_full[j % NS], (j / NS) & 1, 82);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
          const uint64_t dv = dv0 + (uint64_t)(((j & 1) * TBYTES) >> 4);
          const uint32_t tP = tmem + j % NS * CH;
#pragma unroll
          for (int kk = 0; kk < CH / 16; ++kk)
            mma_ts(tO, tP + (kk / (8 / KP)) * (CH / KP) + kk % (8 / KP) * 8,
                   dv + (uint64_t)((kk * 2048) >> 4), id_o, kk > 0 || j > 0 ? 1u : 0u);
          mma_commit(&v_empty[j & 1]);
          mma_commit(&o_done[j % NS]);
        }
        __syncwarp();
      }
    }
    // every product issued here completes before TMEM is freed
    if (elect_one()) mma_commit(&drain_bar);
    __syncwarp();
    mbar_wait(&drain_bar, 0, abort_v, p.dev_flag, 0, false);
  } else if (warp > SM_WARPS) {
    if (warp > SM_WARPS + CV_WARPS) {
      // ---------------------------------------------------------- codes
      if (lane < 2) {  // K's lane and V's, each with half of the ring
        const int kv = lane;
        int i = min(n, 2);
        for (; i < n; ++i) {
          if (!mbar_wait(&raw_empty[2 * (i & 1) + kv], ((i >> 1) & 1) ^ 1, abort_v, p.dev_flag, 89))
            break;
          fetch(i, kv);
        }
        // copies in flight complete before the CTA may exit
        for (int j = max(0, i - 2); j < i; ++j)
          mbar_wait(&raw_full[2 * (j & 1) + kv], (j >> 1) & 1, abort_v, p.dev_flag, 0, false);
      }
    } else {
      // ---------------------------------------------------------- widening: half of the warps K, half V
      constexpr int N = 16 * CV_WARPS;
      const Widen<DH, N> w((tid - 32 * (1 + SM_WARPS)) % N);
      const bool kv = warp > SM_WARPS + CV_WARPS / 2;
      const float inv = c8_inverse(kv ? most.y : most.x) * LIFT;
      uint64_t *full = kv ? v_full : k_full, *empty = kv ? v_empty : k_empty;
      const float *power = (const float *)powers + kv;
      const uint32_t tile = kv ? sV : sK;
      float pa = power[2 * c0], pb = power[2 * second(0)];
      for (int i = 0; i < n; ++i) {
        const int b = i & 1, ph = (i >> 1) & 1, st = 2 * b + kv;
        const float fa = pa * inv, fb = pb * inv;
        if (i + 1 < n) pa = power[2 * (c0 + 2 * i + 2)], pb = power[2 * second(i + 1)];
        const bool ok = mbar_wait(&raw_full[st], ph, abort_v, p.dev_flag, 90) &&
                        (i < 2 || mbar_wait(&empty[b], ph ^ 1, abort_v, p.dev_flag, 84));
        if (!__all_sync(0xffffffffu, ok)) break;
        const uint8_t *codes = raw + st * BB;
        const HalfFactor ha(fa), hb(fb);
        auto widen = [&](auto low) {
#pragma unroll
          for (int j = 0; j < Widen<DH, N>::EACH; ++j)
            w.template store<low>(tile + b * TBYTES, w.load(codes, codes + BB / 2, j),
                                  j < Widen<DH, N>::EACH / 2 ? ha : hb, j);
        };
        // (both products for all pages: 64 rows over 16384 27.4 us, 512 over 5000 48.7; as it is 26.7
        // and 47.4)
        if (ha.low || hb.low)
          widen(std::true_type{});
        else
          widen(std::false_type{});
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&full[b]);
          mbar_arrive(&raw_empty[st]);
        }
      }
    }
  } else {
    // ------------------------------------------------------------ softmax
    const int mq = bd.y * p.grp;
    // (a place without a vector is not masked: it would keep its warp at the masking)
    const int lim = min(real ? p.pos[row] : 0x7FFFFFFF, c1 * KVR_PAGE - 1);
    constexpr int HK = CH / KP, OC = DH / KP;  // keys of a step, columns of O, of this thread
    const uint32_t tl = tmem + ((uint32_t)(quarter * 32) << 16), tO = tl + NS * CH + part * OC;
    const int bar_id = 1 + quarter;
    constexpr int GROUP = 32 * KP;  // threads of a quarter's vectors
    auto group_bar = [&]() { asm volatile("bar.sync %0, %1;" ::"r"(bar_id), "n"(GROUP) : "memory"); };
    auto hand_over = [&](float x, auto f) {  // f over the parts' x, to all of them
      if (part) sx[part - 1][vi] = x;
      group_bar();
      if (!part) {
#pragma unroll
        for (int o = 0; o < KP - 1; ++o) x = f(x, sx[o][vi]);
        sx[0][vi] = x;
      }
      group_bar();
      x = sx[0][vi];
      group_bar();
      return x;
    };
    auto group_any = [&](bool x) {
      int r;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %2, 0;\n\t"
          "barrier.cta.red.or.pred p, %1, %3, q;\n\tselp.s32 %0, 1, 0, p;\n\t}"
          : "=r"(r)
          : "r"(bar_id), "r"(x ? 1 : 0), "n"(GROUP)
          : "memory");
      return r != 0;
    };
    float qk_scale = p.scale * most.x * LIFT_INV;
    {
      float m = 0.f;
#pragma unroll
      for (int k = 0; k < QP; ++k) m = fmaxf(m, bf16_magnitude(qx[k]));
      m = hand_over(m, [](float a, float b) { return fmaxf(a, b); });
      const int e = half_exponent(m);
      qk_scale = fmaxf(qk_scale * exp2_of(e), FLT_MIN);  // (zero would make a masked score NaN)
      const float f = half_factor(m, e);
      const uint32_t q0 = sQ + vi * 128;
#pragma unroll
      for (int k = 0; k < QP; ++k) {
        const int c = part * QP + k;
        qx[k] = halves_of(qx[k], f);
        *(uint4 *)__cvta_shared_to_generic(q0 + (c >> 3) * HB + (((c & 7) ^ (vi & 7)) << 4)) = qx[k];
      }
      if (p.vectors && split == 0) {  // for the weights: the vector itself
        const size_t at = (size_t)g * p.weigh.nv_pad + bd.x * p.grp;
        if (real) {
#pragma unroll
          for (int k = 0; k < QP; ++k)
            *((uint4 *)(p.vectors + (at + vi) * DH) + part * QP + k) = qx[k];
          if (!part) p.factor[at + vi] = qk_scale;
        }
        // behind the last row those that fill a tile there
        const int fill = blockIdx.z + 1 == gridDim.z ? p.weigh.nv_pad - bd.x * p.grp : 0;
        for (int i = real ? vi + QV : vi; i < fill; i += QV) {
#pragma unroll
          for (int k = 0; k < QP; ++k)
            *((uint4 *)(p.vectors + (at + i) * DH) + part * QP + k) = make_uint4(0u, 0u, 0u, 0u);
          if (!part) {
            p.factor[at + i] = 0.f;
            put_weighing(p.weigh, at + i, -1, 0.f, 0.f);
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(&q_full);
    }
    float m = -INFINITY, l = 0.f;  // reference maximum, this part's sum of exponentials
    bool dead = false;             // warp-uniform: a wait ran out; the named barriers go on
    for (int i = 0; i < n; ++i) {
      const int key0 = (c0 + 2 * i) * KVR_PAGE + part * HK;
      const uint32_t tS = tl + i % NS * CH + part * HK;
      if (!dead)
        dead = !__all_sync(0xffffffffu,
                           mbar_wait(&s_full[i % NS], (i / NS) & 1, abort_v, p.dev_flag, 86));
      // The scores in parts of 32: the maximum of all first, then the exponentials, read again
      // (held across the rescaling of O they were spilled).
      uint32_t s[32];
      float ms = -INFINITY;
      bool masked = false;
      auto load_scores = [&](int k) {
        tmem_ld32_nowait(tS + 32 * k, s);
        tmem_wait_ld();
        if (masked) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (key0 + 32 * k + j > lim) s[j] = 0xff800000u;  // -inf
        }
      };
      if (!dead) {
        tc_fence_after();
        masked = !__all_sync(0xffffffffu, key0 + HK - 1 <= lim);
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int k = 0; k < HK / 32; ++k) {
          load_scores(k);
#pragma unroll
          for (int j = 0; j < 32; ++j) mx[j & 3] = fmaxf(mx[j & 3], __uint_as_float(s[j]));
        }
        ms = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * qk_scale;
      }
      if (group_any(ms > m + RESCALE_LOG2)) {
        ms = hand_over(ms, [](float x, float y) { return fmaxf(x, y); });
        const bool grow = ms > m + RESCALE_LOG2;
        const float mn = ceilf(ms);
        const float alpha = grow ? ex2(m - mn) : 1.f;  // m = -inf: 0, and O is exactly zero
        if (!dead && i > 0) {
          // the product before has to be in O (this one waits for P)
          dead = !__all_sync(0xffffffffu, mbar_wait(&o_done[(i - 1) % NS], ((i - 1) / NS) & 1, abort_v,
                                                    p.dev_flag, 87));
          tc_fence_after();
          if (!dead) {
#pragma unroll
            for (int k = 0; k < OC / 16; ++k) {
              float o[16];
              tmem_ld16(tO + 16 * k, o);
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] *= alpha;
              tmem_st16(tO + 16 * k, o);
            }
          }
        }
        l *= alpha;
        if (grow) m = mn;
      }
      if (dead) continue;
      const float nm = m == -INFINITY ? 0.f : HALF_LIFT - m;  // no key yet: P = 0
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < HK / 32; ++k) {
        load_scores(k);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t w[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            float x, y;
            fma2(x, y, s[16 * h + 2 * j], s[16 * h + 2 * j + 1], qk_scale, nm);
            x = ex2(x);
            y = ex2(y);
            const __half2 u = __floats2half2_rn(x, y);
            w[j] = *(const uint32_t *)&u;
            add2(sum[2 * (j & 1)], sum[2 * (j & 1) + 1], x, y);
          }
          tmem_st8_nowait(tS + 16 * k + 8 * h, w);  // below the scores yet to be read
        }
      }
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&p_full[i % NS]);
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
    if (!dead)
      dead = !__all_sync(0xffffffffu, mbar_wait(&o_done[(n - 1) % NS], ((n - 1) / NS) & 1, abort_v,
                                                p.dev_flag, 88));
    const float lt = hand_over(l, [](float a, float b) { return a + b; });
    if (!dead) {
      tc_fence_after();
      // O by way of the Q tile (free now), whose rows' parts are this warp's own
      constexpr int RC = OC / 8;
      uint8_t *st = (uint8_t *)__cvta_shared_to_generic(sQ) + part * OC * 2;
      auto piece = [&](int r, int c) {
        return (uint4 *)(st + r * (DH * 2) + ((c ^ (r & (RC - 1))) << 4));
      };
      const size_t bs = ((size_t)split * p.n_blocks + blockIdx.z) * p.G + g;
      if (p.n_splits == 1) {
        float inv = lt > 0.f ? 1.f / lt : 0.f;
        inv *= most.y * LIFT_INV;
        if (p.vectors && real && part == 0)
          put_weighing(p.weigh, (size_t)g * p.weigh.nv_pad + bd.x * p.grp + vi, p.pos[row], m, lt);
#pragma unroll
        for (int k = 0; k < OC / 16; ++k) {
          uint32_t o[16], y[8];
          tmem_ld16_nowait(tO + 16 * k, o);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const __nv_bfloat162 x = __floats2bfloat162_rn(__uint_as_float(o[2 * j]) * inv,
                                                           __uint_as_float(o[2 * j + 1]) * inv);
            y[j] = *(const uint32_t *)&x;
          }
          *piece(vi, 2 * k) = make_uint4(y[0], y[1], y[2], y[3]);
          *piece(vi, 2 * k + 1) = make_uint4(y[4], y[5], y[6], y[7]);
        }
        __syncwarp();
        for (int e = lane; e < 32 * RC; e += 32) {
          const int r = quarter * 32 + e / RC, c = e % RC;
          if (r < mq)
            *(uint4 *)(p.out + ((size_t)(bd.x + r / p.grp) * p.H + g * p.grp + r % p.grp) * DH +
                       part * OC + c * 8) = *piece(r, c);
        }
      } else {
        // unnormalised O and (max, sum) for the combine, half of the part's columns at a time
        if (real && part == 0) p.ws_ml[bs * WS_MAXQ + vi] = make_float2(m, lt);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          if (half) __syncwarp();
          uint32_t o[OC / 2];
#pragma unroll
          for (int k = 0; k < OC / 16; ++k) tmem_ld8_nowait(tO + half * (OC / 2) + 8 * k, o + 8 * k);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < OC / 8; ++c)
            *piece(vi, c) = make_uint4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
          __syncwarp();
          for (int e = lane; e < 32 * RC; e += 32) {
            const int r = quarter * 32 + e / RC, c = e % RC;
            if (r < mq)
              *(uint4 *)(p.ws_o + (bs * WS_MAXQ + r) * DH + part * OC + half * (OC / 2) + c * 4) =
                  *piece(r, c);
          }
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 0)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                 "r"(TMEM_ROWS)
                 : "memory");
}

// ---- weights ----

constexpr int TILE = 128;      // keys, and query vectors, of a product
constexpr int KT = 2;          // tiles of keys that a CTA holds at once
constexpr int KEY_TILES = 8;   // such pairs of a CTA, at most
constexpr int Q_STAGES = 5;    // tiles of queries in flight
constexpr int S_SLOTS = 3;     // scores in TMEM, of a key tile and a tile of vectors each
constexpr int CONSUMERS = 8;   // warps of a key tile: four lane quarters, each half of the columns
constexpr int NT = 64 + 32 * CONSUMERS * KT;
constexpr uint32_t TMEM_COLS = 512;  // scores, then K (two halves a column)

// After attention by way of pages: the vectors of each KV head, row by row, as halves scaled by a
// power of two, and of each what takes a product to the log2 of its weight and the last key that it
// sees: -1 where its softmax is not finite.  Eight entries a lane.  Bound by its launch and L2: 4096
// rows of 28 heads, 29 MB in and out, 14 us.
template <int DH>
__global__ void __launch_bounds__(256)
    k_c8_vectors(const C8ManyArgs p, const __nv_bfloat16 *q, int ldq) {
  constexpr int LANES = DH / 8, PER = 256 / LANES;  // lanes of a vector, vectors of a CTA at once
  const int g = blockIdx.y, piece = threadIdx.x % LANES;
  __shared__ uint32_t s_max[2];
  if (threadIdx.x < 2) s_max[threadIdx.x] = 0;
  pdl_trigger();
  pdl_wait();
  __syncthreads();
  const float power =
      largest_powers<256>(p.cache.power + p.cache.index(p.layer, g, 0), p.n_pages, s_max).x * LIFT_INV;
  if (blockIdx.x == 0 && threadIdx.x == 0) p.key_power[g] = power;
  for (int v = blockIdx.x * PER + threadIdx.x / LANES; v < p.nv_pad; v += gridDim.x * PER) {
    const size_t at = (size_t)g * p.nv_pad + v;
    uint4 x = make_uint4(0, 0, 0, 0);
    float2 stats = make_float2(0.f, 0.f);
    float factor = 0.f, minus = -INFINITY, inverse = 0.f;
    int pos = -1, last = -1;
    if (v < p.rows * p.grp) {
      const int row = v / p.grp, head = g * p.grp + v % p.grp;
      x = *(const uint4 *)(q + (size_t)row * ldq + (size_t)head * DH + 8 * piece);
      stats = p.stats[(size_t)row * p.H + head];
      pos = p.pos[row];
    }
    float m = bf16_magnitude(x);
#pragma unroll
    for (int o = LANES / 2; o; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
    const int e = half_exponent(m);
    *(uint4 *)(p.vectors + at * DH + 8 * piece) = halves_of(x, half_factor(m, e));
    if (piece == 0) {
      if (stats.y > 0.f && stats.y < INFINITY) {
        factor = exp2_of(e) * p.scale * power;
        minus = -stats.x;
        inverse = stats.y;
        last = pos;
      }
      p.factor[at] = factor;
      p.minus[at] = minus;
      p.inverse[at] = inverse;
      p.last[at] = last;
    }
  }
}

__device__ __forceinline__ void add_weight(const C8ManyArgs &p, int g, int e, float sum) {
  float *w = p.weight + (size_t)g * p.cache.pages * KVR_PAGE + e;
  *w = p.decay == 0.f ? sum : fmaf(p.decay, *w, sum);
}

// A CTA takes some pairs of tiles of 128 keys of a KV head, one after another, and a run of tiles
// of 128 query vectors:
//   S = K Q^T   M 128 keys x N 128 vectors x K head_dim, K from TMEM (its codes widened into it once
//               a pair, from registers that they reached during the pair before), Q from shared
//               memory, S in one of three places in TMEM: products run while others are summed;
//   sums        eight warps a key tile: a thread has four keys (TMEM lanes) and an eighth of the
//               vectors, so that the sum over vectors of 2^(c S - m) / l stays in its registers from
//               the first tile to the last (with one key a thread, c and m of every
//               vector were 128 wavefronts a warp and tile: 2048 clocks).
// One run's sums go to the weights, several runs' to partial sums, which k_c8_add adds in order.
// With K in shared memory, too, a product of 64 clocks took 104: 8 KB of operands each, beside Q's
// arrival. 4096 rows of 28 heads over 12345 entries, 302 GFLOP: 270 us (1.1 PFLOP/s); a tile of
// vectors and a pair of key tiles take 2140 clocks, of which the tensor cores are busy for 1000,
// the exponentials' unit for 1000 and the schedulers for 1170.  Without exponentials it takes 37 us
// less, without loads of c, m and l 42, with an eighth of the products 15, without Q's arrival the
// same: no unit bounds it, but four warps a scheduler in the order of their scores do.  Slower were
// all scores of a thread's half in registers at once (17 us: 96 registers a thread, spills), sixteen
// vectors at a time, the next ones on their way (10), and warps with a quarter of the vectors for
// both key tiles (31, with half of the loads of c, m and l).
template <int DH>
__global__ void __launch_bounds__(NT, 1)
    k_c8_weigh_many(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ C8ManyArgs p) {
  constexpr int HALVES = DH / 64;          // 128-byte column blocks of a row
  constexpr uint32_t HB = TILE * 128;      // one of them, of a tile
  constexpr uint32_t TBYTES = HB * HALVES;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(16) float s_c[Q_STAGES][TILE], s_ref[Q_STAGES][TILE], s_inv[Q_STAGES][TILE];
  __shared__ __align__(16) int s_last[Q_STAGES][TILE];
  __shared__ float s_sum[KT][TILE];
  __shared__ __align__(8) uint64_t k_full, q_full[Q_STAGES], q_empty[Q_STAGES], s_full[S_SLOTS],
      s_empty[S_SLOTS], drain_bar;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_f, s_first[KEY_TILES];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // key tiles are the slowest index: the last CTAs, of the last keys, have the fewest vectors
  const int g = blockIdx.y, G = p.cache.G, kt0 = blockIdx.z * p.key_tiles, run = blockIdx.x;
  const int n_kt = min(p.key_tiles, p.keys / (KT * TILE) - kt0);
  const uint32_t base = (su32(smem_raw) + 1023u) & ~1023u;
  const uint32_t sQ = base;
  volatile int *abort_v = &abort_f;

  if (tid == 0) {
    mbar_init(&k_full, CONSUMERS * KT);
    for (int i = 0; i < Q_STAGES; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&q_empty[i], 1 + CONSUMERS * KT);
    }
    for (int i = 0; i < S_SLOTS; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&s_empty[i], CONSUMERS);
    }
    mbar_init(&drain_bar, 1);
    abort_f = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // the tiles of this CTA's run that see any of a pair's keys: from the first one whose last row
  // does
  const int t1 = min(p.n_tiles, (run + 1) * p.per);
  if (warp >= 2)
    for (int k = warp - 2; k < n_kt; k += CONSUMERS * KT) {
      int t = run * p.per;
      for (; t < t1; t += 32) {
        const int row = min(p.rows - 1, ((t + lane + 1) * TILE - 1) / p.grp);
        const uint32_t hit =
            __ballot_sync(0xFFFFFFFFu, t + lane < t1 && p.pos[row] >= (kt0 + k) * KT * TILE);
        if (hit) {
          t += __ffs(hit) - 1;
          break;
        }
      }
      if (lane == 0) s_first[k] = min(t, t1);
    }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                     su32(&tmem_slot)),
                 "r"(TMEM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  pdl_trigger();  // every CTA of the grid that is to allocate TMEM has it by then

  if (warp == 0) {
    // ------------------------------------------------------------ queries
    pdl_wait();
    if (lane == 0) {
      tma_prefetch_desc(&tm_q);
      int it = 0;
      bool ok = true;
      for (int k = 0; k < n_kt && ok; ++k)
        for (int t = s_first[k]; t < t1; ++t, ++it) {
          const int st = it % Q_STAGES;
          ok = it < Q_STAGES ||
               mbar_wait(&q_empty[st], (it / Q_STAGES - 1) & 1, abort_v, p.dev_flag, 72);
          if (!ok) break;
          const int at = g * p.nv_pad + t * TILE;
          mbar_expect_tx(&q_full[st], TBYTES + TILE * 16);
#pragma unroll
          for (int h = 0; h < HALVES; ++h)
            tma_load_2d((void *)__cvta_shared_to_generic(sQ + st * TBYTES + h * HB), &tm_q,
                        &q_full[st], h * 64, at);
          bulk_load(s_c[st], p.factor + at, TILE * 4, &q_full[st]);
          bulk_load(s_ref[st], p.minus + at, TILE * 4, &q_full[st]);
          bulk_load(s_inv[st], p.inverse + at, TILE * 4, &q_full[st]);
          bulk_load(s_last[st], p.last + at, TILE * 4, &q_full[st]);
        }
      // copies in flight complete before the CTA may exit
      for (int i = max(0, it - Q_STAGES); i < it; ++i)
        mbar_wait(&q_full[i % Q_STAGES], (i / Q_STAGES) & 1, abort_v, p.dev_flag, 0, false);
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMA
    const uint32_t id = idesc_16(true, TILE, TILE);
    const uint64_t dq0 = sw128_desc(sQ);
    auto wait = [&](uint64_t *bar, int parity, int code) -> bool {
      return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_v, p.dev_flag, code));
    };
    bool ok = true;
    int it = 0;
    for (int k = 0, used = 0; k < n_kt && ok; ++k) {
      if (s_first[k] >= t1) continue;
      ok = wait(&k_full, used++ & 1, 73);
      for (int t = s_first[k]; t < t1 && ok; ++t, ++it) {
        const int st = it % Q_STAGES;
        ok = wait(&q_full[st], (it / Q_STAGES) & 1, 74);
        for (int u = 0; u < KT && ok; ++u) {
          const int j = it * KT + u, slot = j % S_SLOTS;
          ok = j < S_SLOTS || wait(&s_empty[slot], (j / S_SLOTS - 1) & 1, 75);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t dq = dq0 + (uint64_t)((st * TBYTES) >> 4);
            const uint32_t tK = tmem + S_SLOTS * TILE + u * (DH / 2);
#pragma unroll
            for (int kk = 0; kk < DH / 16; ++kk)
              mma_ts(tmem + slot * TILE, tK + kk * 8,
                     dq + (uint64_t)(((kk >> 2) * HB + (kk & 3) * 32) >> 4), id, kk > 0 ? 1u : 0u);
            mma_commit(&s_full[slot]);
            if (u == KT - 1) mma_commit(&q_empty[st]);
          }
          __syncwarp();
        }
      }
    }
    // every product issued here completes before TMEM is freed
    if (elect_one()) mma_commit(&drain_bar);
    __syncwarp();
    mbar_wait(&drain_bar, 0, abort_v, p.dev_flag, 0, false);
  } else {
    // ------------------------------------------------------------ keys and sums
    const int u = (warp - 2) / CONSUMERS, quarter = warp & 3, half = (warp - 2) >> 2 & 1;
    const int lg = lane >> 2, lt = lane & 3;
    const uint32_t tl = tmem + ((uint32_t)(quarter * 32) << 16);
    const size_t head = p.cache.index(p.layer, g, 0);
    // this thread's part of a key tile: half of the entries of one key, in the key's TMEM lane
    constexpr int EACH = DH / 32;  // pieces of 16 entries
    const int kr = quarter * 32 + lane;
    uint4 codes[EACH];
    float power = 0.f;
    pdl_wait();
    const float down = 1.f / p.key_power[g];  // (a power of two)
    auto load = [&](int k) {
      // past the last page the last one again: no vector sees those keys
      const int page = min(2 * ((kt0 + k) * KT + u) + kr / KVR_PAGE, p.n_pages - 1), r = kr % KVR_PAGE;
      const uint8_t *row = p.cache.blocks + (head + page) * c8_block_bytes(DH) + r * DH;
#pragma unroll
      for (int j = 0; j < EACH; ++j)
        codes[j] = *(const uint4 *)(row + 16 * c8_piece<DH>(r, half * EACH + j));
      power = p.cache.power[head + page].x;
    };
    load(0);
    bool dead = false;
    int it = 0;
    for (int k = 0; k < n_kt; ++k) {
      const int key0 = ((kt0 + k) * KT + u) * TILE, key = key0 + quarter * 32 + lg;
      // (the products of the pair before are done: this warp has seen the last one's scores)
      const int t0 = s_first[k];
      if (t0 < t1) {
        const HalfFactor f(power * down);  // (a warp's keys are of one page)
        auto store = [&](auto low) {
#pragma unroll
          for (int j = 0; j < EACH; ++j) {
            const uint32_t w[4] = {codes[j].x, codes[j].y, codes[j].z, codes[j].w};
            uint32_t o[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              c8_halves(w[i], o[2 * i], o[2 * i + 1]);
              o[2 * i] = times<low>(o[2 * i], f);
              o[2 * i + 1] = times<low>(o[2 * i + 1], f);
            }
            tmem_st8_nowait(tl + S_SLOTS * TILE + u * (DH / 2) + (half * EACH + j) * 8, o);
          }
        };
        if (f.low)
          store(std::true_type{});
        else
          store(std::false_type{});
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&k_full);
      }
      if (k + 1 < n_kt) load(k + 1);
      float sum[4][2] = {};  // of the lane's keys, its even vectors and its odd ones
      for (int t = t0; t < t1 && !dead; ++t, ++it) {
        const int st = it % Q_STAGES, job = it * KT + u, slot = job % S_SLOTS;
        const uint32_t ts = tl + slot * TILE + half * (TILE / 2);
        dead = !__all_sync(
            0xffffffffu, mbar_wait(&s_full[slot], (job / S_SLOTS) & 1, abort_v, p.dev_flag, 76) &&
                             mbar_wait(&q_full[st], (it / Q_STAGES) & 1, abort_v, p.dev_flag, 77));
        if (dead) break;
        tc_fence_after();
        const int own = half * (TILE / 2) + 2 * lt;
        const float *c = s_c[st] + own, *ref = s_ref[st] + own, *inv = s_inv[st] + own;
        const int *last = s_last[st] + half * (TILE / 2);
        // vectors that see only some of the tile's keys, or none
        const bool part = __any_sync(0xffffffffu, min(last[lane], last[lane + 32]) < key0 + TILE - 1);
#pragma unroll
        for (int x0 = 0; x0 < TILE / 2; x0 += 32) {
          // keys lg, + 8, + 16, + 24 of the quarter; vectors 2 lt, + 1 of every eight
          uint32_t s[2][16];
          tmem_ld_16x256_nowait(ts + x0, s[0]);
          tmem_ld_16x256_nowait(ts + (16u << 16) + x0, s[1]);
          tmem_wait_ld();
          if (x0 == TILE / 2 - 32) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&s_empty[slot]);
          }
          auto add = [&](auto some) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float2 f = *(const float2 *)&c[x0 + 8 * i], l = *(const float2 *)&ref[x0 + 8 * i],
                           w = *(const float2 *)&inv[x0 + 8 * i];
              int2 z;
              if (some) z = *(const int2 *)&last[x0 + 8 * i + 2 * lt];
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                float y0, y1;
                fma2(y0, y1, s[r >> 1][4 * i + 2 * (r & 1)], s[r >> 1][4 * i + 2 * (r & 1) + 1], f.x,
                     f.y, l.x, l.y);
                y0 = ex2(y0);
                y1 = ex2(y1);
                if (some) {
                  if (key + 8 * r > z.x) y0 = 0.f;
                  if (key + 8 * r > z.y) y1 = 0.f;
                }
                fma2_add(sum[r][0], sum[r][1], y0, y1, w.x, w.y);
              }
            }
          };
          if (part)
            add(std::true_type{});
          else
            add(std::false_type{});
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&q_empty[st]);
      }
      // a key's four lanes, then the halves
      float all = 0.f;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        float x = sum[r][0] + sum[r][1];
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        if (lt == r) all = x;
      }
      const int own = quarter * 32 + 8 * lt + lg;
      if (half == 1) s_sum[u][own] = all;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + u), "n"(32 * CONSUMERS) : "memory");
      if (half == 0) {
        all += s_sum[u][own];
        if (p.runs > 1)
          p.partial[((size_t)run * G + g) * p.keys + key0 + own] = all;
        else if (key0 + own < p.len)
          add_weight(p, g, key0 + own, all);
      }
      if (k + 1 < n_kt)
        asm volatile("bar.sync %0, %1;" ::"r"(1 + u), "n"(32 * CONSUMERS) : "memory");
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                 "r"(TMEM_COLS)
                 : "memory");
}

// The runs' sums, in order, onto the document's weights.
__global__ void __launch_bounds__(256) k_c8_add(const C8ManyArgs p) {
  const int e = blockIdx.x * 256 + threadIdx.x, g = blockIdx.y;
  pdl_trigger();
  pdl_wait();
  if (e >= p.len) return;
  float sum = 0.f;
  if (e < p.keys)
    for (int z = 0; z < p.runs; ++z) sum += p.partial[((size_t)z * p.cache.G + g) * p.keys + e];
  add_weight(p, g, e, sum);
}

template <int DH>
const char *weigh(C8ManyArgs p, const void *q, int ldq, int *n, cudaStream_t s) {
  constexpr size_t smem = 1024 + Q_STAGES * (size_t)TILE * DH * 2;
  static PerDevice<size_t> limit;
  if (const char *e = smem_opt_in(limit, k_c8_weigh_many<DH>, smem)) return e;
  CUtensorMap tm_q;
  if (!make_tmap_bf16(&tm_q, p.vectors, p.cache.G * p.nv_pad, DH, TILE)) return "tensor map of vectors";
  // one run's CTAs reach all entries: those past the last one that is seen only decay
  if (p.runs == 1) p.keys = std::max(p.keys, (p.len + KT * TILE - 1) / (KT * TILE) * (KT * TILE));
  const int G = p.cache.G, groups = (p.keys / (KT * TILE) + p.key_tiles - 1) / p.key_tiles;
  if (q)
    launch_pdl(k_c8_vectors<DH>, dim3(std::min(p.nv_pad * DH / 2048, 1216 / G + 1), G), 256, 0, s, p,
               (const __nv_bfloat16 *)q, ldq);
  launch_pdl(k_c8_weigh_many<DH>, dim3(p.runs, G, groups), NT, smem, s, tm_q, p);
  if (p.runs > 1) launch_pdl(k_c8_add, dim3((p.len + 255) / 256, p.cache.G), 256, 0, s, p);
  *n = 1 + (q != nullptr) + (p.runs > 1);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

template <int DH>
const char *rows(const C8RowsArgs &p, bool settled, cudaStream_t s) {
  constexpr size_t smem = 1024 + 5 * (size_t)CH * DH * 2 + RAW * c8_block_bytes(DH);
  static PerDevice<size_t> limit;
  if (const char *e = smem_opt_in(limit, k_c8_rows<DH>, smem)) return e;
  const dim3 grid(p.n_splits, p.G, p.n_blocks);
  if (settled)
    launch_pdl(k_c8_rows<DH>, grid, NTR, smem, s, p);
  else
    k_c8_rows<DH><<<grid, NTR, smem, s>>>(p);
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace

void launch_c8_unpack(const C8View &v, int layer, int n_pages, void *pages, float2 *page_power,
                      bool settled, cudaStream_t s) {
  auto *kernel = v.dh == 128 ? k_c8_unpack<128> : k_c8_unpack<64>;
  const dim3 grid(v.G, n_pages);
  if (settled)
    launch_pdl(kernel, grid, dim3(256), 0, s, v, layer, n_pages, (__half *)pages, page_power);
  else
    kernel<<<grid, 256, 0, s>>>(v, layer, n_pages, (__half *)pages, page_power);
}

// Runs of up to 32 tiles; pairs of key tiles of a CTA that make it at least sixteen products, as long
// as every SM has work.
C8ManyShape c8_many_shape(int rows, int grp, int n_pages, int G, int num_sms) {
  C8ManyShape x;
  x.tiles = (rows * grp + TILE - 1) / TILE;
  x.nv_pad = x.tiles * TILE;
  const int pairs = (n_pages + 2 * KT - 1) / (2 * KT);
  x.keys = pairs * KT * TILE;
  x.per = std::min(x.tiles, 32);
  x.runs = (x.tiles + x.per - 1) / x.per;
  const long long all = (long long)pairs * G * x.runs;
  x.key_tiles = (int)std::min<long long>(std::min(KEY_TILES, (8 + x.per - 1) / x.per),
                                         (all + num_sms - 1) / num_sms);
  return x;
}

const char *launch_c8_weigh_many(const C8ManyArgs &p, const void *q, int ldq, int dh, int *n,
                                 cudaStream_t s) {
  return dh == 128 ? weigh<128>(p, q, ldq, n, s) : weigh<64>(p, q, ldq, n, s);
}

const char *launch_c8_rows(const C8RowsArgs &p, int dh, bool settled, cudaStream_t s) {
  return dh == 128 ? rows<128>(p, settled, s) : rows<64>(p, settled, s);
}

}  // namespace kvr
