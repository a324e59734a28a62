// k_packed_attn.cu -- attention over packed caches (packed.cuh): a few query vectors
// against the 4-bit keys and values of their document, all of them up to the row's
// position or those of listed blocks.
//
// A CTA owns a tile of up to eight query vectors (a row's heads of one KV head,
// for several rows as many as fit) and a part of its pages; a warp takes every
// WARPS-th page of the part by itself.  Per page, with keys as the rows of
// m16n8k16 products (so that eight vectors fill one):
//   S^T = K Q^T    the page's K half arrives in shared memory by one bulk copy, in
//                  the order of the products' A fragments: a 16-byte load is four
//                  fragments, each four conversions of two codes and four products with
//                  the scales, which are exact in half;
//                  (V's scales are widened once a page, into the memory that K has left);
//   softmax        over the lane's own keys: the reference of a vector is raised only
//                  when a score exceeds it by 8 in the log2 domain, so a page costs a
//                  vote instead of a reduction; the sums stay apart until the end;
//   O^T += V^T P^T P in half, its fragments transposed by movmatrix; V^T like K.
// q is scaled by a power of two per vector so that it is a half as exactly as it
// was a bf16; an fp32 model's q and P go as two halves each (22 bits; P's second 2^11 above
// the first, so that a small weight, whose first is subnormal or zero, keeps its bits down
// to 2^-43 of the largest), with a page's products added to O in fp32 registers.  All sums
// are in fp32.
// The warps' (max, sum, O) meet in shared memory; those of a cluster's CTAs are brought
// into the memory of the CTA that adds the slice (0.5 us sooner than read from there: a
// token over 5000 positions 6.9 to 6.4); of several clusters the last to arrive adds
// them all, in order.
//
// The floor is the cache's bytes: one token over 131072 positions of 8 KV heads reads 151 MB,
// 22.3 us at the copy rate, and takes 30.5; sixteen documents of 8191 positions the same
// in 30.5.  Of that about 5 us are the launch, the first copy's way and the sums; between
// them an SM's 12 warps take 12 pages in 2.5 us, 6.7 TB/s over the chip, while its
// schedulers issue half the time (918 instructions a page and warp, 256 of them
// conversions of codes and 256 products with scales).  mma.sync serves because
// eight columns are all there is: with 128 rows of a tcgen05 tile a token's heads
// would leave 120 empty, and the widened keys would have to pass through shared memory.
// Many rows go that way (many_attention).
//
// A key whose row held a NaN or an infinity has NaN scales: its score is NaN for the
// vectors that see it, and its V scales are cleared before the products, so
// vectors that do not see it are untouched.
#include <cooperative_groups.h>
#include <math.h>

#include "packed.cuh"
#include "tc_ptx.cuh"

namespace kvr {
namespace {
using namespace ptx;

constexpr int STAGES = 2;           // pages in flight per warp
constexpr float RAISE = 8.f;        // headroom of the reference (log2)
constexpr float LOW = 2048.f;       // what the second half of a weight is lifted by
constexpr int SPARSE_MAX = 128;     // listed blocks of a part

// One contiguous copy into shared memory, counted at bar.
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes,
                                          uint64_t *bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
      ::"r"(su32(dst)), "l"(src), "r"(bytes), "r"(su32(bar))
      : "memory");
}

// D (16 x 8, fp32) += A (16 x 16) B (16 x 8), halves.
__device__ __forceinline__ void mma16816(float *d, const uint32_t *a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*(const __half2 *)&a, *(const __half2 *)&b);
  return *(const uint32_t *)&r;
}
__device__ __forceinline__ uint32_t half2_of(float lo, float hi) {
  const __half2 r = __floats2half2_rn(lo, hi);
  return *(const uint32_t *)&r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Fragments of a K or V word: registers of the tile's rows 0-7 (bytes 0, 1) and 8-15
// (bytes 2, 3), columns 0-7 (bytes 0, 2) and 8-15.  K: a scale for each half of the rows,
// the same half of s0 and of s1; V: one for each half of the columns.
template <int HI>
__device__ __forceinline__ uint32_t mul_by(uint32_t a, uint32_t s) {
  const __half2 s2 = *(const __half2 *)&s;
  const __half2 r = __hmul2(*(const __half2 *)&a, HI ? __high2half2(s2) : __low2half2(s2));
  return *(const uint32_t *)&r;
}
template <int HI>
__device__ __forceinline__ void k_fragment(uint32_t w, uint32_t s0, uint32_t s1, uint32_t *a) {
  uint32_t v[4];
  pack_values(w, v);
  a[0] = mul_by<HI>(v[0], s0);
  a[2] = mul_by<HI>(v[1], s0);
  a[1] = mul_by<HI>(v[2], s1);
  a[3] = mul_by<HI>(v[3], s1);
}
__device__ __forceinline__ void v_fragment(uint32_t w, uint32_t s0, uint32_t s1, uint32_t *a) {
  uint32_t v[4];
  pack_values(w, v);
  a[0] = mul2(v[0], s0);
  a[2] = mul2(v[1], s1);
  a[1] = mul2(v[2], s0);
  a[3] = mul2(v[3], s1);
}
// Four scale codes as two half2.
__device__ __forceinline__ void scales(uint32_t w, uint32_t &a, uint32_t &b) {
  a = __byte_perm(w, 0, 0x4140) << 7;
  b = __byte_perm(w, 0, 0x4342) << 7;
}

// Scales as halves: whether any is NaN (their sum is, and only then: none is negative), and
// those that are made zero (the larger of it and zero).
__device__ __forceinline__ __half2 half2_in(uint32_t x) { return *(const __half2 *)&x; }
__device__ __forceinline__ bool some_nan(uint4 x, uint4 y) {
  const __half2 a = __hadd2(__hadd2(half2_in(x.x), half2_in(x.y)),
                            __hadd2(half2_in(x.z), half2_in(x.w))),
                b = __hadd2(__hadd2(half2_in(y.x), half2_in(y.y)),
                            __hadd2(half2_in(y.z), half2_in(y.w))),
                c = __hadd2(a, b);
  return !__hbeq2(c, c);
}
__device__ __forceinline__ void no_nan(uint4 &x) {
  auto f = [](uint32_t &u) {
    const __half2 r = __hmax2(half2_in(u), __half2half2(__ushort_as_half(0)));
    u = *(const uint32_t *)&r;
  };
  f(x.x), f(x.y), f(x.z), f(x.w);
}

// Four entries of a row of q.
__device__ __forceinline__ void load4(const __nv_bfloat16 *p, float *x) {
  const uint2 u = *(const uint2 *)p;
  x[0] = __uint_as_float(u.x << 16);
  x[1] = __uint_as_float(u.x & 0xFFFF0000u);
  x[2] = __uint_as_float(u.y << 16);
  x[3] = __uint_as_float(u.y & 0xFFFF0000u);
}
__device__ __forceinline__ void load4(const float *p, float *x) {
  const float4 u = *(const float4 *)p;
  x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
}
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float a, float b, float c, float d) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(a, b), y = __floats2bfloat162_rn(c, d);
  *(uint2 *)p = make_uint2(*(const uint32_t *)&x, *(const uint32_t *)&y);
}
__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) {
  *(float4 *)p = make_float4(a, b, c, d);
}
__device__ __forceinline__ void add4(float4 &x, float f, float4 y) {
  x.x += f * y.x, x.y += f * y.y, x.z += f * y.z, x.w += f * y.w;
}

// Weight of partial sums (m, l) under the common maximum M; NaN sums stay NaN.
__device__ __forceinline__ float merge_weight(float m, float l, float M) {
  return l != l ? l : m == -INFINITY ? 0.f : ex2(m - M);
}

// CTAs of an SM: its registers hold 12 warps of a bf16 query, 8 of an fp32 one.
template <typename T>
constexpr int ctas_per_sm(int warps) {
  return sizeof(T) == 4 ? 8 / warps : 12 / warps;
}

template <int DH, typename T, bool SPARSE, int WARPS>
__global__ void __launch_bounds__(WARPS * 32, ctas_per_sm<T>(WARPS))
    k_packed_attn(const __grid_constant__ PackedAttnArgs p) {
  constexpr bool SPLIT = sizeof(T) == 4;
  constexpr int HB = pack_half_bytes(DH), CB = pack_code_bytes(DH), DB = DH / 16, DQ = DH / 64;
  extern __shared__ __align__(128) uint8_t smem[];  // [WARPS][STAGES][K half, V half]
  __shared__ __align__(8) uint64_t full[WARPS][STAGES][2];
  __shared__ float2 s_ml[WARPS][PACK_VEC];
  __shared__ float s_wgt[WARPS][PACK_VEC];
  __shared__ float2 s_tot[PACK_VEC];
  __shared__ int s_list[SPARSE ? SPARSE_MAX : 1], s_count, s_last, abort_f;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lg = lane >> 2, lt = lane & 3;
  const int g = blockIdx.y;
  volatile int *abort_v = &abort_f;

  if (lane == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full[warp][s][0], 1);
      mbar_init(&full[warp][s][1], 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid == 0) abort_f = 0;
  pdl_trigger();
  // the tables were sent ahead of the kernel before this one (a.settled), or this launch
  // waited for all before it: they are read ahead of the wait
  int vec0, nvec, n_parts, part, slot, counter, n_pages, page0 = 0;
  const uint8_t *blocks;
  if (SPARSE) {
    const int hc = (p.grp + PACK_VEC - 1) / PACK_VEC;  // chunks of a row's heads
    const int tile = blockIdx.x / p.parts_per_row, row = tile / hc, h0 = tile % hc * PACK_VEC;
    const PackedRow r = p.rows[row];
    part = blockIdx.x % p.parts_per_row;
    n_parts = p.parts_per_row;
    vec0 = row * p.grp + h0;
    nvec = min(PACK_VEC, p.grp - h0);
    slot = tile * n_parts;
    counter = tile;
    blocks = r.doc.block(p.layer, g, 0);
    pdl_wait();
    const int per = (p.n_blocks + n_parts - 1) / n_parts, i0 = part * per,
              i1 = min(p.n_blocks, i0 + per);
    const int own = r.pos < 0 ? -1 : r.pos / KVR_PAGE;
    if (warp == 0) {
      const int32_t *list = p.blocks + ((size_t)row * p.G + g) * p.n_blocks;
      int n = 0;
      for (int i = i0; i < i1; i += 32) {
        const int b = i + lane < i1 ? list[i + lane] : -1;
        const bool take = b >= 0 && b <= own;
        const uint32_t m = __ballot_sync(0xFFFFFFFFu, take);
        if (take) s_list[n + __popc(m & ((1u << lane) - 1))] = b;
        n += __popc(m);
      }
      if (lane == 0) s_count = n;
    }
    __syncthreads();
    n_pages = s_count;
  } else {
    const PackedPart t = p.parts[blockIdx.x];
    vec0 = t.vec0, nvec = t.nvec, n_parts = t.n_parts;
    part = t.part;
    slot = t.slot;
    counter = t.tile;
    page0 = t.page0;
    n_pages = t.page1 - t.page0;
    blocks = t.blocks + ((size_t)p.layer * p.G + g) * t.pages * pack_block_bytes(DH);
    __syncthreads();
    pdl_wait();
  }
  uint8_t *ring = smem + warp * (STAGES * 2 * HB);
  const int n_my = n_pages > warp ? (n_pages - warp + WARPS - 1) / WARPS : 0;
  auto page = [&](int i) {
    const int at = warp + i * WARPS;
    return SPARSE ? s_list[at] : page0 + at;
  };
  auto fetch = [&](int i, int kv) {  // one lane
    uint64_t *bar = &full[warp][i % STAGES][kv];
    mbar_expect_tx(bar, HB);
    bulk_load(ring + (i % STAGES * 2 + kv) * HB,
              blocks + (size_t)page(i) * (2 * HB) + kv * HB, HB, bar);
  };
  if (lane == 0)
    for (int i = 0; i < min(n_my, STAGES); ++i) {
      fetch(i, 0);
      fetch(i, 1);
    }

  // q: this lane's vector lg, four entries of every 16
  uint32_t qh[DB][2], ql[SPLIT ? DB : 1][2];
  float qscale;  // of the products, into the log2 domain
  {
    float x[DB][4], a = 0.f;
    const int vec = vec0 + lg;
    const bool in = lg < nvec;
    const T *q = (const T *)p.q + (size_t)(vec / p.grp) * p.ldq +
                 (size_t)(g * p.grp + vec % p.grp) * DH + 4 * lt;
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      if (in)
        load4(q + 16 * b, x[b]);
      else
        x[b][0] = x[b][1] = x[b][2] = x[b][3] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) a = fmaxf(a, fabsf(x[b][i]));
    }
    a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 1));
    a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, 2));
    const int e = half_exponent(a);
    const float down = half_factor(a, e);
    qscale = exp2_of(e) * p.scale;
#pragma unroll
    for (int b = 0; b < DB; ++b) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[b][i] *= down;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        qh[b][i] = half2_of(x[b][2 * i], x[b][2 * i + 1]);
        if (SPLIT) {
          const float2 f = __half22float2(*(const __half2 *)&qh[b][i]);
          ql[b][i] = half2_of(x[b][2 * i] - f.x, x[b][2 * i + 1] - f.y);
        }
      }
    }
  }
  // the vectors of this lane's columns of S^T and O^T: 2 lt and 2 lt + 1
  float sc[2];
  int pos[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    sc[c] = __shfl_sync(0xFFFFFFFFu, qscale, 4 * (2 * lt + c));
    // a column without a vector is never masked: its results go nowhere
    pos[c] = 2 * lt + c < nvec ? p.pos[(vec0 + 2 * lt + c) / p.grp] : 0x7FFFFFFF;
  }
  int least = min(pos[0], pos[1]);
  least = min(least, __shfl_xor_sync(0xFFFFFFFFu, least, 1));
  least = min(least, __shfl_xor_sync(0xFFFFFFFFu, least, 2));

  float o[DB][4], ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int b = 0; b < DB; ++b) o[b][0] = o[b][1] = o[b][2] = o[b][3] = 0.f;

  int done = 0;
  for (; done < n_my; ++done) {
    const int st = done % STAGES;
    uint8_t *kb = ring + st * 2 * HB, *vb = kb + HB;
    const int voff = (int)(vb - smem) + 16 * lane;  // (HB is whole 128s)
    bool ok = mbar_wait(&full[warp][st][0], done / STAGES & 1, abort_v, p.dev_flag, 1 << 12);
    if (!__all_sync(0xFFFFFFFFu, ok)) break;
    float s[4][4];
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
      s[kt][0] = s[kt][1] = s[kt][2] = s[kt][3] = 0.f;
      uint32_t sw[2 * DQ], ks[2][DQ][2];  // scales of the two keys
      if constexpr (DQ == 2) {
        const uint4 u = *(const uint4 *)(kb + CB + (kt * 8 + lg) * 2 * DB);
        sw[0] = u.x, sw[1] = u.y, sw[2] = u.z, sw[3] = u.w;
      } else {
        const uint2 u = *(const uint2 *)(kb + CB + (kt * 8 + lg) * 2 * DB);
        sw[0] = u.x, sw[1] = u.y;
      }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < DQ; ++b) scales(sw[h * DQ + b], ks[h][b][0], ks[h][b][1]);
#pragma unroll
      for (int d4 = 0; d4 < DQ; ++d4) {
        const uint4 w4 = *(const uint4 *)(kb + ((kt * DQ + d4) * 32 + lane) * 16);
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          uint32_t a[4];
          if (b & 1)
            k_fragment<1>(w[b], ks[0][d4][b >> 1], ks[1][d4][b >> 1], a);
          else
            k_fragment<0>(w[b], ks[0][d4][b >> 1], ks[1][d4][b >> 1], a);
          mma16816(s[kt], a, qh[4 * d4 + b][0], qh[4 * d4 + b][1]);
          if (SPLIT) mma16816(s[kt], a, ql[4 * d4 + b][0], ql[4 * d4 + b][1]);
        }
      }
    }
    const int first = page(done) * KVR_PAGE;
    ok = mbar_wait(&full[warp][st][1], done / STAGES & 1, abort_v, p.dev_flag, 1 << 13);
    if (!__all_sync(0xFFFFFFFFu, ok)) break;
    // scores; masked keys get none
    float top[2] = {-INFINITY, -INFINITY};
    // V's scales as halves, once for the eight lanes that take each, where K was
    uint4 *vs16 = (uint4 *)kb;  // [pairs of tiles 0 1, 2 3][db][t]
    uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
    if (lane < 4 * DB) {
      const uint4 c4 = *(const uint4 *)(vb + CB + lane * 16);
      scales(c4.x, x.x, x.y);
      scales(c4.y, x.z, x.w);
      scales(c4.z, y.x, y.y);
      scales(c4.w, y.z, y.w);
    }
    if (__any_sync(0xFFFFFFFFu, some_nan(x, y))) {
      // rows marked NaN (all their scales): their scores become NaN, their scales zero
      const uint4 n4 = *(const uint4 *)(vb + CB + lt * 16);
      const uint32_t nan[4] = {__vcmpeq4(n4.x, 0xFFFFFFFFu), __vcmpeq4(n4.y, 0xFFFFFFFFu),
                               __vcmpeq4(n4.z, 0xFFFFFFFFu), __vcmpeq4(n4.w, 0xFFFFFFFFu)};
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        const uint32_t m = __shfl_sync(0xFFFFFFFFu, nan[kt], lg >> 1);  // keys 4 (lg / 2) .. + 3
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (m >> (8 * ((lg & 1) + 2 * h)) & 1) s[kt][2 * h] = s[kt][2 * h + 1] = NAN;
      }
      no_nan(x);
      no_nan(y);
    }
    __syncwarp();
    if (lane < 4 * DB) {
      vs16[lane] = x;
      vs16[4 * DB + lane] = y;
    }
    if (first + KVR_PAGE - 1 > least) {
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (first + 16 * kt + pack_key_of(lg) + (i & 2) > pos[i & 1]) s[kt][i] = -INFINITY;
    }
#pragma unroll
    for (int kt = 0; kt < 4; ++kt)
#pragma unroll
      for (int i = 0; i < 4; ++i) top[i & 1] = fmaxf(top[i & 1], s[kt][i]);
    top[0] *= sc[0];  // scales are positive: the largest stays the largest
    top[1] *= sc[1];
    if (__any_sync(0xFFFFFFFFu, top[0] > ref[0] + RAISE || top[1] > ref[1] + RAISE)) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int x = 4; x < 32; x *= 2)
          top[c] = fmaxf(top[c], __shfl_xor_sync(0xFFFFFFFFu, top[c], x));
        if (top[c] > ref[c]) {
          if (ref[c] != -INFINITY) {  // before, all sums are zero (or NaN)
            const float f = ex2(ref[c] - top[c]);
            l[c] *= f;
#pragma unroll
            for (int b = 0; b < DB; ++b) {
              o[b][c] *= f;
              o[b][c + 2] *= f;
            }
          }
          ref[c] = top[c];
        }
      }
    }
    uint32_t ph[4][2], pl[SPLIT ? 4 : 1][2];  // fragments of P^T: 16 keys, lane's vector lg
    {
      const float base[2] = {HALF_LIFT - (ref[0] == -INFINITY ? 0.f : ref[0]),
                             HALF_LIFT - (ref[1] == -INFINITY ? 0.f : ref[1])};
#pragma unroll
      for (int kt = 0; kt < 4; ++kt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float x = ex2(fmaf(s[kt][2 * h], sc[0], base[0])),
                      y = ex2(fmaf(s[kt][2 * h + 1], sc[1], base[1]));
          const uint32_t u = half2_of(x, y);
          ph[kt][h] = transpose8x8(u);
          if (SPLIT) {
            const float2 f = __half22float2(*(const __half2 *)&u);
            pl[kt][h] = transpose8x8(half2_of((x - f.x) * LOW, (y - f.y) * LOW));
            l[0] += x;
            l[1] += y;
          }
        }
      if (!SPLIT) {  // the sums of the weights as they are used: a product with ones
        float t[4] = {l[0], l[1], 0.f, 0.f};
        const uint32_t ones[4] = {0x3C003C00u, 0, 0x3C003C00u, 0};  // rows 0-7
#pragma unroll
        for (int kt = 0; kt < 4; ++kt) mma16816(t, ones, ph[kt][0], ph[kt][1]);
        l[0] = t[0];
        l[1] = t[1];
      }
    }
    __syncwarp();
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      const uint4 w4 = *(const uint4 *)(smem + (voff ^ 16 * b) + 512 * b);  // unit lane ^ b
      const uint4 x4 = vs16[b * 4 + lt], y4 = vs16[4 * DB + b * 4 + lt];
      const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
      const uint32_t vs[8] = {x4.x, x4.y, x4.z, x4.w, y4.x, y4.y, y4.z, y4.w};
      float acc[4] = {0.f, 0.f, 0.f, 0.f}, low[4] = {0.f, 0.f, 0.f, 0.f};
      float *d = SPLIT ? acc : o[b];
#pragma unroll
      for (int kt = 0; kt < 4; ++kt) {
        uint32_t a[4];
        v_fragment(w[kt], vs[2 * kt], vs[2 * kt + 1], a);
        mma16816(d, a, ph[kt][0], ph[kt][1]);
        if (SPLIT) mma16816(low, a, pl[kt][0], pl[kt][1]);
      }
      if (SPLIT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[b][i] += fmaf(low[i], 1.f / LOW, acc[i]);
      }
    }
    // what was written here comes before the copies into the same memory
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0 && done + STAGES < n_my) {
      fetch(done + STAGES, 0);
      fetch(done + STAGES, 1);
    }
  }
  // after a wait that ran out: the copies in flight end before the memory is reused
  if (done < n_my)
    for (int i = done; i < min(n_my, done + STAGES); ++i)
      for (int kv = 0; kv < 2; ++kv)
        mbar_wait(&full[warp][i % STAGES][kv], i / STAGES & 1, abort_v, p.dev_flag, 0, false);
  __syncwarp();

  const int cl = p.cluster, rank = part % cl, nc = n_parts / cl;
  if (cl > 1) cluster_arrive();  // this CTA is done with its copies' memory

  // ---- the warps' sums, rows SD apart so that a column's four lanes meet four banks ----
  constexpr int SD = DH + 4, D4 = DH / 4;
  float *so = (float *)ring;  // [PACK_VEC][SD]
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int x = 4; x < 32 && SPLIT; x *= 2) l[c] += __shfl_xor_sync(0xFFFFFFFFu, l[c], x);
    if (lg == 0) s_ml[warp][2 * lt + c] = make_float2(ref[c], l[c]);
#pragma unroll
    for (int b = 0; b < DB; ++b) {
      so[(2 * lt + c) * SD + 16 * b + lg] = o[b][c];
      so[(2 * lt + c) * SD + 16 * b + lg + 8] = o[b][c + 2];
    }
  }
  __syncthreads();
  if (tid < 16 * PACK_VEC) {  // sixteen lanes a vector, a lane a warp
    const int vi = tid >> 4, w = tid & 15;
    const float2 ml = w < WARPS ? s_ml[w][vi] : make_float2(-INFINITY, 0.f);
    float M = ml.x;
#pragma unroll
    for (int x = 8; x; x /= 2) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, x));
    const float f = merge_weight(ml.x, ml.y, M);
    float L = f * ml.y;
#pragma unroll
    for (int x = 8; x; x /= 2) L += __shfl_xor_sync(0xFFFFFFFFu, L, x);
    if (w < WARPS) s_wgt[w][vi] = f;
    if (w == 0) s_tot[vi] = make_float2(M, L);
  }
  __syncthreads();
  auto out4 = [&](int i, float4 x, float L) {  // entries 4 (i % D4) .. of the tile's vector i / D4
    const int vec = vec0 + i / D4;
    const float f = L == 0.f ? 0.f : 1.f / L;  // no key: zeros
    store4((T *)p.out + ((size_t)(vec / p.grp) * p.H + g * p.grp + vec % p.grp) * DH + 4 * (i % D4),
           x.x * f, x.y * f, x.z * f, x.w * f);
  };
  auto warps_sum = [&](int i) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WARPS; ++w)
      add4(x, s_wgt[w][i / D4],
           *(const float4 *)(smem + w * (STAGES * 2 * HB) + (i / D4 * SD + i % D4 * 4) * 4));
    return x;
  };
  // ---- the cluster's sums: each CTA adds a slice of them, which the others bring ----
  const int n4 = nvec * D4, per4 = (n4 + cl - 1) / cl;
  const int i0 = min(n4, rank * per4), i1 = min(n4, i0 + per4);
  const size_t slot0 = ((size_t)(slot / cl) * p.G + g), at = slot0 + (size_t)(part / cl) * p.G;
  auto finish = [&](int i, float4 x, float M, float L) {
    if (nc == 1) {
      out4(i, x, L);
      return;
    }
    ((float4 *)p.ws_o)[at * PACK_VEC * D4 + i] = x;
    if (i == i0 || i % D4 == 0)
      p.ws_ml[(at * PACK_CLUSTER + rank) * PACK_VEC + i / D4] = make_float2(M, L);
  };
  if (cl == 1) {
    for (int i = tid; i < n4; i += WARPS * 32)
      finish(i, warps_sum(i), s_tot[i / D4].x, s_tot[i / D4].y);
  } else {
    namespace cg = cooperative_groups;
    const cg::cluster_group cluster = cg::this_cluster();
    // behind the first warp's sums: [rank][per4] sums, [rank][PACK_VEC] (max, sum)
    float4 *sums = (float4 *)(smem + 64 * DH);
    float2 *mls = (float2 *)(smem + 112 * DH);
    static_assert(PACK_VEC * SD * 4 <= 64 * DH &&
                      64 * DH + (PACK_VEC * D4 + PACK_CLUSTER) * 16 <= 112 * DH &&
                      112 * DH + PACK_CLUSTER * PACK_VEC * 8 <= STAGES * 2 * HB,
                  "within a warp's ring");
    cluster_wait();  // all are done with theirs
    for (int i = tid; i < n4; i += WARPS * 32) {
      const int to = i / per4;
      cluster.map_shared_rank(sums, to)[rank * per4 + i - to * per4] = warps_sum(i);
    }
    for (int i = tid; i < cl * PACK_VEC; i += WARPS * 32)
      cluster.map_shared_rank(mls, i / PACK_VEC)[rank * PACK_VEC + i % PACK_VEC] =
          s_tot[i % PACK_VEC];
    cluster_arrive();
    cluster_wait();
    for (int i = i0 + tid; i < i1; i += WARPS * 32) {
      const int vi = i / D4;
      float M = -INFINITY, L = 0.f;
      for (int k = 0; k < cl; ++k) M = fmaxf(M, mls[k * PACK_VEC + vi].x);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < cl; ++k) {
        const float2 ml = mls[k * PACK_VEC + vi];
        const float f = merge_weight(ml.x, ml.y, M);
        L += f * ml.y;
        add4(x, f, sums[k * per4 + i - i0]);
      }
      finish(i, x, M, L);
    }
  }
  if (nc == 1) return;
  // one thread's arrival releases, after the barrier, what all of the CTA wrote, and acquires
  // what the others did
  __syncthreads();
  int *arrived = p.counters + ((size_t)counter * p.G + g) * PACK_CLUSTER + rank;
  if (tid == 0) {
    int before;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;"
                 : "=r"(before)
                 : "l"(arrived)
                 : "memory");
    s_last = before == nc - 1;
  }
  __syncthreads();
  if (!s_last) return;
  if (tid == 0) *arrived = 0;
  // ---- the last cluster's CTAs add the slices of all, in order: MERGE clusters' sums in
  // flight a thread, the first of them while the weights are found (16 lanes a vector) ----
  constexpr int T32 = WARPS * 32, IT = (PACK_VEC * D4 + T32 - 1) / T32;  // entries of a thread / 4
  constexpr int MERGE = 20 / IT;
  float *wgt = (float *)smem;  // [nc][PACK_VEC]
  static_assert(PACK_MERGE * PACK_VEC * 4 <= WARPS * STAGES * 2 * HB, "within the rings");
  const size_t step = p.G;
  const float4 *src = (const float4 *)p.ws_o + slot0 * PACK_VEC * D4;
  float4 y[IT][MERGE];
  auto fetch_sums = [&](int k0) {
#pragma unroll
    for (int t = 0; t < IT; ++t)
#pragma unroll
      for (int k = 0; k < MERGE; ++k)
        if (i0 + tid + t * T32 < i1 && k0 + k < nc)
          y[t][k] = __ldcg(src + i0 + tid + t * T32 + (k0 + k) * step * PACK_VEC * D4);
  };
  fetch_sums(0);
  if (tid < 16 * PACK_VEC) {
    const int vi = tid >> 4, l16 = tid & 15;
    const int n = i0 < i1 && vi >= i0 / D4 && vi <= (i1 - 1) / D4 ? nc : 0;
    const float2 *part_ml = p.ws_ml + (slot0 * PACK_CLUSTER + rank) * PACK_VEC + vi;
    auto part_of = [&](int k) {
      return k < n ? __ldcg(&part_ml[k * step * PACK_CLUSTER * PACK_VEC])
                   : make_float2(-INFINITY, 0.f);
    };
    const float2 first = part_of(l16), second = part_of(l16 + 16);
    float M = fmaxf(first.x, second.x), L = 0.f;
    for (int k = l16 + 32; k < n; k += 16) M = fmaxf(M, part_of(k).x);
#pragma unroll
    for (int x = 8; x; x /= 2) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, x));
    for (int k = l16; k < n; k += 16) {
      const float2 ml = k < 16 ? first : k < 32 ? second : part_of(k);
      const float f = merge_weight(ml.x, ml.y, M);
      wgt[k * PACK_VEC + vi] = f;
      L += f * ml.y;
    }
#pragma unroll
    for (int x = 8; x; x /= 2) L += __shfl_xor_sync(0xFFFFFFFFu, L, x);
    if (l16 == 0) s_tot[vi] = make_float2(M, L);
  }
  __syncthreads();
  float4 x[IT];
#pragma unroll
  for (int t = 0; t < IT; ++t) x[t] = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < nc; k0 += MERGE) {
    if (k0) fetch_sums(k0);
#pragma unroll
    for (int t = 0; t < IT; ++t) {
      const int i = i0 + tid + t * T32;
#pragma unroll
      for (int k = 0; k < MERGE; ++k)
        if (i < i1 && k0 + k < nc) add4(x[t], wgt[(k0 + k) * PACK_VEC + i / D4], y[t][k]);
    }
  }
#pragma unroll
  for (int t = 0; t < IT; ++t) {
    const int i = i0 + tid + t * T32;
    if (i < i1) out4(i, x[t], s_tot[i / D4].y);
  }
}

template <int DH, typename T, bool SPARSE, int WARPS>
const char *run(const PackedAttnArgs &a, cudaStream_t s) {
  static PerDevice<size_t> state;
  auto *kernel = k_packed_attn<DH, T, SPARSE, WARPS>;
  const size_t smem = (size_t)WARPS * STAGES * pack_block_bytes(DH);
  if (const char *e = smem_opt_in(state, kernel, smem)) return e;
  const int hc = (a.grp + PACK_VEC - 1) / PACK_VEC;
  const dim3 grid(SPARSE ? a.n_rows * hc * a.parts_per_row : a.n_parts, a.G);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(WARPS * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = a.cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = g_pdl && a.settled ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}
template <int DH, typename T>
const char *run(const PackedAttnArgs &a, cudaStream_t s) {
  constexpr int MANY = sizeof(T) == 4 ? 8 : 12;
  if (a.blocks)
    return a.warps == 4 ? run<DH, T, true, 4>(a, s) : run<DH, T, true, MANY>(a, s);
  return a.warps == 4 ? run<DH, T, false, 4>(a, s) : run<DH, T, false, MANY>(a, s);
}

}  // namespace

int packed_attn_ctas_per_sm(int dtype, int warps) {
  return dtype == KVR_DTYPE_BF16 ? ctas_per_sm<__nv_bfloat16>(warps) : ctas_per_sm<float>(warps);
}
int packed_attn_max_blocks_per_part() { return SPARSE_MAX; }

const char *launch_packed_attention(const PackedAttnArgs &a, cudaStream_t s) {
  if (a.dtype == KVR_DTYPE_BF16)
    return a.dh == 128 ? run<128, __nv_bfloat16>(a, s) : run<64, __nv_bfloat16>(a, s);
  return a.dh == 128 ? run<128, float>(a, s) : run<64, float>(a, s);
}

}  // namespace kvr
