// k_packed.cu -- the packed cache's rows and blocks: quantising K/V rows as they are
// written, reading them back, and selecting blocks by their bounds.
#include <math.h>

#include "packed.cuh"

namespace kvr {
namespace {

// The rows [r0, r1) of segment seg and their page.
struct Segment {
  int page, r0, r1;
};
__device__ __forceinline__ int position(const PackedRows &r, int i) {
  return r.first >= 0 ? r.first + i : r.pos_d ? r.pos_d[i] : r.pos[i];
}
__device__ __forceinline__ Segment segment(const PackedRows &r, int seg) {
  Segment s;
  if (r.first >= 0) {
    s.page = r.first / KVR_PAGE + seg;
    s.r0 = max(0, s.page * KVR_PAGE - r.first);
    s.r1 = min(r.n, (s.page + 1) * KVR_PAGE - r.first);
    return s;
  }
  s.r0 = r.pos_d ? r.pos_d[r.n + seg] : r.seg[seg];
  s.r1 = r.pos_d ? r.pos_d[r.n + seg + 1] : r.seg[seg + 1];
  s.page = position(r, s.r0) / KVR_PAGE;
  return s;
}

// Eight entries of a row.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  static __device__ __forceinline__ void load(const __nv_bfloat16 *p, float *x) {
    const uint4 u = __ldcs((const uint4 *)p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ void store(__nv_bfloat16 *p, const float *x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *(const uint32_t *)&b;
    }
    __stcs((uint4 *)p, make_uint4(w[0], w[1], w[2], w[3]));
  }
  // x / s on the grid of the codes.  With r the rounded reciprocal of the four-bit s,
  // x r + 768 rounds to whole steps of 2^-14, far above r's error and far below the
  // distance of an eight-bit x from a midpoint of the codes (at least 2^-10 where
  // it is not one), so ties are ties and everything else keeps its side.
  static __device__ __forceinline__ float quotient(float x, float, float r) {
    return __fadd_rn(__fmaf_rn(x, r, 768.f), -768.f);
  }
};
template <>
struct Eight<float> {
  static __device__ __forceinline__ void load(const float *p, float *x) {
    const float4 a = __ldcs((const float4 *)p), b = __ldcs((const float4 *)p + 1);
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
  static __device__ __forceinline__ void store(float *p, const float *x) {
    __stcs((float4 *)p, make_float4(x[0], x[1], x[2], x[3]));
    __stcs((float4 *)p + 1, make_float4(x[4], x[5], x[6], x[7]));
  }
  static __device__ __forceinline__ float quotient(float x, float s, float) {
    return __fdiv_rn(x, s);
  }
};

// Four keys (4 kg ..) x eight entries (8 ch ..) of a block's half in shared memory, as one
// thread takes them: a word of eight codes per key.
template <int DH>
__device__ __forceinline__ void k_codes_load(const uint8_t *half, int kg, int ch, uint32_t *c) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const uint32_t a = *(const uint32_t *)(half + pack_k_code(DH, 4 * kg + j, 8 * ch));
    const uint32_t b = *(const uint32_t *)(half + pack_k_code(DH, 4 * kg + j, 8 * ch + 4));
    c[j] = __byte_perm(a, b, 0x5410);
    c[j + 2] = __byte_perm(a, b, 0x7632);
  }
}
template <int DH>
__device__ __forceinline__ void k_codes_store(uint8_t *half, int kg, int ch, const uint32_t *c) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    *(uint32_t *)(half + pack_k_code(DH, 4 * kg + j, 8 * ch)) = __byte_perm(c[j], c[j + 2], 0x5410);
    *(uint32_t *)(half + pack_k_code(DH, 4 * kg + j, 8 * ch + 4)) =
        __byte_perm(c[j], c[j + 2], 0x7632);
  }
}
__device__ __forceinline__ void v_codes_load(const uint8_t *half, int kg, int ch, uint32_t *c) {
  c[0] = c[1] = c[2] = c[3] = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t h = *(const uint16_t *)(half + pack_v_code(kg, 8 * ch + i));
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] |= (h >> (4 * j) & 15u) << (4 * i);
  }
}
__device__ __forceinline__ void v_codes_store(uint8_t *half, int kg, int ch, const uint32_t *c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    uint32_t h = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) h |= (c[j] >> (4 * i) & 15u) << (4 * j);
    *(uint16_t *)(half + pack_v_code(kg, 8 * ch + i)) = (uint16_t)h;
  }
}

// Values of eight codes with scale code sc, as halves (exact).
__device__ __forceinline__ void eight_values(uint32_t c, uint32_t sc, __half2 *v) {
  const uint32_t s2 = sc << 7 | sc << 23;
  const __half2 s = *(const __half2 *)&s2;
  uint32_t w[4];
  pack_values(c, w);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = __hmul2(*(const __half2 *)&w[i], s);
}

// The smallest power of two u with a <= 127 u.
__device__ __forceinline__ float unit_of(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = (int)(u >> 23) - 6 + ((u & 0x7FFFFFu) > 0x7E0000u);
  return __uint_as_float((uint32_t)max(e, 27) << 23);  // 2^-100 and up
}

// A CTA per (KV head, page, layer): the page's rows are quantised into a copy of the
// block in shared memory (the present one where the call does not write all of
// it), the key bounds taken over all rows present, and the block stored whole.
template <int DH, typename T>
__global__ void __launch_bounds__(2 * DH)
    k_packed_write(const PackedView v, const __grid_constant__ PackedRows rows, int len, int l0,
                   const T *k, const T *val) {
  constexpr int NT = 2 * DH, CH = DH / 8, HB = pack_half_bytes(DH);
  __shared__ __align__(16) uint8_t blk[2 * HB];
  __shared__ int row_of[KVR_PAGE];
  __shared__ __half2 red[2][NT / 32][DH / 2];
  __shared__ float amax[DH / 32];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = blockIdx.x, l = blockIdx.z;
  pdl_trigger();
  pdl_wait();
  const Segment sg = segment(rows, blockIdx.y);
  const int present = min(KVR_PAGE, len - sg.page * KVR_PAGE);
  const bool whole = sg.r1 - sg.r0 == KVR_PAGE;
  uint8_t *dst = v.block(l0 + l, g, sg.page);
  if (tid < KVR_PAGE) row_of[tid] = -1;
  if (!whole)
    for (int i = tid; i < 2 * HB / 16; i += NT) ((uint4 *)blk)[i] = ((const uint4 *)dst)[i];
  __syncthreads();
  for (int i = sg.r0 + tid; i < sg.r1; i += NT) row_of[position(rows, i) % KVR_PAGE] = i;
  __syncthreads();

  // four keys, eight entries a thread; the CH threads of a row are neighbours
  const int kg = tid / CH, ch = tid % CH;
  const uint32_t rowmask = (CH == 16 ? 0xFFFFu : 0xFFu) << (lane & ~(CH - 1));
  int rr[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) rr[j] = row_of[4 * kg + j];
  const bool any = rr[0] >= 0 || rr[1] >= 0 || rr[2] >= 0 || rr[3] >= 0;
  const bool all = rr[0] >= 0 && rr[1] >= 0 && rr[2] >= 0 && rr[3] >= 0;
  __half2 hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    hi[i] = __half2half2(__ushort_as_half(0xFC00));  // -inf
    lo[i] = __half2half2(__ushort_as_half(0x7C00));
  }
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const T *src = kv ? val : k;
    uint8_t *half = blk + kv * HB;
    uint32_t c[4] = {0, 0, 0, 0}, sc[4];
    float x[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (rr[j] >= 0) {
        Eight<T>::load(src + (((size_t)rr[j] * gridDim.z + l) * v.G + g) * DH + 8 * ch, x[j]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j][i] = 0.f;
      }
    if (!all) {
      if (kv)
        v_codes_load(half, kg, ch, c);
      else
        k_codes_load<DH>(half, kg, ch, c);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      int m = 0;  // largest magnitude's bits: infinities and NaN lie above all others
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, (int)(__float_as_uint(x[j][i]) & 0x7FFFFFFFu));
      const bool bad = (__ballot_sync(0xFFFFFFFFu, m >= 0x7F800000) & rowmask) != 0;
      m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
      const int at = kv ? pack_v_scale(DH, 4 * kg + j, ch >> 1)
                        : pack_k_scale(DH, 4 * kg + j, ch >> 1);
      if (rr[j] < 0) {
        sc[j] = half[at];
        continue;
      }
      sc[j] = bad ? PACK_NAN : pack_scale_code(__int_as_float(m));
      const float s = pack_scale(sc[j]), r = s > 0.f ? __frcp_rn(s) : 0.f;
      uint32_t w = 0;
      if (!bad && s > 0.f) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w |= pack_codes(Eight<T>::quotient(x[j][2 * i], s, r),
                          Eight<T>::quotient(x[j][2 * i + 1], s, r))
               << (8 * i);
      }
      c[j] = w;
      if (!(ch & 1)) half[at] = (uint8_t)sc[j];
    }
    if (any) {
      if (kv)
        v_codes_store(half, kg, ch, c);
      else
        k_codes_store<DH>(half, kg, ch, c);
    }
    if (!kv) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (4 * kg + j >= present || sc[j] == PACK_NAN) continue;
        __half2 y[4];
        eight_values(c[j], sc[j], y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          hi[i] = __hmax2(hi[i], y[i]);
          lo[i] = __hmin2(lo[i], y[i]);
        }
      }
    }
  }
  // bounds: over the key groups of the warp, then over the warps
#pragma unroll
  for (int i = 0; i < 4; ++i) {
#pragma unroll
    for (int o = CH; o < 32; o *= 2) {
      hi[i] = __hmax2(hi[i], __shfl_xor_sync(0xFFFFFFFFu, hi[i], o));
      lo[i] = __hmin2(lo[i], __shfl_xor_sync(0xFFFFFFFFu, lo[i], o));
    }
    if (lane < CH) {
      red[0][warp][4 * lane + i] = hi[i];
      red[1][warp][4 * lane + i] = lo[i];
    }
  }
  __syncthreads();
  float h = -INFINITY, b = INFINITY;
  if (tid < DH) {
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
      h = fmaxf(h, __half2float(((const __half *)red[0][w])[tid]));
      b = fminf(b, __half2float(((const __half *)red[1][w])[tid]));
    }
    if (h < b) h = b = 0.f;  // no finite row
    float a = fmaxf(fabsf(h), fabsf(b));
#pragma unroll
    for (int o = 16; o; o /= 2) a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
    if (lane == 0) amax[warp] = a;
  }
  for (int i = tid; i < 2 * HB / 16; i += NT) ((uint4 *)dst)[i] = ((const uint4 *)blk)[i];
  __syncthreads();
  if (tid < DH) {
    float a = amax[0];
#pragma unroll
    for (int w = 1; w < DH / 32; ++w) a = fmaxf(a, amax[w]);
    const float u = unit_of(a), r = __frcp_rn(u);  // powers of two: exact
    const size_t at = v.index(l0 + l, g, sg.page);
    v.bounds[at * 2 * DH + tid] = (int8_t)ceilf(h * r);
    v.bounds[at * 2 * DH + DH + tid] = (int8_t)floorf(b * r);
    if (tid == 0) v.unit[at] = u;
  }
}

// A CTA per (KV head, page, layer): the block into shared memory, the rows asked for out
// of it.
template <int DH, typename T>
__global__ void __launch_bounds__(2 * DH)
    k_packed_read(const PackedView v, const __grid_constant__ PackedRows rows, int l0, T *k,
                  T *val) {
  constexpr int NT = 2 * DH, CH = DH / 8, HB = pack_half_bytes(DH);
  __shared__ __align__(16) uint8_t blk[2 * HB];
  __shared__ int row_of[KVR_PAGE];
  const int tid = threadIdx.x, g = blockIdx.x, l = blockIdx.z;
  pdl_trigger();
  pdl_wait();
  const Segment sg = segment(rows, blockIdx.y);
  const uint8_t *src = v.block(l0 + l, g, sg.page);
  if (tid < KVR_PAGE) row_of[tid] = -1;
  for (int i = tid; i < 2 * HB / 16; i += NT) ((uint4 *)blk)[i] = ((const uint4 *)src)[i];
  __syncthreads();
  for (int i = sg.r0 + tid; i < sg.r1; i += NT) row_of[position(rows, i) % KVR_PAGE] = i;
  __syncthreads();
  const int kg = tid / CH, ch = tid % CH;
  int rr[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) rr[j] = row_of[4 * kg + j];
  if (rr[0] < 0 && rr[1] < 0 && rr[2] < 0 && rr[3] < 0) return;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const uint8_t *half = blk + kv * HB;
    T *dst = kv ? val : k;
    uint32_t c[4];
    if (kv)
      v_codes_load(half, kg, ch, c);
    else
      k_codes_load<DH>(half, kg, ch, c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (rr[j] < 0) continue;
      const int at = kv ? pack_v_scale(DH, 4 * kg + j, ch >> 1)
                        : pack_k_scale(DH, 4 * kg + j, ch >> 1);
      __half2 y[4];
      float x[8];
      eight_values(c[j], half[at], y);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(y[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
      }
      Eight<T>::store(dst + (((size_t)rr[j] * gridDim.z + l) * v.G + g) * DH + 8 * ch, x);
    }
  }
}

// What the attention of many rows reads, in halves (both exact).  Grid (G, pages + q's
// CTAs): a CTA per (KV head, page) widens the block into pages [page][K, V][G][KVR_PAGE][DH];
// the others take UNPACK_Q vectors (row, head) of q a warp, each divided by a power of two
// that brings its largest magnitude into [2^8, 2^9).
constexpr int UNPACK_Q = 4;
struct UnpackArgs {
  PackedView v;
  int layer, n_pages;
  __half *pages;
  const __nv_bfloat16 *q;
  int ldq, H, n_vec;
  __half *q_out;
  float *q_scale;
};
template <int DH>
__global__ void __launch_bounds__(2 * DH) k_packed_unpack(const UnpackArgs a) {
  constexpr int NT = 2 * DH, CH = DH / 8, HB = pack_half_bytes(DH), PER = DH / 32;
  __shared__ __align__(16) uint8_t blk[2 * HB];
  const int tid = threadIdx.x, g = blockIdx.x, page = blockIdx.y, G = gridDim.x;
  pdl_trigger();
  pdl_wait();
  if (page >= a.n_pages) {
    const int lane = tid & 31;
    const long long v0 = ((long long)((page - a.n_pages) * G + g) * (NT / 32) + (tid >> 5)) * UNPACK_Q;
    float x[UNPACK_Q][PER];
#pragma unroll
    for (int i = 0; i < UNPACK_Q; ++i) {
      const long long vec = min(v0 + i, (long long)a.n_vec - 1), row = vec / a.H;
      const __nv_bfloat16 *src = a.q + row * a.ldq + (vec - row * a.H) * DH + PER * lane;
#pragma unroll
      for (int j = 0; j < PER; ++j) x[i][j] = __bfloat162float(src[j]);
    }
#pragma unroll
    for (int i = 0; i < UNPACK_Q; ++i) {
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < PER; ++j) m = fmaxf(m, fabsf(x[i][j]));
#pragma unroll
      for (int o = 16; o; o /= 2) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
      const int e = pack_q_exponent(m);
      const float down = pack_exp2(-e);
      if (v0 + i >= a.n_vec) break;
      __half *dst = a.q_out + (v0 + i) * DH + PER * lane;
#pragma unroll
      for (int j = 0; j < PER; ++j) dst[j] = __float2half_rn(x[i][j] * down);
      if (lane == 0) a.q_scale[v0 + i] = pack_exp2(e);
    }
    return;
  }
  const uint8_t *src = a.v.block(a.layer, g, page);
  for (int i = tid; i < 2 * HB / 16; i += NT) ((uint4 *)blk)[i] = ((const uint4 *)src)[i];
  __syncthreads();
  const int kg = tid / CH, ch = tid % CH;
  bool bad[4];  // any scale of a row tells
#pragma unroll
  for (int j = 0; j < 4; ++j)
    bad[j] = blk[pack_k_scale(DH, 4 * kg + j, 0)] == PACK_NAN ||
             blk[HB + pack_v_scale(DH, 4 * kg + j, 0)] == PACK_NAN;
#pragma unroll
  for (int kv = 0; kv < 2; ++kv) {
    const uint8_t *half = blk + kv * HB;
    uint32_t c[4];
    if (kv)
      v_codes_load(half, kg, ch, c);
    else
      k_codes_load<DH>(half, kg, ch, c);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = kv ? pack_v_scale(DH, 4 * kg + j, ch >> 1)
                        : pack_k_scale(DH, 4 * kg + j, ch >> 1);
      __align__(16) __half2 y[4];
      eight_values(c[j], bad[j] ? (kv ? 0 : PACK_NAN) : half[at], y);
      *(uint4 *)(a.pages + ((((size_t)page * 2 + kv) * G + g) * KVR_PAGE + 4 * kg + j) * DH +
                 8 * ch) = *(const uint4 *)y;
    }
  }
}

// ------------------------------------------------------------ block selection

// A CTA per (row, KV head): P_c = sum over the group's heads of max(q, 0), N_c that of
// min(q, 0) (in head order), both in 8 bits of a common power of two; a block's
// score is u sum_c (P_c hi_c + N_c lo_c), an upper bound (up to the roundings) of the
// sum of the heads' largest products with a key of the block.  The sum is of whole
// numbers below 2^23 and u a power of two, so a score is exact and does not depend on the
// order of its sum.  The row's own block is always taken; of the earlier ones those with
// the highest scores, ties to the lowest.
constexpr int SEL_THREADS = 256;
template <int DH, typename T>
__global__ void __launch_bounds__(SEL_THREADS)
    k_packed_select(const T *q, int ldq, const PackedRow *rows, int layer, int grp, int count,
                    int32_t *blocks) {
  extern __shared__ uint32_t keys[];  // ordered scores of the blocks before the own
  __shared__ __align__(16) int8_t qs[2][DH];
  __shared__ float amax[DH / 32];
  __shared__ int tot[SEL_THREADS / 32][2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x, g = blockIdx.y, G = gridDim.y;
  pdl_trigger();
  pdl_wait();
  const int pos = rows[row].pos;
  int32_t *out = blocks + ((size_t)row * G + g) * count;
  if (pos < 0) {
    for (int i = tid; i < count; i += SEL_THREADS) out[i] = -1;
    return;
  }
  const PackedView v = rows[row].doc;
  const int own = pos / KVR_PAGE;
  if (own + 1 <= count) {  // every block that the row sees
    for (int i = tid; i < count; i += SEL_THREADS) out[i] = i <= own ? i : -1;
    return;
  }
  float up = 0.f, down = 0.f;
  if (tid < DH) {
    const T *x = q + (size_t)row * ldq + (size_t)g * grp * DH + tid;
    for (int h = 0; h < grp; ++h) {
      const float f = (float)x[h * DH];
      up = __fadd_rn(up, f > 0.f ? f : f != f ? f : 0.f);
      down = __fadd_rn(down, f < 0.f ? f : 0.f);
    }
    float a = fmaxf(up, -down);
    if (up != up || down != down) a = INFINITY;
#pragma unroll
    for (int o = 16; o; o /= 2) a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
    if (lane == 0) amax[warp] = a;
  }
  __syncthreads();
  if (tid < DH) {
    float a = amax[0];
#pragma unroll
    for (int w = 1; w < DH / 32; ++w) a = fmaxf(a, amax[w]);
    // queries that are not finite score nothing: the lowest blocks are taken
    const float r = a < INFINITY ? __frcp_rn(unit_of(a)) : 0.f;
    qs[0][tid] = a < INFINITY ? (int8_t)__float2int_rn(up * r) : 0;
    qs[1][tid] = a < INFINITY ? (int8_t)__float2int_rn(down * r) : 0;
  }
  __syncthreads();
  const size_t at = v.index(layer, g, 0);
  for (int b = tid; b < own; b += SEL_THREADS) {
    const int4 *w = (const int4 *)(v.bounds + (at + b) * 2 * DH);
    const int4 *x = (const int4 *)qs;
    int s = 0;
#pragma unroll
    for (int i = 0; i < 2 * DH / 16; ++i) {
      const int4 a = w[i], c = x[i];
      s = __dp4a(a.x, c.x, s);
      s = __dp4a(a.y, c.y, s);
      s = __dp4a(a.z, c.z, s);
      s = __dp4a(a.w, c.w, s);
    }
    const float f = (float)s * v.unit[at + b];
    const uint32_t u = __float_as_uint(f == 0.f ? 0.f : f);
    keys[b] = u >> 31 ? ~u : u | 0x80000000u;
  }
  __syncthreads();
  // the (count - 1)-th largest key, bit by bit: the largest t with at least that many >= t
  const int want = count - 1;
  uint32_t t = 0;
  for (int bit = 31; bit >= 0 && want > 0; --bit) {
    const uint32_t c = t | 1u << bit;
    int n = 0;
    for (int b = tid; b < own; b += SEL_THREADS) n += keys[b] >= c;
    n = __reduce_add_sync(0xFFFFFFFFu, n);
    if (lane == 0) tot[warp][bit & 1] = n;
    __syncthreads();
    n = 0;
#pragma unroll
    for (int w = 0; w < SEL_THREADS / 32; ++w) n += tot[w][bit & 1];
    if (n >= want) t = c;
  }
  // in order: keys above t, and as many of those equal to it as are wanted
  if (warp == 0) {
    int above = 0;
    for (int b = lane; b < own; b += 32) above += keys[b] > t;
    above = __reduce_add_sync(0xFFFFFFFFu, above);
    int ties = want - above, n = 0;
    for (int b0 = 0; b0 < own && n < want; b0 += 32) {
      const uint32_t kx = b0 + lane < own ? keys[b0 + lane] : 0;
      const uint32_t gt = __ballot_sync(0xFFFFFFFFu, b0 + lane < own && kx > t);
      uint32_t eq = __ballot_sync(0xFFFFFFFFu, b0 + lane < own && kx == t);
      const uint32_t below = (1u << lane) - 1;
      const bool take = (gt >> lane & 1) || ((eq >> lane & 1) && __popc(eq & below) < ties);
      const uint32_t took = __ballot_sync(0xFFFFFFFFu, take);
      if (take) out[n + __popc(took & below)] = b0 + lane;
      n += __popc(took);
      ties -= min(ties, __popc(eq));
    }
    if (lane == 0) out[want] = own;
  }
}

PerDevice<size_t> sel_smem[4];

}  // namespace

void launch_packed_write(const PackedView &v, int dtype, const PackedRows &rows, int len, int l0,
                         int nl, const void *k, const void *val, cudaStream_t s) {
  const dim3 grid(v.G, rows.n_seg, nl);
  auto run = [&](auto kernel, auto *kk, auto *vv) {
    launch_pdl(kernel, grid, dim3(2 * v.dh), 0, s, v, rows, len, l0, kk, vv);
  };
  if (dtype == KVR_DTYPE_BF16) {
    using T = __nv_bfloat16;
    run(v.dh == 128 ? k_packed_write<128, T> : k_packed_write<64, T>, (const T *)k, (const T *)val);
  } else {
    run(v.dh == 128 ? k_packed_write<128, float> : k_packed_write<64, float>, (const float *)k,
        (const float *)val);
  }
}

void launch_packed_read(const PackedView &v, int dtype, const PackedRows &rows, int l0, int nl,
                        void *k, void *val, cudaStream_t s) {
  const dim3 grid(v.G, rows.n_seg, nl);
  auto run = [&](auto kernel, auto *kk, auto *vv) {
    launch_pdl(kernel, grid, dim3(2 * v.dh), 0, s, v, rows, l0, kk, vv);
  };
  if (dtype == KVR_DTYPE_BF16) {
    using T = __nv_bfloat16;
    run(v.dh == 128 ? k_packed_read<128, T> : k_packed_read<64, T>, (T *)k, (T *)val);
  } else {
    run(v.dh == 128 ? k_packed_read<128, float> : k_packed_read<64, float>, (float *)k,
        (float *)val);
  }
}

void launch_packed_unpack(const PackedView &v, int layer, int n_pages, void *pages, const void *q,
                          int ldq, int H, int rows, void *q_out, float *q_scale, bool settled,
                          cudaStream_t s) {
  auto *kernel = v.dh == 128 ? k_packed_unpack<128> : k_packed_unpack<64>;
  const int per = v.G * (2 * v.dh / 32) * UNPACK_Q;  // vectors of a line of CTAs
  const dim3 grid(v.G, n_pages + (rows * H + per - 1) / per);
  const UnpackArgs a{v, layer, n_pages, (__half *)pages, (const __nv_bfloat16 *)q, ldq, H, rows * H,
                     (__half *)q_out, q_scale};
  if (settled)
    launch_pdl(kernel, grid, dim3(2 * v.dh), 0, s, a);
  else
    kernel<<<grid, 2 * v.dh, 0, s>>>(a);
}

const char *launch_packed_select(const PackedAttnArgs &a, int max_pages, int32_t *blocks,
                                 cudaStream_t s) {
  const size_t smem = (size_t)max_pages * sizeof(uint32_t);
  const dim3 grid(a.n_rows, a.G);
  auto run = [&](auto kernel, auto *q, int which) -> const char * {
    if (smem > 40 * 1024)
      if (const char *e = smem_opt_in(sel_smem[which], kernel, smem)) return e;
    const cudaError_t e =
        launch_pdl(kernel, grid, dim3(SEL_THREADS), smem, s, q, a.ldq, a.rows, a.layer, a.grp,
                   a.n_blocks, blocks);
    return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
  };
  if (a.dtype == KVR_DTYPE_BF16) {
    auto *q = (const __nv_bfloat16 *)a.q;
    return a.dh == 128 ? run(k_packed_select<128, __nv_bfloat16>, q, 0)
                       : run(k_packed_select<64, __nv_bfloat16>, q, 1);
  }
  auto *q = (const float *)a.q;
  return a.dh == 128 ? run(k_packed_select<128, float>, q, 2)
                     : run(k_packed_select<64, float>, q, 3);
}

}  // namespace kvr
