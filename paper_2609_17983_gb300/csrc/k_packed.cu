// k_packed.cu -- the packed cache's rows and blocks: quantising K/V rows as they are
// written, reading them back, and selecting blocks by their bounds.
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "packed.cuh"

namespace kvr {
namespace {

// The rows [r0, r1) of segment seg and their page; the row of a slot of it, or -1.
struct Segment {
  int page, r0, r1;
};
__device__ __forceinline__ int position(const PackedRun &r, int i) { return r.pos_d[i]; }
__device__ __forceinline__ int position(const PackedList &r, int i) { return r.pos[i]; }
__device__ __forceinline__ int start(const PackedRun &r, int s) { return r.pos_d[r.n + s]; }
__device__ __forceinline__ int start(const PackedList &r, int s) { return r.seg[s]; }
template <class Rows>
__device__ __forceinline__ Segment segment(const Rows &r, int seg) {
  Segment s;
  if (r.first >= 0) {
    s.page = r.first / KVR_PAGE + seg;
    s.r0 = max(0, s.page * KVR_PAGE - r.first);
    s.r1 = min(r.n, (s.page + 1) * KVR_PAGE - r.first);
    return s;
  }
  s.r0 = start(r, seg);
  s.r1 = start(r, seg + 1);
  s.page = position(r, s.r0) / KVR_PAGE;
  return s;
}
// Rows of the slots 4 kg .. 4 kg + 3 (every thread of the CTA calls it; row_of: shared
// [KVR_PAGE], used for lists).
template <class Rows>
__device__ __forceinline__ void rows_of_slots(const Rows &r, const Segment &s, int *row_of, int kg,
                                              int *rr) {
  if (r.first >= 0) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = s.page * KVR_PAGE + 4 * kg + j - r.first;
      rr[j] = i >= s.r0 && i < s.r1 ? i : -1;
    }
    return;
  }
  if (threadIdx.x < KVR_PAGE) row_of[threadIdx.x] = -1;
  __syncthreads();
  for (int i = s.r0 + threadIdx.x; i < s.r1; i += blockDim.x)
    row_of[position(r, i) % KVR_PAGE] = i;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < 4; ++j) rr[j] = row_of[4 * kg + j];
}

// The larger of two unsigned 16-bit numbers, twice.
__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Eight entries of a row: loaded, the bits of their largest magnitude as a float
// (infinities and NaN lie above all others), a group's scale, the codes under a
// scale s.
template <typename T>
struct Eight;
template <>
struct Eight<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void load(const __nv_bfloat16 *p) { u = __ldcs((const uint4 *)p); }
  // largest magnitudes of the even entries (low half) and of the odd ones
  __device__ __forceinline__ uint32_t magnitudes() const {
    return max_u16x2(max_u16x2(u.x & 0x7FFF7FFFu, u.y & 0x7FFF7FFFu),
                     max_u16x2(u.z & 0x7FFF7FFFu, u.w & 0x7FFF7FFFu));
  }
  __device__ __forceinline__ uint32_t magnitude() const {
    const uint32_t m = magnitudes();
    return max(m & 0xFFFF0000u, m << 16);
  }
  static __device__ __forceinline__ uint32_t scale_code(float a) { return pack_scale_code_bf16(a); }
  // x / s on the grid of the codes.  With r a reciprocal of the four-bit s, off by 2^-22
  // at most, x r + 768 rounds to whole steps of 2^-14, far above r's error and far below
  // the distance of an eight-bit x from a midpoint of the codes (at least 2^-10 where it
  // is not one), so ties are ties and everything else keeps its side.
  __device__ __forceinline__ uint32_t codes(float s) const {
    float r, y[8];
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      asm("{\n\t.reg .b64 x, r, c, d;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 r, {%4, %4};\n\t"
          "mov.b64 c, {%5, %5};\n\tmov.b64 d, {%6, %6};\n\tfma.rn.f32x2 x, x, r, c;\n\t"
          "add.rn.f32x2 x, x, d;\n\tmov.b64 {%0, %1}, x;\n\t}"
          : "=f"(y[2 * i]), "=f"(y[2 * i + 1])
          : "r"(w[i] << 16), "r"(w[i] & 0xFFFF0000u), "f"(r), "f"(768.f), "f"(-768.f));
    return pack_codes(y);
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
};
template <>
struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float *p) {
    a = __ldcs((const float4 *)p);
    b = __ldcs((const float4 *)p + 1);
  }
  __device__ __forceinline__ uint32_t magnitude() const {
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    return m;
  }
  static __device__ __forceinline__ uint32_t scale_code(float x) { return pack_scale_code(x); }
  // As above, but a 24-bit x may lie nearer to a midpoint than a step of 2^-14: where x r + 768
  // is a multiple of a quarter, as every midpoint is, the entries are divided.
  __device__ __forceinline__ uint32_t codes(float s) const {
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    float r, y[8];
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    uint32_t near = 0xFFFu;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float f = __fmaf_rn(x[i], r, 768.f);
      near = min(near, __float_as_uint(f) & 0xFFFu);
      y[i] = __fadd_rn(f, -768.f);
    }
    if (near == 0)
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = __fdiv_rn(x[i], s);
    return pack_codes(y);
  }
  static __device__ __forceinline__ void store(float *p, const float *x) {
    __stcs((float4 *)p, make_float4(x[0], x[1], x[2], x[3]));
    __stcs((float4 *)p + 1, make_float4(x[4], x[5], x[6], x[7]));
  }
};

// Scale code of a row's group, as this thread's eight entries and its neighbour's (lane ^ 1)
// make it up; rows with a NaN or an infinity anywhere (rowmask: the lanes of a row) get
// PACK_NAN.
template <typename T>
__device__ __forceinline__ uint32_t scale_code(const Eight<T> &x, uint32_t rowmask) {
  uint32_t m = x.magnitude();
  const bool bad = (__ballot_sync(0xFFFFFFFFu, m >= 0x7F800000u) & rowmask) != 0;
  m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
  return bad ? PACK_NAN : Eight<T>::scale_code(__uint_as_float(m));
}
// Those of N rows.
template <int N>
__device__ __forceinline__ void scale_codes(const Eight<float> *x, uint32_t rowmask, uint32_t *sc) {
#pragma unroll
  for (int j = 0; j < N; ++j) sc[j] = scale_code(x[j], rowmask);
}
// Two bf16 rows at a time: their magnitudes, halves of the sixths and codes in the 16-bit
// halves of one register each (see pack_scale_code_bf16).
template <int N>
__device__ __forceinline__ void scale_codes(const Eight<__nv_bfloat16> *x, uint32_t rowmask,
                                            uint32_t *sc) {
  uint32_t m[N / 2], worst = 0, least = 0xFFFFFFFFu;
#pragma unroll
  for (int j = 0; j < N / 2; ++j) {
    const uint32_t a = x[2 * j].magnitudes(), b = x[2 * j + 1].magnitudes();
    m[j] = max_u16x2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632));
    worst = max_u16x2(worst, m[j]);
    m[j] = max_u16x2(m[j], __shfl_xor_sync(0xFFFFFFFFu, m[j], 1));
    least = __vminu2(least, m[j]);
#pragma unroll
    for (int h = 0; h < 2; ++h) sc[2 * j + h] = 0;
    const __half2 s = __floats2half2_rn(__uint_as_float(m[j] << 16) * (1.f / 6.f),
                                        __uint_as_float(m[j] & 0xFFFF0000u) * (1.f / 6.f));
    const uint32_t u = *(const uint32_t *)&s;
    const uint32_t c = __vminu2((u + 0x003F003Fu + (u >> 7 & 0x00010001u)) >> 7 & 0x01FF01FFu,
                                PACK_MAX_CODE * 0x00010001u);
    sc[2 * j] = c & 0xFFFFu;
    sc[2 * j + 1] = c >> 16;
  }
  // anything not finite, or below 6 * 2^-14 (bf16 bits 0x39C0): rare
  const bool odd = (worst & 0xFFFFu) >= 0x7F80u || worst >> 16 >= 0x7F80u ||
                   (least & 0xFFFFu) < 0x39C0u || least >> 16 < 0x39C0u;
  if (__any_sync(0xFFFFFFFFu, odd)) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t own = x[j].magnitude();
      const bool bad = (__ballot_sync(0xFFFFFFFFu, own >= 0x7F800000u) & rowmask) != 0;
      const uint32_t g = j & 1 ? m[j / 2] & 0xFFFF0000u : m[j / 2] << 16;
      sc[j] = bad ? PACK_NAN : pack_scale_code_bf16(__uint_as_float(g));
    }
  }
}

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
// V: the nibbles of four keys' words and of eight entries' half-words are each other's
// transpose (h: entries 0 and 2, 4 and 6, 1 and 3, 5 and 7).
__device__ __forceinline__ void transpose_out(const uint32_t *c, uint32_t *h) {
  constexpr uint32_t M = 0x0F0F0F0Fu;
  const uint32_t a0 = (c[0] & M) | (c[1] << 4 & ~M), a1 = (c[0] >> 4 & M) | (c[1] & ~M);
  const uint32_t b0 = (c[2] & M) | (c[3] << 4 & ~M), b1 = (c[2] >> 4 & M) | (c[3] & ~M);
  h[0] = __byte_perm(a0, b0, 0x5140);
  h[1] = __byte_perm(a0, b0, 0x7362);
  h[2] = __byte_perm(a1, b1, 0x5140);
  h[3] = __byte_perm(a1, b1, 0x7362);
}
__device__ __forceinline__ void transpose_in(const uint32_t *h, uint32_t *c) {
  constexpr uint32_t M = 0x0F0F0F0Fu;
  const uint32_t a0 = __byte_perm(h[0], h[1], 0x6420), b0 = __byte_perm(h[0], h[1], 0x7531);
  const uint32_t a1 = __byte_perm(h[2], h[3], 0x6420), b1 = __byte_perm(h[2], h[3], 0x7531);
  c[0] = (a0 & M) | (a1 << 4 & ~M);
  c[1] = (a0 >> 4 & M) | (a1 & ~M);
  c[2] = (b0 & M) | (b1 << 4 & ~M);
  c[3] = (b0 >> 4 & M) | (b1 & ~M);
}
__device__ __forceinline__ void v_codes_load(const uint8_t *half, int kg, int ch, uint32_t *c) {
  uint32_t e[8], h[4];
#pragma unroll
  for (int i = 0; i < 8; ++i) e[i] = *(const uint16_t *)(half + pack_v_code(kg, 8 * ch + i));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = (i & 1) * 4 + (i >> 1);
    h[i] = e[x] | e[x + 2] << 16;
  }
  transpose_in(h, c);
}
__device__ __forceinline__ uint32_t bits(__half2 x) { return *(const uint32_t *)&x; }
__device__ __forceinline__ __half2 half2_of(uint32_t x) { return *(const __half2 *)&x; }

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

// Bounds of the keys of a block, over the finite rows of the slots below `present`, by the
// first DH / 64 warps of the CTA: warp d4 holds its db's 4 d4 .. + 3, a thread four
// entries of two keys of each of the four key tiles (w: codes, sc: the keys' scales).
// What is left is over the eight lanes of a column: each exchange halves what a lane
// goes on with.  (By all eight warps, a key tile each, the exchanges alone cost as much
// as all the rest.)
template <int DH>
__device__ __forceinline__ void block_bounds(float *amax, const uint32_t (*w)[4],
                                             const uint32_t (*sc)[2], int present, int8_t *bounds,
                                             float *unit) {
  const int lane = threadIdx.x & 31, d4 = threadIdx.x / 32, lg = lane >> 2, lt = lane & 3;
  __half2 hi[8], lo[8];  // [db of the four][entries 4 lt, 4 lt + 2]
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    hi[i] = __half2half2(__ushort_as_half(0xFC00));  // -inf
    lo[i] = __half2half2(__ushort_as_half(0x7C00));
  }
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
    uint32_t v[4][4];
#pragma unroll
    for (int b = 0; b < 4; ++b) pack_values(w[kt][b], v[b]);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // all scales of a row marked NaN are
      if (16 * kt + pack_key_of(lg) + 2 * h >= present || (sc[kt][h] & 0xFF) == PACK_NAN) continue;
      const uint32_t s01 = __byte_perm(sc[kt][h], 0, 0x4140) << 7,
                     s23 = __byte_perm(sc[kt][h], 0, 0x4342) << 7;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const __half2 two = half2_of(b < 2 ? s01 : s23);
        const __half2 s2 = b & 1 ? __high2half2(two) : __low2half2(two);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const __half2 y = __hmul2(*(const __half2 *)&v[b][2 * h + x], s2);
          hi[2 * b + x] = __hmax2(hi[2 * b + x], y);
          lo[2 * b + x] = __hmin2(lo[2 * b + x], y);
        }
      }
    }
  }
  // lanes apart by 16, 8, 4: each keeps the half of its entries that its bit of lg names
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    const int n = 4 >> k, o = 16 >> k;
    const bool upper = lane & o;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      // (of the registers, not of the half2s: choosing between those is choosing between
      // addresses, and takes the arrays to local memory)
      const uint32_t h0 = bits(hi[i]), h1 = bits(hi[i + n]), l0 = bits(lo[i]), l1 = bits(lo[i + n]);
      const uint32_t sh = __shfl_xor_sync(0xFFFFFFFFu, upper ? h0 : h1, o),
                     sl = __shfl_xor_sync(0xFFFFFFFFu, upper ? l0 : l1, o);
      hi[i] = __hmax2(half2_of(upper ? h1 : h0), half2_of(sh));
      lo[i] = __hmin2(half2_of(upper ? l1 : l0), half2_of(sl));
    }
  }
  // lane (lg, lt) holds db 4 d4 + lg / 2, entries 4 lt + 2 (lg & 1) and the next
  const int at = 16 * (4 * d4 + (lg >> 1)) + 4 * lt + 2 * (lg & 1);
  float2 h = __half22float2(hi[0]), l = __half22float2(lo[0]);
  if (h.x < l.x) h = l = make_float2(0.f, 0.f);  // no finite row
  float a = fmaxf(fmaxf(fabsf(h.x), fabsf(h.y)), fmaxf(fabsf(l.x), fabsf(l.y)));
#pragma unroll
  for (int o = 16; o; o /= 2) a = fmaxf(a, __shfl_xor_sync(0xFFFFFFFFu, a, o));
  if (DH > 64) {
    if (lane == 0) amax[d4] = a;
    asm volatile("bar.sync 1, %0;" ::"n"(DH / 2) : "memory");
#pragma unroll
    for (int i = 0; i < DH / 64; ++i) a = fmaxf(a, amax[i]);
  }
  const float u = unit_of(a), r = __frcp_rn(u);  // powers of two: exact
  auto pair = [](float x, float y) { return (uint16_t)((int)x & 0xFF | (int)y << 8); };
  *(uint16_t *)(bounds + at) = pair(ceilf(h.x * r), ceilf(h.y * r));
  *(uint16_t *)(bounds + DH + at) = pair(floorf(l.x * r), floorf(l.y * r));
  if (threadIdx.x == 0) *unit = u;
}
// The same from a K half in memory.
template <int DH>
__device__ __forceinline__ void block_bounds(float *amax, const uint8_t *kb, int present,
                                             int8_t *bounds, float *unit) {
  const int lane = threadIdx.x & 31, d4 = threadIdx.x / 32;
  uint32_t w[4][4], sc[4][2];
#pragma unroll
  for (int kt = 0; kt < 4; ++kt) {
    const uint4 x = *(const uint4 *)(kb + ((kt * (DH / 64) + d4) * 32 + lane) * 16);
    w[kt][0] = x.x, w[kt][1] = x.y, w[kt][2] = x.z, w[kt][3] = x.w;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      sc[kt][h] = *(const uint32_t *)(kb + pack_code_bytes(DH) +
                                      ((kt * 8 + (lane >> 2)) * 2 + h) * (DH / 16) + 4 * d4);
  }
  block_bounds<DH>(amax, w, sc, present, bounds, unit);
}

// Pages of n consecutive positions from the start of page0 (the last page may end early: the
// document ends there, and the slots behind stay zero): a CTA per (KV head, page, layer)
// quantises the page's rows into shared memory (four keys, eight entries of K and of V a
// thread), takes the bounds from there, and stores the block as it lies there.  By its
// bytes it should be bound by HBM (5000 rows of 32 layers, 655 MB in, 184 MB out: 124 us
// at the copy rate); its instructions come close (1443 a warp at first, 280 us): hence two
// rows' scales in one register, packed fp32 pairs, addresses that differ by constants,
// and bounds by two of the eight warps.  147 us, 5.7 TB/s.
template <int DH, typename T>
__global__ void __launch_bounds__(2 * DH, sizeof(T) == 2 ? 512 / DH : 256 / DH)
    k_packed_write_pages(const PackedView v, int page0, int n, int l0, const T *k, const T *val) {
  constexpr int NT = 2 * DH, CH = DH / 8, HB = pack_half_bytes(DH);
  __shared__ __align__(16) uint8_t blk[2 * HB];
  __shared__ float amax[2];
  const int tid = threadIdx.x, lane = tid & 31;
  const int g = blockIdx.x, l = blockIdx.z, page = page0 + blockIdx.y;
  pdl_trigger();
  pdl_wait();
  const int kg = tid / CH, ch = tid % CH;  // the CH threads of a row are neighbours
  const uint32_t rowmask = (CH == 16 ? 0xFFFFu : 0xFFu) << (lane & ~(CH - 1));
  const size_t row = (size_t)gridDim.z * v.G * DH;
  const size_t src = ((size_t)(KVR_PAGE * blockIdx.y + 4 * kg) * gridDim.z + l) * v.G * DH +
                     (size_t)g * DH + 8 * ch;
  const int present = min(KVR_PAGE, n - KVR_PAGE * (int)blockIdx.y);
  Eight<T> x[8];  // K's four rows, V's four
  if (present == KVR_PAGE) {
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j].load(k + src + j * row);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[4 + j].load(val + src + j * row);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = x[4 + j] = Eight<T>{};
      if (4 * kg + j < present) {
        x[j].load(k + src + j * row);
        x[4 + j].load(val + src + j * row);
      }
    }
  }
  uint32_t sc[8], c[8];
  scale_codes<8>(x, rowmask, sc);
#pragma unroll
  for (int j = 0; j < 8; ++j)
    c[j] = sc[j] == 0 || sc[j] == PACK_NAN ? 0 : x[j].codes(pack_scale(sc[j]));
  // K: words of keys j and j + 2 lie 64 bytes on for the next j, 16 for four more entries
  uint8_t *kb = blk, *vb = blk + HB;
  uint32_t *kw = (uint32_t *)(kb + pack_k_code(DH, 4 * kg, 8 * ch));
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    kw[16 * j] = __byte_perm(c[j], c[j + 2], 0x5410);
    kw[16 * j + 4] = __byte_perm(c[j], c[j + 2], 0x7632);
  }
  // V: entry i's half-word lies 64 (i ^ db / 4) bytes on
  uint32_t h[4];
  transpose_out(c + 4, h);
  const int flip = ch >> 3;
  uint8_t *v0 = vb + pack_v_code(kg, 8 * ch) - 64 * flip;  // of i = 0 where db < 4
  uint16_t *ve = (uint16_t *)(v0 + 64 * flip), *vo = (uint16_t *)(v0 - 64 * flip);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = (i & 1) * 4 + (i >> 1);  // entries e and e + 2: both even or both odd
    uint16_t *at = (e & 1) ? vo : ve;
    at[32 * e] = (uint16_t)h[i];
    at[32 * (e + 2)] = (uint16_t)(h[i] >> 16);
  }
  if (!(ch & 1)) {
    uint8_t *ks = kb + pack_k_scale(DH, 4 * kg, ch >> 1);
    ks[0] = (uint8_t)sc[0];  // keys 0 and 2 of the four, 1 and 3
    ks[DH / 16] = (uint8_t)sc[2];
    ks[2 * (DH / 16)] = (uint8_t)sc[1];
    ks[3 * (DH / 16)] = (uint8_t)sc[3];
    *(uint32_t *)(vb + pack_v_scale(DH, 4 * kg, ch >> 1)) =
        sc[4] | sc[5] << 8 | sc[6] << 16 | sc[7] << 24;
  }
  __syncthreads();
  uint4 *dst = (uint4 *)v.block(l0 + l, g, page);
  for (int i = tid; i < 2 * HB / 16; i += NT) dst[i] = ((const uint4 *)blk)[i];
  if (tid >= DH / 2) return;
  const size_t at = v.index(l0 + l, g, page);
  block_bounds<DH>(amax, kb, present, v.bounds + at * 2 * DH, v.unit + at);
}

// The bounds of a page alone, of the layers but [l0, l1).  Grid (G, layers), DH / 2 threads.
template <int DH>
__global__ void __launch_bounds__(DH / 2)
    k_packed_bounds(const PackedView v, int page, int present, int l0, int l1) {
  __shared__ float amax[2];
  pdl_trigger();
  pdl_wait();
  const int g = blockIdx.x, l = (int)blockIdx.y < l0 ? blockIdx.y : blockIdx.y + l1 - l0;
  const size_t at = v.index(l, g, page);
  block_bounds<DH>(amax, v.block(l, g, page), present, v.bounds + at * 2 * DH, v.unit + at);
}

// The slots of positions from `len` on, in the pages from its own, as if nothing had been
// written there: zeros, and the bounds over the slots before.  Grid (G, pages, layers),
// 2 DH threads.
template <int DH>
__global__ void __launch_bounds__(2 * DH) k_packed_clear(const PackedView v, int len) {
  constexpr int NT = 2 * DH, DB = DH / 16, DQ = DH / 64, CB = pack_code_bytes(DH),
                HB = pack_half_bytes(DH);
  __shared__ float amax[2];
  pdl_trigger();
  pdl_wait();
  const int g = blockIdx.x, l = blockIdx.z, page = len / KVR_PAGE + blockIdx.y;
  const int present = max(0, len - page * KVR_PAGE);
  uint8_t *kb = v.block(l, g, page), *vb = kb + HB;
  for (int i = threadIdx.x; i < CB / 4; i += NT) {
    // K: [kt][db / 4][lane][db % 4], a key in each half of a word
    const int key = 16 * (i / (128 * DQ)) + pack_key_of((i / 4 & 31) >> 2);
    uint32_t *w = (uint32_t *)kb + i;
    if (key >= present)
      *w = 0;
    else if (key + 2 >= present)
      *w &= 0xFFFFu;
    // V: [db][lane ^ db][kt], four keys in each half
    const int key4 = 16 * (i & 3) + 4 * (((i / 4 & 31) ^ i / 128) & 3);
    const int keep = min(4, max(0, present - key4));
    ((uint32_t *)vb)[i] &= ((1u << (4 * keep)) - 1) * 0x00010001u;
  }
  for (int i = threadIdx.x; i < KVR_PAGE * DB; i += NT) {
    const int key = i / DB, db = i % DB;
    if (key >= present) kb[pack_k_scale(DH, key, db)] = vb[pack_v_scale(DH, key, db)] = 0;
  }
  __syncthreads();
  if (threadIdx.x >= DH / 2) return;
  const size_t at = v.index(l, g, page);
  block_bounds<DH>(amax, kb, present, v.bounds + at * 2 * DH, v.unit + at);
}

// The units of blocks of zeros.
__global__ void k_packed_units(float *unit, size_t n) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) unit[i] = unit_of(0.f);
}

// Pages that a call writes in part: a CTA per (KV head, page, layer).  The new rows are
// quantised, K and V side by side in a warp, into shared memory, while the block's K
// codes are on their way to registers and so are the V codes of the first groups of four
// keys that change; words with a new key are patched and stored, and the bounds taken
// over all rows present.  NT: 2 DH threads, of which a group's V takes DH / 8, who turn four
// rows' codes at once; or DH / 2 (the bounds' warps alone, whose registers then hold all
// they need), which take the rows one after another but four times as many blocks at once.
// few_rows chooses; 28 layers, 4 KV heads, us by DH / 2 and by 2 DH threads:
//   pages               3 rows of 1   3 of 10   12 of 10   12 of 40   32 of 10
//   DH / 2 | 2 DH         4.5 | 3.9   7.4 | 8.5   13.9 | 11.2   27.8 | 36.2   23.4 | 13.5
// (a row of each of 40 pages 11.7 | 25.3).  which: the segments of a run that are not whole
// pages (a list's are blockIdx.y).
constexpr int PATCH_FEW = 32;
template <int DH, typename T, class Rows, int NT>
__global__ void __launch_bounds__(NT, (sizeof(T) == 2 ? 1024 : 768) / NT)
    k_packed_patch(const PackedView v, const __grid_constant__ Rows rows, int2 which, int len,
                   int l0, const T *k, const T *val) {
  constexpr int CH = DH / 8, DB = DH / 16, DQ = DH / 64, HB = pack_half_bytes(DH),
                CB = pack_code_bytes(DH), WARPS = NT / 32,
                KPT = 2 * DH / NT;  // 16-byte pieces of K a thread
  constexpr bool FEW = KPT == 4;
  constexpr int ROWS = FEW ? PATCH_FEW : KVR_PAGE;  // rows in shared memory
  // groups of V at a time, and a thread's words of each: entries vi .. and the eighth past each
  constexpr int VG = FEW ? 1 : NT / CH, VW = FEW ? 1 : 4;
  __shared__ float amax[2];
  __shared__ __align__(16) uint32_t code[ROWS][2][CH];
  __shared__ __align__(8) uint8_t scale[ROWS][2][DB];
  __shared__ __align__(4) uint8_t row_at[KVR_PAGE];  // of a slot that is written
  __shared__ __align__(16) uint8_t kbuf[FEW ? 16 : HB];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, lg = lane >> 2, lt = lane & 3;
  const int g = blockIdx.x, l = blockIdx.z;
  pdl_trigger();
  pdl_wait();
  const Segment sg = segment(rows, rows.first < 0 ? blockIdx.y : blockIdx.y ? which.y : which.x);
  const int present = min(KVR_PAGE, len - sg.page * KVR_PAGE), count = sg.r1 - sg.r0;
  auto slot_of = [&](int i) {
    return (rows.first >= 0 ? rows.first + sg.r0 + i : position(rows, sg.r0 + i)) % KVR_PAGE;
  };
  uint8_t *kb = v.block(l0 + l, g, sg.page), *vb = kb + HB;
  // K codes: 16 bytes of key tile kt_of(i), db's 4 d4 .. of this lane
  const int d4 = warp % DQ;
  auto kt_of = [&](int i) { return FEW ? i : warp / DQ; };
  uint32_t w[KPT][4], sc[KPT][2];
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const uint4 x = *(const uint4 *)(kb + ((kt_of(i) * DQ + d4) * 32 + lane) * 16);
    w[i][0] = x.x, w[i][1] = x.y, w[i][2] = x.z, w[i][3] = x.w;
    const uint8_t *ks = kb + CB + (kt_of(i) * 8 + lg) * 2 * DB;  // of both keys
    if constexpr (DQ == 2) {
      const uint4 y = *(const uint4 *)ks;
      sc[i][0] = d4 ? y.y : y.x;
      sc[i][1] = d4 ? y.w : y.z;
    } else {
      const uint2 y = *(const uint2 *)ks;
      sc[i][0] = y.x;
      sc[i][1] = y.y;
    }
  }
  // the slots that are written
  uint32_t mlo = 0, mhi = 0;
  for (int i = lane; i < count; i += 32) {
    const int s = slot_of(i);
    (s < 32 ? mlo : mhi) |= 1u << (s & 31);
    if (warp == 0) row_at[s] = (uint8_t)i;
  }
  const unsigned long long mask = __reduce_or_sync(0xFFFFFFFFu, mlo) |
                                  (unsigned long long)__reduce_or_sync(0xFFFFFFFFu, mhi) << 32;
  // V: the groups of four slots that change; threads of vi = 0 take the scales of their db too
  const int vch = tid % CH, vdb = FEW ? tid >> 3 : vch >> 1, vi = FEW ? tid & 7 : 4 * (vch & 1);
  uint32_t mine = __ballot_sync(0xFFFFFFFFu, lane < 16 && (mask >> (4 * (lane & 15)) & 15));
  const int n_groups = __popc(mine);
  if (!FEW)
    for (int i = 0; i < tid / CH; ++i) mine &= mine - 1;
  int kg;
  uint32_t old[VW], old_s;
  auto v_word = [&](int i) { return (uint32_t *)(vb + pack_v_code(kg, 16 * vdb + vi + i)); };
  auto v_scales = [&]() { return (uint32_t *)(vb + pack_v_scale(DH, 4 * kg, vdb)); };
  auto v_load = [&]() {  // what the thread's next group holds
    kg = __ffs(mine) - 1;
    if (kg < 0) return;
#pragma unroll
    for (int i = 0; i < VW; ++i) old[i] = *v_word(i);
    if (vi == 0) old_s = *v_scales();
  };
  v_load();
  // the new rows, up to PRE of a warp's in flight
  {
    const int sub = lane / CH, ch = lane % CH;  // rows' halves side by side: K, V (twice for 64)
    const uint32_t rowmask = (CH == 16 ? 0xFFFFu : 0xFFu) << (lane & ~(CH - 1));
    constexpr int RPW = 32 / (2 * CH), PRE = FEW ? 2 : 4;  // rows of a warp at a time
    for (int i0 = warp * RPW; i0 < count; i0 += WARPS * RPW * PRE) {
      Eight<T> x[PRE];  // (past the last row: that one again)
      uint32_t sc[PRE];
#pragma unroll
      for (int j = 0; j < PRE; ++j) {
        if (FEW && i0 + j * WARPS * RPW >= count) break;
        const int i = min(i0 + j * WARPS * RPW + sub / 2, count - 1);
        x[j].load((sub & 1 ? val : k) + (((size_t)(sg.r0 + i) * gridDim.z + l) * v.G + g) * DH +
                  8 * ch);
      }
      if (!FEW) scale_codes<PRE>(x, rowmask, sc);
#pragma unroll
      for (int j = 0; j < PRE; ++j) {
        const int i = i0 + j * WARPS * RPW + sub / 2;
        if (i0 + j * WARPS * RPW >= count) break;
        if (FEW) sc[j] = scale_code(x[j], rowmask);
        if (i < count) {
          code[i][sub & 1][ch] =
              sc[j] == 0 || sc[j] == PACK_NAN ? 0 : x[j].codes(pack_scale(sc[j]));
          if (!(ch & 1)) scale[i][sub & 1][ch >> 1] = (uint8_t)sc[j];
        }
        __syncwarp();
      }
    }
  }
  __syncthreads();
  // K: the half-words of this thread's keys
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    bool changed = false;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int key = 16 * kt_of(i) + pack_key_of(lg) + 2 * h;
      if (mask >> key & 1) {
        changed = true;
        const int r = row_at[key];
        const uint16_t *c = (const uint16_t *)code[r][0] + 16 * d4 + lt;
#pragma unroll
        for (int b = 0; b < 4; ++b) w[i][b] = __byte_perm(w[i][b], c[4 * b], h ? 0x5410 : 0x3254);
        sc[i][h] = *(const uint32_t *)&scale[r][0][4 * d4];
        if (lt == 0)
          *(uint32_t *)(kb + CB + ((kt_of(i) * 8 + lg) * 2 + h) * DB + 4 * d4) = sc[i][h];
      }
    }
    const int off = ((kt_of(i) * DQ + d4) * 32 + lane) * 16;
    if (changed) *(uint4 *)(kb + off) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
    if constexpr (!FEW) {
      *(uint4 *)(kbuf + off) = make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
      if (lt == 0)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          *(uint32_t *)(kbuf + CB + ((kt_of(i) * 8 + lg) * 2 + h) * DB + 4 * d4) = sc[i][h];
    }
  }
  // V: the words of the groups
  for (int n = 0; n < n_groups; n += VG) {
    const uint32_t in = kg < 0 ? 0 : (uint32_t)(mask >> (4 * kg)) & 15;  // slots that are written
    const uint32_t r4 = kg < 0 ? 0 : *(const uint32_t *)&row_at[4 * kg];
    uint32_t w[VW] = {}, c[4], sn = 0, bytes = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      c[j] = 0;
      if (in >> j & 1) {
        const int r = r4 >> (8 * j) & 0xFF;
        if (FEW) {
          const uint32_t *x = code[r][1] + 2 * vdb;
          w[0] |= ((x[0] >> (4 * vi) & 15u) | (x[1] >> (4 * vi) & 15u) << 16) << (4 * j);
        } else {
          c[j] = code[r][1][vch];
        }
        sn |= (uint32_t)scale[r][1][vdb] << (8 * j);
        bytes |= 0xFFu << (8 * j);
      }
    }
    if constexpr (!FEW) {
      uint32_t h[4];
      transpose_out(c, h);
      // half-words of entries 0 2, 1 3 (of those past them: 4 6, 5 7) against the neighbour's
      const uint32_t k0 = vi ? h[1] : h[0], k1 = vi ? h[3] : h[2],
                     g0 = __shfl_xor_sync(0xFFFFFFFFu, vi ? h[0] : h[1], 1),
                     g1 = __shfl_xor_sync(0xFFFFFFFFu, vi ? h[2] : h[3], 1);
      const uint32_t lo[2] = {vi ? g0 : k0, vi ? g1 : k1}, hi[2] = {vi ? k0 : g0, vi ? k1 : g1};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        w[i] = __byte_perm(lo[i & 1], hi[i & 1], i & 2 ? 0x7632 : 0x5410);
    }
    if (kg >= 0) {
      uint32_t nibbles = (__byte_perm(bytes, 0, 0x4420) & 0x0F0Fu) |
                         (__byte_perm(bytes, 0, 0x4431) & 0xF0F0u);
      nibbles |= nibbles << 16;
#pragma unroll
      for (int i = 0; i < VW; ++i) *v_word(i) = (old[i] & ~nibbles) | w[i];
      if (vi == 0) *v_scales() = (old_s & ~bytes) | sn;
    }
    for (int i = 0; i < VG; ++i) mine &= mine - 1;
    v_load();
  }
  const size_t at = v.index(l0 + l, g, sg.page);
  if constexpr (FEW) {
    block_bounds<DH>(amax, w, sc, present, v.bounds + at * 2 * DH, v.unit + at);
  } else {
    __syncthreads();
    if (tid < DH / 2)
      block_bounds<DH>(amax, kbuf, present, v.bounds + at * 2 * DH, v.unit + at);
  }
}

// A CTA per (KV head, page, layer): the block into shared memory, the rows asked for out
// of it.  Bound by HBM: 5000 rows of 32 layers, 184 MB in, 655 MB out, 137 us (6.1 TB/s).
template <int DH, typename T, class Rows>
__global__ void __launch_bounds__(2 * DH)
    k_packed_read(const PackedView v, const __grid_constant__ Rows rows, int l0, T *k, T *val) {
  constexpr int NT = 2 * DH, CH = DH / 8, HB = pack_half_bytes(DH);
  __shared__ __align__(16) uint8_t blk[2 * HB];
  __shared__ int row_of[KVR_PAGE];
  const int tid = threadIdx.x, g = blockIdx.x, l = blockIdx.z;
  pdl_trigger();
  pdl_wait();
  const Segment sg = segment(rows, blockIdx.y);
  const uint8_t *src = v.block(l0 + l, g, sg.page);
  for (int i = tid; i < 2 * HB / 16; i += NT) ((uint4 *)blk)[i] = ((const uint4 *)src)[i];
  const int kg = tid / CH, ch = tid % CH;
  int rr[4];
  rows_of_slots(rows, sg, row_of, kg, rr);
  __syncthreads();
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

// Few rows of each page: a row's K and V of a layer and KV head by DH / 8 lanes each,
// straight from the block.  40 rows of 40 pages, 112 of these each: 3.4 us by the kernel
// above 7.0, which brings 9 KB for 150 bytes.
constexpr int ROW_THREADS = 256;
template <int DH, typename T, class Rows>
__global__ void __launch_bounds__(ROW_THREADS)
    k_packed_read_rows(const PackedView v, const __grid_constant__ Rows rows, int l0, int nl, T *k,
                       T *val) {
  constexpr int CH = DH / 8;
  const int kv = threadIdx.x / CH & 1, ch = threadIdx.x % CH;
  const long long item = (long long)blockIdx.x * (ROW_THREADS / (2 * CH)) + threadIdx.x / (2 * CH);
  pdl_trigger();
  pdl_wait();
  if (item >= (long long)rows.n * nl * v.G) return;
  const int g = (int)(item % v.G), l = (int)(item / v.G % nl), i = (int)(item / v.G / nl);
  const int pos = rows.first >= 0 ? rows.first + i : position(rows, i), key = pos % KVR_PAGE;
  const uint8_t *half = v.block(l0 + l, g, pos / KVR_PAGE) + kv * pack_half_bytes(DH);
  uint32_t c = 0, sc;
  if (kv) {
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      h[e] = *(const uint16_t *)(half + pack_v_code(key >> 2, 8 * ch + e));
    sc = half[pack_v_scale(DH, key, ch >> 1)];
#pragma unroll
    for (int e = 0; e < 8; ++e) c |= (h[e] >> (4 * (key & 3)) & 15u) << (4 * e);
  } else {
    c = *(const uint16_t *)(half + pack_k_code(DH, key, 8 * ch)) |
        (uint32_t)*(const uint16_t *)(half + pack_k_code(DH, key, 8 * ch + 4)) << 16;
    sc = half[pack_k_scale(DH, key, ch >> 1)];
  }
  __half2 y[4];
  float x[8];
  eight_values(c, sc, y);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float2 f = __half22float2(y[e]);
    x[2 * e] = f.x;
    x[2 * e + 1] = f.y;
  }
  Eight<T>::store((kv ? val : k) + item * DH + 8 * ch, x);
}

// A CTA per (KV head, page): the block widened (exactly) into pages of halves [page][K, V]
// [G][KVR_PAGE][DH].
template <int DH>
__global__ void __launch_bounds__(2 * DH)
    k_packed_unpack(const PackedView v, int layer, __half *pages) {
  constexpr int NT = 2 * DH, CH = DH / 8, HB = pack_half_bytes(DH);
  __shared__ __align__(16) uint8_t blk[2 * HB];
  const int tid = threadIdx.x, g = blockIdx.x, page = blockIdx.y, G = gridDim.x;
  pdl_trigger();
  pdl_wait();
  const uint8_t *src = v.block(layer, g, page);
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
      *(uint4 *)(pages + ((((size_t)page * 2 + kv) * G + g) * KVR_PAGE + 4 * kg + j) * DH +
                 8 * ch) = *(const uint4 *)y;
    }
  }
}

// ------------------------------------------------------------ block selection

// P_c = sum over the group's heads of max(q, 0), N_c that of min(q, 0) (in head order),
// both in 8 bits of a common power of two; a block's score is u sum_c (P_c hi_c + N_c
// lo_c), an upper bound (up to the roundings) of the sum of the heads' largest products
// with a key of the block.  The sum is of whole numbers below 2^23 and u a power of two,
// so a score is exact and does not depend on the order of its sum.  The row's own
// block is always taken; of the earlier ones those with the highest scores, ties to the
// lowest.
//
// A cluster of CTAs per (row, KV head), each with a slice of the blocks: eight lanes a
// block, SEL_AHEAD blocks of a lane in flight from the start (their loads cover those
// of q).  The scores meet in the first CTA's shared memory, ordered as unsigned
// numbers; it counts them into SEL_BINS bins of their range, then those of the bin that
// holds the last one wanted into bins of its range, until a threshold parts as many as
// are wanted (twice, as a rule; bisection took 14 rounds, 3 us of 6.8 for 1024 blocks);
// and writes the blocks in order, a warp a stretch of them.
constexpr int SEL_THREADS = 256, SEL_WARPS = SEL_THREADS / 32, SEL_AHEAD = 4;
constexpr int SEL_BINS = 256, SEL_PASSES = 4;  // 8 bits of the 32 a pass
template <int DH, typename T>
__global__ void __launch_bounds__(SEL_THREADS)
    k_packed_select(const T *q, int ldq, const PackedRow *rows, int layer, int grp, int count,
                    int cl, int32_t *blocks) {
  constexpr int W = 2 * DH / 8 / 16;  // 16-byte pieces of a block's bounds a lane
  extern __shared__ uint32_t keys[];  // ordered scores of the blocks before the own
  __shared__ __align__(16) int8_t qs[2][DH];
  __shared__ float amax[DH / 32];
  __shared__ uint32_t range[2][SEL_WARPS];
  __shared__ int tot[2][SEL_WARPS];
  __shared__ __align__(16) int bins[SEL_PASSES][SEL_BINS];
  namespace cg = cooperative_groups;
  const cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int row = blockIdx.x / cl, rank = blockIdx.x % cl, g = blockIdx.y, G = gridDim.y;
  pdl_trigger();
  const PackedRow r = rows[row];
  pdl_wait();
  int32_t *out = blocks + ((size_t)row * G + g) * count;
  const int own = r.pos < 0 ? -1 : r.pos / KVR_PAGE;
  if (own < count) {  // every block that the row sees (the same for all of the cluster)
    for (int i = tid; i < count && rank == 0; i += SEL_THREADS) out[i] = i <= own ? i : -1;
    return;
  }
  if (cl > 1) cluster_arrive();  // this CTA runs
  if (rank == 0)
    for (int i = tid; i < SEL_PASSES * SEL_BINS; i += SEL_THREADS) (&bins[0][0])[i] = 0;
  const int per = (own + cl - 1) / cl, b0 = rank * per, b1 = min(own, b0 + per);
  const int sub = lane >> 3, piece = lane & 7;
  const size_t at = r.doc.index(layer, g, 0);
  int4 x[SEL_AHEAD][W];
  float u[SEL_AHEAD];
  auto fetch = [&](int b) {
#pragma unroll
    for (int k = 0; k < SEL_AHEAD; ++k) {
      const int bk = b + k * 4 * SEL_WARPS;
      if (bk >= b1) continue;
      const int4 *p = (const int4 *)(r.doc.bounds + (at + bk) * 2 * DH) + piece * W;
#pragma unroll
      for (int i = 0; i < W; ++i) x[k][i] = p[i];
      u[k] = r.doc.unit[at + bk];
    }
  };
  const int first = b0 + 4 * warp + sub;
  fetch(first);
  float up = 0.f, down = 0.f;
  if (tid < DH) {
    const T *x = q + (size_t)row * ldq + (size_t)g * grp * DH + tid;
#pragma unroll 4
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
    const float f = a < INFINITY ? __frcp_rn(unit_of(a)) : 0.f;
    qs[0][tid] = a < INFINITY ? (int8_t)__float2int_rn(up * f) : 0;
    qs[1][tid] = a < INFINITY ? (int8_t)__float2int_rn(down * f) : 0;
  }
  __syncthreads();
  int4 qv[W];
#pragma unroll
  for (int i = 0; i < W; ++i) qv[i] = ((const int4 *)qs)[piece * W + i];
  uint32_t *all = cl > 1 ? cluster.map_shared_rank(keys, 0) : keys;
  if (cl > 1) cluster_wait();  // so does the first, whose memory is written
  for (int b = first; b - sub - 4 * warp < b1; b += 4 * SEL_WARPS * SEL_AHEAD) {
    if (b != first) fetch(b);
#pragma unroll
    for (int k = 0; k < SEL_AHEAD; ++k) {
      const int bk = b + k * 4 * SEL_WARPS;
      int s = 0;
      if (bk < b1) {
#pragma unroll
        for (int i = 0; i < W; ++i) {
          s = __dp4a(x[k][i].x, qv[i].x, s);
          s = __dp4a(x[k][i].y, qv[i].y, s);
          s = __dp4a(x[k][i].z, qv[i].z, s);
          s = __dp4a(x[k][i].w, qv[i].w, s);
        }
      }
#pragma unroll
      for (int o = 4; o; o /= 2) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
      if (bk < b1 && piece == 0) {
        const float f = (float)s * u[k];
        const uint32_t v = __float_as_uint(f == 0.f ? 0.f : f);
        all[bk] = v >> 31 ? ~v : v | 0x80000000u;
      }
    }
  }
  if (cl > 1) {
    cluster_arrive();
    cluster_wait();
    if (rank) return;
  } else {
    __syncthreads();
  }
  // the want-th largest key: the largest t with at least that many >= t
  const int want = count - 1;
  uint32_t lo = 0xFFFFFFFFu, hi = 0;
  for (int b = tid; b < own; b += SEL_THREADS) lo = min(lo, keys[b]), hi = max(hi, keys[b]);
  lo = __reduce_min_sync(0xFFFFFFFFu, lo);
  hi = __reduce_max_sync(0xFFFFFFFFu, hi);
  if (lane == 0) range[0][warp] = lo, range[1][warp] = hi;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SEL_WARPS; ++w) lo = min(lo, range[0][w]), hi = max(hi, range[1][w]);
  // `above` keys are > hi, fewer than wanted; with those in [lo, hi] it is as many at least
  int above = 0;
  for (int pass = 0; lo < hi && want > 0; ++pass) {
    const int shift = max(0, 24 - __clz(hi - lo));  // the range's bits, but for eight
    for (int b = tid; b < own; b += SEL_THREADS) {
      const uint32_t x = keys[b];
      if (x >= lo && x <= hi) atomicAdd(&bins[pass][(x - lo) >> shift], 1);
    }
    __syncthreads();
    // every warp: eight bins a lane, the highest first
    int n[8], sum = 0;
    *(int4 *)&n[0] = *(const int4 *)&bins[pass][SEL_BINS - 8 - 8 * lane];
    *(int4 *)&n[4] = *(const int4 *)&bins[pass][SEL_BINS - 4 - 8 * lane];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += n[i];
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += x;
    }
    const uint32_t reach = __ballot_sync(0xFFFFFFFFu, above + upto >= want);
    const int at_lane = __ffs(reach) - 1;
    int before = above + upto - sum, bin = 0, held = 0;  // (those of lane at_lane count)
    bool found = false;
#pragma unroll
    for (int i = 7; i >= 0; --i)
      if (!found) {
        if (before + n[i] >= want)
          found = true, bin = SEL_BINS - 8 - 8 * lane + i, held = n[i];
        else
          before += n[i];
      }
    bin = __shfl_sync(0xFFFFFFFFu, bin, at_lane);
    held = __shfl_sync(0xFFFFFFFFu, held, at_lane);
    above = __shfl_sync(0xFFFFFFFFu, before, at_lane);
    lo += (uint32_t)bin << shift;
    // all of the bin, or some of it
    hi = above + held == want ? lo : lo + min(hi - lo, (1u << shift) - 1);
  }
  const uint32_t t = lo;
  // keys above t, and as many of those equal to it as are wanted, in order
  const int span = (own + SEL_WARPS - 1) / SEL_WARPS, w0 = warp * span, w1 = min(own, w0 + span);
  int gt = 0, eq = 0;
  for (int b = w0 + lane; b < w1; b += 32) gt += keys[b] > t, eq += keys[b] == t;
  gt = __reduce_add_sync(0xFFFFFFFFu, gt);
  eq = __reduce_add_sync(0xFFFFFFFFu, eq);
  if (lane == 0) tot[0][warp] = gt, tot[1][warp] = eq;
  __syncthreads();
  int gts = 0, eqs = 0;  // before this warp's stretch
  above = 0;
#pragma unroll
  for (int w = 0; w < SEL_WARPS; ++w) {
    above += tot[0][w];
    if (w < warp) gts += tot[0][w], eqs += tot[1][w];
  }
  const int ties = want - above;
  for (int b = w0; b < w1 && want > 0; b += 32) {
    const uint32_t kx = b + lane < w1 ? keys[b + lane] : 0, below = (1u << lane) - 1;
    const uint32_t mg = __ballot_sync(0xFFFFFFFFu, b + lane < w1 && kx > t),
                   me = __ballot_sync(0xFFFFFFFFu, b + lane < w1 && kx == t);
    const int e = eqs + __popc(me & below);
    if ((mg >> lane & 1) || ((me >> lane & 1) && e < ties))
      out[gts + __popc(mg & below) + min(e, ties)] = b + lane;
    gts += __popc(mg);
    eqs += __popc(me);
  }
  if (tid == 0) out[want] = own;
}

}  // namespace

namespace {
// Whether DH / 2 threads take a page's rows (most of them on a page, blocks in all): as long
// as the rows past the first are at most 1.6 w^2, with w waves of CTAs of 2 DH threads.
// Over 150 launches of 1 to 32 rows on each of 1 to 40 pages the kernel taken is 0.1% slower
// than the other on average, 5% at most.
template <int DH, typename T>
bool few_rows(int most, long long blocks, int sms) {
  const long long places = (long long)sms * ((sizeof(T) == 2 ? 1024 : 768) / (2 * DH));
  return most <= PATCH_FEW && 5 * (most - 1) * places * places <= 8 * blocks * blocks;
}
// Pages that a run writes whole by k_packed_write_pages, all others by k_packed_patch.
template <int DH, typename T, class Rows>
int write_rows(const PackedView &v, const Rows &rows, int len, int l0, int nl, const void *k,
               const void *val, int sms, cudaStream_t s) {
  int2 part{0, 0};
  int parts = rows.n_seg, launches = 0, most = rows.most;
  if (rows.first >= 0) {
    // whole pages [p0, p1), the last of which may end where the document does
    const int end = rows.first + rows.n, p0 = (rows.first + KVR_PAGE - 1) / KVR_PAGE,
              p1 = end == len ? (end + KVR_PAGE - 1) / KVR_PAGE : end / KVR_PAGE;
    const int head = rows.first % KVR_PAGE ? std::min(rows.n, p0 * KVR_PAGE - rows.first) : 0;
    const int tail = p1 * KVR_PAGE >= end ? 0 : end - std::max(p1 * KVR_PAGE, rows.first + head);
    parts = most = 0;
    if (head) parts = 1, most = head;
    if (tail) (parts ? part.y : part.x) = rows.n_seg - 1, ++parts, most = std::max(most, tail);
    if (p1 > p0) {
      const size_t skip = (size_t)(p0 * KVR_PAGE - rows.first) * nl * v.G * DH;
      launch_pdl(k_packed_write_pages<DH, T>, dim3(v.G, p1 - p0, nl), dim3(2 * DH), 0, s, v, p0,
                 end - p0 * KVR_PAGE, l0, (const T *)k + skip, (const T *)val + skip);
      ++launches;
    }
  }
  if (parts) {
    auto patch = [&](auto kernel, int threads) {
      launch_pdl(kernel, dim3(v.G, parts, nl), dim3(threads), 0, s, v, rows, part, len, l0,
                 (const T *)k, (const T *)val);
    };
    if (few_rows<DH, T>(most, (long long)v.G * parts * nl, sms))
      patch(k_packed_patch<DH, T, Rows, DH / 2>, DH / 2);
    else
      patch(k_packed_patch<DH, T, Rows, 2 * DH>, 2 * DH);
    ++launches;
  }
  return launches;
}
template <int DH, typename T, class Rows>
void read_rows(const PackedView &v, const Rows &rows, int l0, int nl, void *k, void *val,
               cudaStream_t s) {
  if (rows.n <= 4 * rows.n_seg) {  // 4 rows a page: as fast either way
    const long long items = (long long)rows.n * nl * v.G;
    const int per = ROW_THREADS / (DH / 4);
    launch_pdl(k_packed_read_rows<DH, T, Rows>, dim3((unsigned)((items + per - 1) / per)),
               dim3(ROW_THREADS), 0, s, v, rows, l0, nl, (T *)k, (T *)val);
    return;
  }
  launch_pdl(k_packed_read<DH, T, Rows>, dim3(v.G, rows.n_seg, nl), dim3(2 * DH), 0, s, v, rows, l0,
             (T *)k, (T *)val);
}
// f with the head size, the type and the kind of rows as template arguments.
template <class F>
void by_kind(int dh, int dtype, const PackedRows &rows, F f) {
  auto typed = [&](auto d, auto t) {
    if (rows.inlined)
      f(d, t, rows.list);
    else
      f(d, t, (const PackedRun &)rows.list);
  };
  auto sized = [&](auto d) {
    if (dtype == KVR_DTYPE_BF16)
      typed(d, __nv_bfloat16{});
    else
      typed(d, float{});
  };
  if (dh == 128)
    sized(std::integral_constant<int, 128>{});
  else
    sized(std::integral_constant<int, 64>{});
}
}  // namespace

int launch_packed_write(const PackedView &v, int dtype, const PackedRows &rows, int len, int l0,
                        int nl, const void *k, const void *val, int sms, cudaStream_t s) {
  int launches = 0;
  by_kind(v.dh, dtype, rows, [&](auto d, auto t, const auto &r) {
    launches = write_rows<decltype(d)::value, decltype(t)>(v, r, len, l0, nl, k, val, sms, s);
  });
  return launches;
}

void launch_packed_read(const PackedView &v, int dtype, const PackedRows &rows, int l0, int nl,
                        void *k, void *val, cudaStream_t s) {
  by_kind(v.dh, dtype, rows, [&](auto d, auto t, const auto &r) {
    read_rows<decltype(d)::value, decltype(t)>(v, r, l0, nl, k, val, s);
  });
}

void launch_packed_bounds(const PackedView &v, int page, int len, int nl, int l0, int l1,
                          cudaStream_t s) {
  const int present = std::min(KVR_PAGE, len - page * KVR_PAGE);
  launch_pdl(v.dh == 128 ? k_packed_bounds<128> : k_packed_bounds<64>, dim3(v.G, nl - (l1 - l0)),
             dim3(v.dh / 2), 0, s, v, page, present, l0, l1);
}

void launch_packed_clear(const PackedView &v, int len, int end, int nl, cudaStream_t s) {
  launch_pdl(v.dh == 128 ? k_packed_clear<128> : k_packed_clear<64>,
             dim3(v.G, (end - 1) / KVR_PAGE - len / KVR_PAGE + 1, nl), dim3(2 * v.dh), 0, s, v, len);
}

void launch_packed_units(float *unit, size_t n, cudaStream_t s) {
  k_packed_units<<<(unsigned)((n + 255) / 256), 256, 0, s>>>(unit, n);
}

void launch_packed_unpack(const PackedView &v, int layer, int n_pages, void *pages, bool settled,
                          cudaStream_t s) {
  auto *kernel = v.dh == 128 ? k_packed_unpack<128> : k_packed_unpack<64>;
  const dim3 grid(v.G, n_pages);
  if (settled)
    launch_pdl(kernel, grid, dim3(2 * v.dh), 0, s, v, layer, (__half *)pages);
  else
    kernel<<<grid, 2 * v.dh, 0, s>>>(v, layer, (__half *)pages);
}

namespace {
template <int DH, typename T>
const char *select_blocks(const PackedAttnArgs &a, int max_pages, int32_t *blocks, cudaStream_t s) {
  static PerDevice<size_t> state;
  auto *kernel = k_packed_select<DH, T>;
  const size_t smem = (size_t)max_pages * sizeof(uint32_t);
  if (smem > 40 * 1024)
    if (const char *e = smem_opt_in(state, kernel, smem)) return e;
  // A CTA for every 128 blocks or more of a row, its warps' loads in flight at once, as long as
  // the chip takes all of them together (four an SM); for fewer than 256 blocks a CTA where
  // half the SMs would idle.  1024 blocks: 8 (row, KV head)s by 8 CTAs each 6.0 us (by one
  // 11.3), 128 by 4 CTAs 10.6 (one 14.1, eight 14.1); 193 blocks: 8 by 2 4.5 (one 4.7), 128
  // by one 6.1 (two 6.6).
  int cl = 1;
  while (cl < 8 && max_pages > 128 * cl &&
         (long long)a.n_rows * a.G * cl * 4 <=
             (long long)a.num_sms * (max_pages >= 256 * cl ? 8 : 1))
    cl *= 2;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(a.n_rows * cl, a.G);
  cfg.blockDim = dim3(SEL_THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cl;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = g_pdl && a.settled ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, (const T *)a.q, a.ldq, a.rows, a.layer,
                                           a.grp, a.n_blocks, cl, blocks);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}
}  // namespace

const char *launch_packed_select(const PackedAttnArgs &a, int max_pages, int32_t *blocks,
                                 cudaStream_t s) {
  if (a.dtype == KVR_DTYPE_BF16)
    return a.dh == 128 ? select_blocks<128, __nv_bfloat16>(a, max_pages, blocks, s)
                       : select_blocks<64, __nv_bfloat16>(a, max_pages, blocks, s);
  return a.dh == 128 ? select_blocks<128, float>(a, max_pages, blocks, s)
                     : select_blocks<64, float>(a, max_pages, blocks, s);
}

}  // namespace kvr
