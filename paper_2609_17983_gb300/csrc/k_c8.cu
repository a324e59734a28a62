// k_c8.cu -- the 8-bit cache's entries (c8.cuh): quantising K/V rows as they are written, reading
// them back, choosing the ones to keep by their weight, and moving those together.
#include <cooperative_groups.h>
#include <math.h>

#include <algorithm>

#include "c8.cuh"
#include "row_segments.cuh"

namespace kvr {
namespace {

constexpr int NT = 256, WRITE_NT = 128, KEEP_NT = 128;

// Sixteen entries of a row: loaded, the bits of their largest magnitude as a float (infinities and
// NaN lie above all others), their codes under the inverse of a power, stored.
template <typename T>
struct Sixteen;
template <>
struct Sixteen<__nv_bfloat16> {
  uint4 u[2];
  __device__ __forceinline__ void load(const __nv_bfloat16 *p) {
    u[0] = __ldcs((const uint4 *)p);
    u[1] = __ldcs((const uint4 *)p + 1);
  }
  __device__ __forceinline__ uint32_t magnitude() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      m = max_u16x2(m, max_u16x2(u[i].x & 0x7FFF7FFFu, u[i].y & 0x7FFF7FFFu));
      m = max_u16x2(m, max_u16x2(u[i].z & 0x7FFF7FFFu, u[i].w & 0x7FFF7FFFu));
    }
    return max(m & 0xFFFF0000u, m << 16);
  }
  __device__ __forceinline__ uint4 codes(float f) const {
    auto two = [&](uint32_t a, uint32_t b) {
      return c8_codes(__uint_as_float(a << 16) * f, __uint_as_float(a & 0xFFFF0000u) * f,
                      __uint_as_float(b << 16) * f, __uint_as_float(b & 0xFFFF0000u) * f);
    };
    return make_uint4(two(u[0].x, u[0].y), two(u[0].z, u[0].w), two(u[1].x, u[1].y),
                      two(u[1].z, u[1].w));
  }
};
template <>
struct Sixteen<float> {
  float4 u[4];
  __device__ __forceinline__ void load(const float *p) {
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __ldcs((const float4 *)p + i);
  }
  __device__ __forceinline__ uint32_t magnitude() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m = max(m, __float_as_uint(u[i].x) & 0x7FFFFFFFu);
      m = max(m, __float_as_uint(u[i].y) & 0x7FFFFFFFu);
      m = max(m, __float_as_uint(u[i].z) & 0x7FFFFFFFu);
      m = max(m, __float_as_uint(u[i].w) & 0x7FFFFFFFu);
    }
    return m;
  }
  __device__ __forceinline__ uint4 codes(float f) const {
    auto four = [&](float4 x) { return c8_codes(x.x * f, x.y * f, x.z * f, x.w * f); };
    return make_uint4(four(u[0]), four(u[1]), four(u[2]), four(u[3]));
  }
};

// 32 bytes: WIDE, where all places are a multiple of 32, by one store, else by two, each of which is
// half of every sector that a warp reaches (the read of 4096 entries of 256 heads of 128 in bf16 121 us
// and 125, of 5000 of 56 in fp32 55 and 90).
template <bool WIDE>
__device__ __forceinline__ void store32(void *p, const uint32_t *x) {
  if (WIDE) {
    asm volatile("st.global.cs.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(x[0]),
                 "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7])
                 : "memory");
  } else {
    __stcs((uint4 *)p, make_uint4(x[0], x[1], x[2], x[3]));
    __stcs((uint4 *)p + 1, make_uint4(x[4], x[5], x[6], x[7]));
  }
}
// Sixteen values of codes under a power.
template <bool WIDE>
__device__ __forceinline__ void store16(__nv_bfloat16 *p, uint4 c, float power) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 x = c8_values(w[i], power);
    const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
    o[2 * i] = *(const uint32_t *)&a;
    o[2 * i + 1] = *(const uint32_t *)&b;
  }
  store32<WIDE>(p, o);
}
template <bool WIDE>
__device__ __forceinline__ void store16(float *p, uint4 c, float power) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 4; i += 2) {
    const float4 x = c8_values(w[i], power), y = c8_values(w[i + 1], power);
    const uint32_t o[8] = {__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(x.z),
                           __float_as_uint(x.w), __float_as_uint(y.x), __float_as_uint(y.y),
                           __float_as_uint(y.z), __float_as_uint(y.w)};
    store32<WIDE>(p + 4 * i, o);
  }
}

// Codes under another power, f times as small a one (f: old / new); a NaN stays.
__device__ __forceinline__ uint4 recode(uint4 c, float f) {
  auto word = [&](uint32_t w) {
    const float4 x = c8_values(w, f);
    return c8_codes(x.x, x.y, x.z, x.w);
  };
  return make_uint4(word(c.x), word(c.y), word(c.z), word(c.w));
}

// The factor of kept codes from their block's power to the new one.  A code that is not zero, 2^-9 or
// more, makes the new power at least 2^-17 of the old one; zeros alone may meet a quotient of up to
// 2^220, which is infinite and would make them NaN.
__device__ __forceinline__ float kept_factor(float old, float power) {
  return fminf(old * c8_inverse(power), 131072.f);
}

// Where a thread of a block's CTA of N works: piece `c` of the rows `row + j * STEP`.
template <int DH, int N>
struct Place {
  static constexpr int PIECES = DH / 16, STEP = N / PIECES, ROWS = KVR_PAGE / STEP;
  int c, row;
  __device__ Place() : c(threadIdx.x % PIECES), row(threadIdx.x / PIECES) {}
  __device__ int slot(int j) const { return row + j * STEP; }
  __device__ int offset(int slot) const { return slot * DH + 16 * c8_piece<DH>(slot, c); }
  // the lanes of this thread's row
  __device__ uint32_t row_lanes() const {
    return ((1u << PIECES) - 1) << (threadIdx.x % 32 / PIECES * PIECES);
  }
};

// The largest of every thread's x, in s (shared, 0 before; a barrier follows by the caller).
__device__ __forceinline__ void block_max(uint32_t x, uint32_t *s) {
  x = __reduce_max_sync(0xFFFFFFFFu, x);
  if (threadIdx.x % 32 == 0) atomicMax(s, x);
}

// A CTA quantises the rows of one block of a layer and KV head: their largest magnitudes give the
// powers (with the old ones, where other entries stay), every thread has its rows' pieces in
// registers from the load to the codes.  Bound by HBM: 5000 entries of 28 layers of 4, 287 MB in,
// 143 MB out, 66.4 us (6.5 TB/s; of 256 threads 67.4, of 64 70.3).
template <int DH, typename T, class Rows>
__global__ void __launch_bounds__(WRITE_NT)
    k_c8_write(const C8View v, const __grid_constant__ Rows rows, int len, int shift, int l0,
               int stride, const T *k, const T *val) {
  using P = Place<DH, WRITE_NT>;
  const P at;
  __shared__ int row_of[KVR_PAGE];
  __shared__ uint32_t s_max[2];
  pdl_trigger();
  pdl_wait();
  const Segment seg = segment(rows, blockIdx.z);
  const int tid = threadIdx.x, lg = blockIdx.y, g = blockIdx.x, layer = l0 + lg;
  if (tid < KVR_PAGE) row_of[tid] = -1;
  if (tid < 2) s_max[tid] = 0;
  __syncthreads();
  for (int i = seg.r0 + tid; i < seg.r1; i += WRITE_NT)
    row_of[rows.first >= 0 ? (rows.first + i) % KVR_PAGE : position(rows, i) % KVR_PAGE] = i;
  __syncthreads();
  const size_t block = v.index(layer, g, seg.page);
  uint8_t *kb = v.blocks + block * c8_block_bytes(DH), *vb = kb + c8_half_bytes(DH);
  const int had = len - seg.page * KVR_PAGE;  // slots below it held entries
  Sixteen<T> x[P::ROWS], y[P::ROWS];
  int r[P::ROWS];
  bool bad[P::ROWS], stays = false;
  uint32_t mk = 0, mv = 0;
#pragma unroll
  for (int j = 0; j < P::ROWS; ++j) {
    r[j] = row_of[at.slot(j)];
    stays = stays || (r[j] < 0 && at.slot(j) < had);
    if (r[j] >= 0) {
      const size_t src = (((size_t)r[j] * stride + lg) * v.G + g) * DH + 16 * at.c;
      x[j].load(k + src);
      y[j].load(val + src);
    }
  }
#pragma unroll
  for (int j = 0; j < P::ROWS; ++j) {
    const uint32_t a = r[j] >= 0 ? x[j].magnitude() : 0, b = r[j] >= 0 ? y[j].magnitude() : 0;
    bad[j] = __ballot_sync(0xFFFFFFFFu, a >= C8_INFINITE || b >= C8_INFINITE) & at.row_lanes();
    if (!bad[j]) mk = max(mk, a), mv = max(mv, b);
  }
  block_max(mk, &s_max[0]);
  block_max(mv, &s_max[1]);
  stays = __syncthreads_or(stays);
  const float2 old = v.power[block];
  float pk = c8_power(s_max[0]), pv = c8_power(s_max[1]);
  if (stays) pk = fmaxf(pk, old.x), pv = fmaxf(pv, old.y);
  const float ik = c8_inverse(pk), iv = c8_inverse(pv);
  const uint4 nan = make_uint4(0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu, 0x7F7F7F7Fu);
#pragma unroll
  for (int j = 0; j < P::ROWS; ++j) {
    const int slot = at.slot(j), o = at.offset(slot);
    if (r[j] >= 0) {
      *(uint4 *)(kb + o) = bad[j] ? nan : x[j].codes(ik);
      *(uint4 *)(vb + o) = bad[j] ? make_uint4(0, 0, 0, 0) : y[j].codes(iv);
      if (at.c == 0 && slot >= had) {
        v.number[block * KVR_PAGE + slot] = seg.page * KVR_PAGE + slot + shift;
        v.weight[block * KVR_PAGE + slot] = 0.f;
      }
    } else if (slot < had) {
      if (pk != old.x) *(uint4 *)(kb + o) = recode(*(const uint4 *)(kb + o), old.x * ik);
      if (pv != old.y) *(uint4 *)(vb + o) = recode(*(const uint4 *)(vb + o), old.y * iv);
    }
  }
  __syncthreads();  // all have read the old powers
  if (tid == 0) v.power[block] = make_float2(pk, pv);
}

// A CTA reads the listed rows of one block of a layer and KV head, a piece of K and V a thread at a
// time.  Bound by HBM: 5000 entries of 28 layers of 4, 143 MB in, 287 MB out, 66.2 us (6.5 TB/s; by
// stores of 16 bytes 68.2, 74.4 in fewer registers, 79.8 with all loads of a thread ahead of its
// stores).
template <int DH, typename T, bool WIDE, class Rows>
__global__ void __launch_bounds__(NT, 5)
    k_c8_read(const C8View v, const __grid_constant__ Rows rows, int l0, T *k, T *val) {
  constexpr int PIECES = DH / 16;
  pdl_trigger();
  pdl_wait();
  const Segment seg = segment(rows, blockIdx.x);
  const int lg = blockIdx.y, g = blockIdx.z;
  const size_t block = v.index(l0 + lg, g, seg.page);
  const uint8_t *kb = v.blocks + block * c8_block_bytes(DH), *vb = kb + c8_half_bytes(DH);
  const float2 power = v.power[block];
  for (int i = threadIdx.x; i < (seg.r1 - seg.r0) * PIECES; i += NT) {
    const int r = seg.r0 + i / PIECES, c = i % PIECES;
    const int slot = (rows.first >= 0 ? rows.first + r : position(rows, r)) % KVR_PAGE;
    const int o = slot * DH + 16 * c8_piece<DH>(slot, c);
    const uint4 x = __ldcs((const uint4 *)(kb + o));
    uint4 y = __ldcs((const uint4 *)(vb + o));
    if ((x.x & 0x7F) == 0x7F) y = x;  // a marked entry
    const size_t to = (((size_t)r * gridDim.y + lg) * v.G + g) * DH + 16 * c;
    store16<WIDE>(k + to, x, power.x);
    store16<WIDE>(val + to, y, power.y);
  }
}

__global__ void k_c8_clear(float2 *power, size_t n) {
  const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i < n) power[i] = make_float2(C8_LEAST_POWER, C8_LEAST_POWER);
}

// Numbers and weights out, or weights in; a row of the grid a layer and KV head.
__global__ void k_c8_entries(const C8View v, int len, int l0, int32_t *number, float *weight,
                             const float *set) {
  const int e = blockIdx.x * blockDim.x + threadIdx.x;
  pdl_trigger();
  pdl_wait();
  if (e >= len) return;
  const size_t at = ((size_t)l0 * v.G + blockIdx.y) * v.pages * KVR_PAGE + e,
               to = (size_t)blockIdx.y * len + e;
  if (set) v.weight[at] = set[to];
  if (number) number[to] = v.number[at];
  if (weight) weight[to] = v.weight[at];
}

// ---- choosing ----

// A weight's place in the order: larger weights have larger keys, equal ones equal keys (-0 and 0
// too); NaN comes last.
__device__ __forceinline__ uint32_t order_key(float w) {
  if (w != w) return 0;
  const uint32_t u = __float_as_uint(w + 0.f);
  return u >> 31 ? ~u : u | 0x80000000u;
}

constexpr int CT = 1024, DIGIT = 11, BINS = 1 << DIGIT;
// A CTA for each layer and KV head finds the keep-th largest key by digits of 11, 11 and 10 bits,
// then writes the entries above it and the lowest of those equal to it in order: each warp owns a
// stretch of entries, counts both kinds in it, and places its own behind those of the warps before
// it. CACHED: the keys lie in shared memory.  Bound by the counting: weights of a few binades meet
// in few bins, of which 11 bits make four a binade.  12345 entries of 256 heads, weights even in
// [0, 1): 16.0 us (with digits of 8 bits 24.4, four keys of a thread fetched ahead of their
// counting 16.7).
template <bool CACHED>
__global__ void __launch_bounds__(CT)
    k_c8_choose(const C8View v, int len, int keep, int first, int recent, int32_t *kept) {
  extern __shared__ uint32_t s_keys[];
  __shared__ int hist[BINS], s_above[CT / 32], s_equal[CT / 32], s_digit, s_left;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const float *w = v.weight + (size_t)blockIdx.x * v.pages * KVR_PAGE;
  int32_t *out = kept + (size_t)blockIdx.x * keep;
  pdl_trigger();
  for (int i = tid; i < BINS; i += CT) hist[i] = 0;
  pdl_wait();
  __syncthreads();
  auto load_key = [&](int e) {
    return e < first || e >= len - recent ? 0xFFFFFFFFu : order_key(w[e]);
  };
  auto key_of = [&](int e) { return CACHED ? s_keys[e] : load_key(e); };
  uint32_t prefix = 0;
  int left = keep;  // of the entries with the prefix, so many belong to the largest
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass < 2 ? BINS : BINS / 2;
    if (pass) {
      for (int i = tid; i < bins; i += CT) hist[i] = 0;
      __syncthreads();
    }
    for (int e = tid; e < len; e += CT) {
      const uint32_t x = pass ? key_of(e) : load_key(e);
      if (CACHED && !pass) s_keys[e] = x;
      if (!pass || x >> (pass == 1 ? 21 : 10) == prefix >> (pass == 1 ? 21 : 10))
        atomicAdd(&hist[x >> shift & (bins - 1)], 1);
    }
    __syncthreads();
    // the digit at which the count from the largest reaches `left`: two bins a thread
    const int lo = bins - 1 - 2 * tid, c0 = 2 * tid < bins ? hist[lo] : 0,
              c1 = 2 * tid < bins ? hist[lo - 1] : 0;
    int upto = c0 + c1;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
      if (lane >= o) upto += y;
    }
    if (lane == 31) s_above[warp] = upto;
    __syncthreads();
    int before = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? s_above[lane] : 0) + upto - c0 - c1;
    if (before < left && left <= before + c0 + c1) {
      const bool second = left > before + c0;
      s_digit = lo - second;
      s_left = left - before - (second ? c0 : 0);
    }
    __syncthreads();
    prefix |= (uint32_t)s_digit << shift;
    left = s_left;
  }
  const int per = (len + CT - 1) / CT * 32, e0 = min(len, warp * per), e1 = min(len, e0 + per);
  int above = 0, equal = 0;
  for (int e = e0 + lane; e < e1; e += 32) {
    const uint32_t x = key_of(e);
    above += x > prefix;
    equal += x == prefix;
  }
  above = __reduce_add_sync(0xFFFFFFFFu, above);
  equal = __reduce_add_sync(0xFFFFFFFFu, equal);
  if (lane == 0) s_above[warp] = above, s_equal[warp] = equal;
  __syncthreads();
  above = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? s_above[lane] : 0);
  equal = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? s_equal[lane] : 0);
  for (int e = e0; e < e1; e += 32) {
    const uint32_t x = e + lane < e1 ? key_of(e + lane) : 0;
    const bool in = e + lane < e1, a = in && x > prefix, b = in && x == prefix;
    const uint32_t ma = __ballot_sync(0xFFFFFFFFu, a), mb = __ballot_sync(0xFFFFFFFFu, b),
                   low = (1u << lane) - 1;
    const int na = above + __popc(ma & low), nb = equal + __popc(mb & low);
    if (a || (b && nb < left)) out[na + min(nb, left)] = e + lane;
    above += __popc(ma);
    equal += __popc(mb);
  }
}

// ---- keeping ----

// CTA x of a layer and KV head makes blocks x, x + gridDim.x, ... of dst from the listed entries of
// src: their rows into registers, the powers from the largest of them, the codes under those. SAME:
// dst is src, and the CTAs of a layer and KV head are one cluster.  An entry's new place is never
// behind its old one, so when all of a round's blocks have been read they may be written: later
// rounds read nothing before them.  Bound by HBM: 4096 of 12345 entries of 256 heads of 128, 268 MB
// in, 268 MB out, 85.1 us (6.3 TB/s; of 256 threads 101, of 64 91.7).
template <int DH, bool SAME>
__global__ void __launch_bounds__(KEEP_NT)
    k_c8_keep(const C8View src, const C8View dst, int len, const int32_t *kept, int n) {
  using P = Place<DH, KEEP_NT>;
  const P at;
  __shared__ int from[KVR_PAGE];
  __shared__ uint32_t s_max[2];
  const int tid = threadIdx.x, h = blockIdx.y;
  const int32_t *list = kept + (size_t)h * n;
  const int blocks = (n + KVR_PAGE - 1) / KVR_PAGE;
  const int rounds = (blocks + gridDim.x - 1) / gridDim.x;
  const size_t s0 = (size_t)h * src.pages, d0 = (size_t)h * dst.pages;
  pdl_trigger();
  pdl_wait();
  for (int round = 0; round < rounds; ++round) {
    const int b = round * gridDim.x + blockIdx.x, e0 = b * KVR_PAGE;
    const bool some = b < blocks;
    if (tid < 2) s_max[tid] = 0;
    int number = -1;
    float weight = 0.f;
    if (tid < KVR_PAGE) {
      const int i = e0 + tid;
      int e = -1;
      if (some && i < n) {
        // as an ascending list has them; anything else is an entry that is not there
        e = list[i];
        if (e < i || e >= len || (i && e <= list[i - 1])) e = -1;
        if (e >= 0) {
          number = src.number[s0 * KVR_PAGE + e];
          weight = src.weight[s0 * KVR_PAGE + e];
        }
      }
      from[tid] = e;
    }
    __syncthreads();
    uint4 x[P::ROWS], y[P::ROWS];
    float2 power[P::ROWS];
    float mk = 0.f, mv = 0.f;
#pragma unroll
    for (int j = 0; j < P::ROWS; ++j) {
      const int e = from[at.slot(j)];
      x[j] = y[j] = make_uint4(0, 0, 0, 0);
      power[j] = make_float2(1.f, 1.f);
      if (e >= 0) {
        const size_t block = s0 + e / KVR_PAGE;
        const uint8_t *p = src.blocks + block * c8_block_bytes(DH) + at.offset(e % KVR_PAGE);
        x[j] = *(const uint4 *)p;
        y[j] = *(const uint4 *)(p + c8_half_bytes(DH));
        power[j] = src.power[block];
      }
    }
#pragma unroll
    for (int j = 0; j < P::ROWS; ++j) {
      auto largest = [](uint4 c) {  // code without sign, of sixteen
        uint32_t m = __vmaxu4(__vmaxu4(c.x & 0x7F7F7F7Fu, c.y & 0x7F7F7F7Fu),
                              __vmaxu4(c.z & 0x7F7F7F7Fu, c.w & 0x7F7F7F7Fu));
        m = __vmaxu4(m, m >> 16);
        return max(m & 0xFF, m >> 8 & 0xFF);
      };
      const uint32_t a = largest(x[j]), c = largest(y[j]);
      if (a != 0x7F) mk = fmaxf(mk, c8_values(a, power[j].x).x);
      mv = fmaxf(mv, c8_values(c, power[j].y).x);
    }
    block_max(__float_as_uint(mk), &s_max[0]);
    block_max(__float_as_uint(mv), &s_max[1]);
    if (SAME) {
      // (also this CTA's barrier before the maxima are read)
      __syncthreads();
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    const float pk = c8_power(s_max[0]), pv = c8_power(s_max[1]);
    if (some) {
      uint8_t *to = dst.blocks + (d0 + b) * c8_block_bytes(DH);
#pragma unroll
      for (int j = 0; j < P::ROWS; ++j) {
        const int slot = at.slot(j), o = at.offset(slot);
        if (e0 + slot >= n) continue;
        *(uint4 *)(to + o) = power[j].x == pk ? x[j] : recode(x[j], kept_factor(power[j].x, pk));
        *(uint4 *)(to + o + c8_half_bytes(DH)) =
            power[j].y == pv ? y[j] : recode(y[j], kept_factor(power[j].y, pv));
      }
      if (tid < KVR_PAGE && e0 + tid < n) {
        dst.number[d0 * KVR_PAGE + e0 + tid] = number;
        dst.weight[d0 * KVR_PAGE + e0 + tid] = weight;
      }
      if (tid == 0) dst.power[d0 + b] = make_float2(pk, pv);
    }
    __syncthreads();
  }
}

template <class F>
void by_shape(int dh, int dtype, F f) {
  if (dtype == KVR_DTYPE_BF16) {
    if (dh == 128)
      f(std::integral_constant<int, 128>{}, __nv_bfloat16{});
    else
      f(std::integral_constant<int, 64>{}, __nv_bfloat16{});
  } else {
    if (dh == 128)
      f(std::integral_constant<int, 128>{}, float{});
    else
      f(std::integral_constant<int, 64>{}, float{});
  }
}

}  // namespace

void launch_c8_write(const C8View &v, int dtype, const PackedRows &rows, int len, int shift, int l0,
                     int nl, int stride, const void *k, const void *val, cudaStream_t s) {
  by_shape(v.dh, dtype, [&](auto dh, auto t) {
    using T = decltype(t);
    // KV heads fastest: neighbouring CTAs read neighbouring rows (by CTAs of 256 threads 67.4 us for
    // 5000 entries of 28 layers of 4; pages fastest 69.7)
    const dim3 grid(v.G, nl, rows.list.n_seg);
    if (rows.inlined)
      launch_pdl(k_c8_write<dh, T, PackedList>, grid, WRITE_NT, 0, s, v, rows.list, len, shift, l0, stride,
                 (const T *)k, (const T *)val);
    else
      launch_pdl(k_c8_write<dh, T, PackedRun>, grid, WRITE_NT, 0, s, v, (const PackedRun &)rows.list, len,
                 shift, l0, stride, (const T *)k, (const T *)val);
  });
}

void launch_c8_read(const C8View &v, int dtype, const PackedRows &rows, int l0, int nl, void *k,
                    void *val, cudaStream_t s) {
  const bool wide = ((uintptr_t)k | (uintptr_t)val) % 32 == 0;
  by_shape(v.dh, dtype, [&](auto dh, auto t) {
    using T = decltype(t);
    // pages fastest: neighbouring CTAs read neighbouring blocks (by stores of 16 bytes 74 us for 5000
    // entries of 28 layers of 4; KV heads fastest 78)
    const dim3 grid(rows.list.n_seg, nl, v.G);
    auto run = [&](auto w) {
      if (rows.inlined)
        launch_pdl(k_c8_read<dh, T, w, PackedList>, grid, NT, 0, s, v, rows.list, l0, (T *)k, (T *)val);
      else
        launch_pdl(k_c8_read<dh, T, w, PackedRun>, grid, NT, 0, s, v, (const PackedRun &)rows.list, l0,
                   (T *)k, (T *)val);
    };
    if (wide)
      run(std::true_type{});
    else
      run(std::false_type{});
  });
}

void launch_c8_clear(const C8View &v, size_t blocks, cudaStream_t s) {
  k_c8_clear<<<(unsigned)((blocks + 255) / 256), 256, 0, s>>>(v.power, blocks);
}

void launch_c8_entries(const C8View &v, int len, int l0, int nl, int32_t *number, float *weight,
                       cudaStream_t s) {
  launch_pdl(k_c8_entries, dim3((len + NT - 1) / NT, nl * v.G), NT, 0, s, v, len, l0, number, weight,
             (const float *)nullptr);
}
void launch_c8_set_weights(const C8View &v, int len, int l0, int nl, const float *weight,
                           cudaStream_t s) {
  launch_pdl(k_c8_entries, dim3((len + NT - 1) / NT, nl * v.G), NT, 0, s, v, len, l0,
             (int32_t *)nullptr, (float *)nullptr, weight);
}

const char *launch_c8_choose(const C8View &v, int len, int L, int keep, int first, int recent,
                             int32_t *kept, cudaStream_t s) {
  constexpr int MOST = 50000;  // keys in shared memory beside the bins
  static PerDevice<size_t> limit;
  const size_t smem = (size_t)len * 4;
  if (len > MOST) {
    launch_pdl(k_c8_choose<false>, dim3(L * v.G), CT, 0, s, v, len, keep, first, recent, kept);
    return nullptr;
  }
  if (smem > 32 * 1024)
    if (const char *e = smem_opt_in(limit, k_c8_choose<true>, smem)) return e;
  launch_pdl(k_c8_choose<true>, dim3(L * v.G), CT, smem, s, v, len, keep, first, recent, kept);
  return nullptr;
}

const char *launch_c8_keep(const C8View &src, const C8View &dst, int len, int L, const int32_t *kept,
                           int n, int num_sms, cudaStream_t s) {
  const bool same = src.blocks == dst.blocks;
  const int blocks = (n + KVR_PAGE - 1) / KVR_PAGE, heads = L * src.G;
  int x = blocks;
  if (same)
    for (x = 1; x < 8 && x < blocks && x * heads < 4 * num_sms;) x *= 2;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(x, heads);
  cfg.blockDim = dim3(KEEP_NT);
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = g_pdl ? 1 : 0;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = x;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = same ? 2 : 1;
  auto *kernel = src.dh == 128 ? (same ? k_c8_keep<128, true> : k_c8_keep<128, false>)
                               : (same ? k_c8_keep<64, true> : k_c8_keep<64, false>);
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, src, dst, len, kept, n);
  return e == cudaSuccess ? nullptr : cudaGetErrorString(e);
}

}  // namespace kvr
