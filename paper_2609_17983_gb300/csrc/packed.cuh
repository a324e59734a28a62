// packed.cuh -- a document's K/V in 4 bits: the stored form and its device helpers.
//
// Values.  Groups of 16 consecutive entries of head_dim share a scale.  With a the
// group's largest magnitude, s = a / 6 rounded to 5 exponent and 3 mantissa bits (to
// nearest, ties to even; at most PACK_MAX_SCALE): a half without its sign and low
// seven bits, so its bits are the code << 7.  An entry's code is x / s rounded (to nearest,
// ties to the even code) to one of {0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign, saturating.
// The value code * s has at most six significant bits: exact in half, bf16 and float.
// A row (position, KV head, K or V) that holds a NaN or an infinity has the scale code
// PACK_NAN throughout and reads back as NaN.
//
// Layout.  64 positions (a page) of one layer and KV head are one block of 72 * dh
// bytes; blocks lie [layer][kv head][page].  A block is K codes, K scales, V codes,
// V scales, in the order in which a warp's m16n8k16 products take them: with lane =
// 4 g + t, tile kt of 16 keys and tile db of 16 entries,
//   K codes   [kt][db / 4][lane][db % 4] 32-bit words: low half-word the four entries
//             db*16 + 4t .. of key kt*16 + key_of(g), high half-word those of the key
//             two further; entry i in bits 4i .. 4i + 3;
//   K scales  [kt][g][high][db] bytes;
//   V codes   [db][lane ^ db][kt] words: low half-word the four keys kt*16 + 4t .. of entry
//             db*16 + g, high half-word those of entry db*16 + g + 8 (lane ^ db: the
//             units of a column of db's lie in different banks for kernels that
//             take a row apart);
//   V scales  [db][t][kt][j] bytes, j the key of the four.
// Slots that nothing wrote are zero (scale 0, value 0).
//
// Bounds.  Per block the largest and the least value of each key entry over the
// finite rows present, as whole numbers hi = ceil(max / u), lo = floor(min / u) of
// the smallest power of two u with every magnitude <= 127 u: [layer][kv head][page][hi, lo][dh]
// bytes, and u (float) [layer][kv head][page].
#pragma once

#include <cuda_fp16.h>

#include <exception>
#include <new>

#include "kvr_internal.cuh"

namespace kvr {

constexpr int PACK_GROUP = 16;
constexpr int PACK_NAN = 0xFF;
constexpr int PACK_MAX_CODE = 0xE2;         // the scale 10240: 6 * 10240 is still a half
constexpr float PACK_MAX_SCALE = 10240.f;

__host__ __device__ constexpr int pack_half_bytes(int dh) { return 36 * dh; }  // K or V of a block
__host__ __device__ constexpr int pack_code_bytes(int dh) { return 32 * dh; }
__host__ __device__ constexpr int pack_block_bytes(int dh) { return 72 * dh; }

// Key (of a tile of 16) whose entries are the low half-words of lanes 4g .. 4g + 3.
__host__ __device__ constexpr int pack_key_of(int g) { return 4 * (g >> 1) + (g & 1); }

// Byte offsets within a block's K half: the half-word of (key, entries e4 .. e4 + 3),
// and the scale of (key, db).
__host__ __device__ inline int pack_k_code(int dh, int key, int e4) {
  const int kt = key >> 4, r = key & 15, g = 2 * (r >> 2) + (r & 1), hi = (r >> 1) & 1;
  const int db = e4 >> 4, t = (e4 & 15) >> 2;
  return (((kt * (dh / 64) + (db >> 2)) * 32 + 4 * g + t) * 4 + (db & 3)) * 4 + 2 * hi;
}
__host__ __device__ inline int pack_k_scale(int dh, int key, int db) {
  const int kt = key >> 4, r = key & 15, g = 2 * (r >> 2) + (r & 1), hi = (r >> 1) & 1;
  return pack_code_bytes(dh) + ((kt * 8 + g) * 2 + hi) * (dh / 16) + db;
}
// Within the V half: the half-word of (keys 4 * key4 .. + 3, entry), and the scale
// of (key, db).
__host__ __device__ inline int pack_v_code(int key4, int entry) {
  const int db = entry >> 4, r = entry & 15, lane = 4 * (r & 7) + (key4 & 3);
  return ((db * 32 + (lane ^ db)) * 4 + (key4 >> 2)) * 4 + 2 * (r >> 3);
}
__host__ __device__ inline int pack_v_scale(int dh, int key, int db) {
  return pack_code_bytes(dh) + ((db * 4 + ((key & 15) >> 2)) * 4 + (key >> 4)) * 4 + (key & 3);
}

// Device view of one packed document.
struct PackedView {
  uint8_t *blocks;
  int8_t *bounds;
  float *unit;
  int pages;  // capacity
  int G, dh;
  __host__ __device__ size_t index(int layer, int g, int page) const {
    return ((size_t)layer * G + g) * pages + page;
  }
  __host__ __device__ uint8_t *block(int layer, int g, int page) const {
    return blocks + index(layer, g, page) * pack_block_bytes(dh);
  }
};

// The cluster's barrier in two steps: what a thread wrote before its arrival, in whosever
// memory, all see after their wait.
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}

// The values of a word's eight codes, a half2 (low nibble first) for each byte.  Taken
// apart into bytes by one mov, the conversions read them where they lie; extracted by
// shifts each cost one more ALU instruction (15 clocks a word instead of 10.5).
__device__ __forceinline__ void pack_values(uint32_t w, uint32_t *v) {
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
      : "r"(w));
}

// The codes of eight entries over their scale, low nibble first.
__device__ __forceinline__ uint32_t pack_codes(const float *y) {
  uint32_t r;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(r)
      : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
  return r;
}

// Scale of a group whose largest magnitude is a (finite), as its code.  The rounding to
// three mantissa bits is done on the float's own bits, below 2^-14 in whole steps of
// 2^-17.
__device__ __forceinline__ uint32_t pack_scale_code(float a) {
  const float s = fminf(__fdiv_rn(a, 6.f), PACK_MAX_SCALE);
  if (s < 6.103515625e-05f) return (uint32_t)__float2int_rn(s * 131072.f);  // 2^-14, 2^17
  uint32_t u = __float_as_uint(s);
  u = (u + 0x7FFFFu + ((u >> 20) & 1u)) >> 20;  // exponent and three mantissa bits
  return u - ((127 - 15) << 3);
}
// The same for a bf16 a.  a / 6 of an eight-bit a is a midpoint of the scales or at least
// 2^-8 of itself away from one, so rounded to a half (2^-11) the product with the
// rounded 1 / 6 is on a midpoint exactly where it should be; halves below 2^-14 are too
// coarse for that.
__device__ __forceinline__ uint32_t pack_scale_code_bf16(float a) {
  if (a < 6.f * 6.103515625e-05f) return pack_scale_code(a);
  const uint32_t h = __half_as_ushort(__float2half_rn(a * (1.f / 6.f)));
  return min((h + 0x3Fu + ((h >> 7) & 1u)) >> 7, (uint32_t)PACK_MAX_CODE);
}
__device__ __forceinline__ float pack_scale(uint32_t code) {
  return __half2float(__ushort_as_half((unsigned short)(code << 7)));
}

// ---- kernels (k_packed.cu, k_packed_attn.cu) ----

// Positions of a call in segments of one page each: a run of consecutive positions, or
// a list, which comes with the launch when it is short and else lies in device memory.
constexpr int PACK_INLINE_POS = 512;
struct PackedRun {
  int n = 0, n_seg = 0, most = 0;  // most: rows of a list's fullest segment
  int first = -1;                  // >= 0: positions first .. first + n - 1
  const int32_t *pos_d = nullptr;  // else device [n], then segment starts [n_seg + 1]
};
struct PackedList : PackedRun {
  uint16_t seg[PACK_INLINE_POS + 1];
  int32_t pos[PACK_INLINE_POS];
};
// Short lists are the only ones that need more than the run's few bytes of arguments.
struct PackedRows {
  PackedList list;
  bool inlined = false;
};
// k, v: [n][nl][G][dh] in the model dtype; len: the document's length after the write.
// Returns the kernels launched.
int launch_packed_write(const PackedView &v, int dtype, const PackedRows &rows, int len, int l0,
                        int nl, const void *k, const void *val, int sms, cudaStream_t s);
void launch_packed_read(const PackedView &v, int dtype, const PackedRows &rows, int l0, int nl,
                        void *k, void *val, cudaStream_t s);

// A tile of the attention is up to 8 query vectors (row * heads per KV head + head) of
// rows of one document; its pages are dealt to parts, a CTA each.
constexpr int PACK_VEC = 8;
constexpr int PACK_CLUSTER = 8;  // parts whose sums meet in shared memory, at most
constexpr int PACK_MERGE = 1024;  // clusters of a tile: their weights lie in a CTA's memory
struct PackedPart {
  const uint8_t *blocks;  // the document's
  int32_t pages;          // its capacity
  int32_t vec0, nvec;
  int32_t page0, page1;
  int32_t part, n_parts;  // of the tile
  int32_t slot;           // the tile's first part among all
  int32_t tile, pad[3];
};
struct PackedRow {
  PackedView doc;
  int32_t pos, pad;
};
struct PackedAttnArgs {
  const void *q;
  void *out;
  int ldq;                  // row stride of q in elements
  int dtype, H, G, grp, dh, layer;
  float scale;              // log2(e) / sqrt(dh)
  const int32_t *pos;       // device [rows]
  const PackedRow *rows;    // device [rows]
  // dense
  const PackedPart *parts;
  int n_parts;
  int warps, cluster;       // of a CTA, CTAs of a cluster: parts of a tile come in whole clusters
  // sparse: blocks [rows][G][n_blocks]
  const int32_t *blocks;
  int n_rows, n_blocks, parts_per_row;
  float *ws_o;      // [cluster][G][PACK_VEC][dh]
  float2 *ws_ml;    // [cluster][G][PACK_CLUSTER][PACK_VEC]
  int *counters;    // [tile][G][PACK_CLUSTER], zero between calls
  int *dev_flag;
  int num_sms;
  bool settled;     // the tables were sent before the kernel that precedes this one
};
int packed_attn_ctas_per_sm(int dtype, int warps);  // CTAs of 4, or 12 (fp32: 8), warps
int packed_attn_max_blocks_per_part();
const char *launch_packed_attention(const PackedAttnArgs &a, cudaStream_t s);
// Blocks of each (row, KV head): blocks [rows][G][n_blocks].
const char *launch_packed_select(const PackedAttnArgs &a, int max_pages, int32_t *blocks,
                                 cudaStream_t s);

// An entry point's body: no C++ exception passes it (host memory that cannot be had is
// KVR_E_NOMEM); `undo` runs after one.
template <class F, class U>
kvr_status guarded(F body, U undo) {
  try {
    return body();
  } catch (const std::bad_alloc &) {
    undo();
    set_last_error("out of host memory");
    return KVR_E_NOMEM;
  } catch (const std::exception &e) {
    undo();
    set_last_error(e.what());
    return KVR_E_INVAL;
  }
}
template <class F>
kvr_status guarded(F body) {
  return guarded(body, [] {});
}

// ---- of api.cu, for the packed entry points ----
// words of 32 bits to the device, ahead of what is queued next on the model's stream
kvr_status upload_words(kvr_model *m, void *dst, const void *src, size_t words);
kvr_status grow_device(kvr_model *m, void *&buf, size_t &have, size_t need, const char *what);
kvr_status synchronize(kvr_model *m);
kvr_status flush_uploads(kvr_model *m);

// Many rows of one document over unpacked pages: the plan of the tensor-core attention
// for rows at ascending positions >= 0 (its tables, int4, to be sent to the device), and
// its launch on pages [page][K, V][G][KVR_PAGE][dh] of one layer.
struct ManyPlan {
  int rows = 0, n_blocks = 0, n_pairs = 0, splits = 1, block_rows = 0, pages = 0;
};
bool many_plan(const kvr_model *m, const int32_t *pos, int rows, std::vector<int32_t> &tables,
               ManyPlan &p);
kvr_status many_attention(kvr_model *m, const ManyPlan &p, const int4 *tables, const void *q,
                          int ldq, const int32_t *pos, void *pages, const int32_t *identity,
                          void *out);
// The first n_pages blocks of a layer as such pages, in halves.  A key row stored as NaN,
// or whose value row is, becomes NaN; NaN value rows become zero.
void launch_packed_unpack(const PackedView &v, int layer, int n_pages, void *pages, bool settled,
                          cudaStream_t s);

}  // namespace kvr

// A document's packed cache.
struct kvr_packed {
  kvr_model *model = nullptr;
  int n = 0, cap = 0, pages = 0;
  std::vector<int32_t> tokens_h;  // of a document that was packed (kvr_pack), else empty
  int32_t *tokens_d = nullptr;    // device [cap]
  uint8_t *blocks = nullptr;
  int8_t *bounds = nullptr;
  float *unit = nullptr;
  bool poisoned = false;
  kvr::PackedView view() const {
    return kvr::PackedView{blocks, bounds, unit, pages, model->dims.G, model->dims.dh};
  }
};

// Query rows over packed documents: the tables of a pass, used by every layer of it.
struct kvr_rows {
  struct Many {  // rows [row0, row0 + plan.rows) of a document, by way of unpacked pages
    int doc, row0;
    size_t table;  // int32 words into many_d
    kvr::ManyPlan plan;
  };
  std::vector<Many> many;
  int32_t *many_d = nullptr, *identity_d = nullptr;
  kvr_model *model = nullptr;
  std::vector<kvr_packed *> docs;  // null: freed since
  std::vector<int32_t> doc_rows, pos;
  int n_parts = 0, n_tiles = 0, max_pages = 0, warps = 0, cluster = 0;
  // how lists of n blocks are dealt (attend_blocks); n = 0: not yet
  struct {
    int n = 0, warps = 0, per = 0, cluster = 0;
  } lists;
  bool merged = false;   // some tile has more than one cluster
  bool sent = false;     // the device holds the tables of pos
  bool settled = false;  // and a kernel was launched behind their upload
  void *mem = nullptr;  // device tables
  size_t mem_bytes = 0;
  kvr::PackedPart *parts_d = nullptr;
  kvr::PackedRow *rows_d = nullptr;
  int32_t *pos_d = nullptr;
};

namespace kvr {

// ---- of packed.cu, for the passes of api.cu ----
kvr_status packed_rows_of(kvr_model *m, const int32_t *pos, int n, PackedRows &rows);
// The model's own rows over one document, at positions (ascending) that may lie past
// its length; their tables are queued for upload.
kvr_status packed_pass_rows(kvr_packed *c, const int32_t *pos, int n, kvr_rows **out);
// Attention of layer `layer` over all positions, or (n_blocks > 0) the selected blocks.
kvr_status packed_attend(kvr_rows *r, int layer, const void *q, void *out, int n_blocks);
// The bounds of one page over its slots below the length len, of layers [0, nl) without
// [l0, l1).
void launch_packed_bounds(const PackedView &v, int page, int len, int nl, int l0, int l1,
                          cudaStream_t s);
// Positions [len, end), the last ones with anything written, as if nothing had been: zeros,
// and their blocks' bounds over the positions before; of layers [0, nl).
void launch_packed_clear(const PackedView &v, int len, int end, int nl, cudaStream_t s);
// The units of n blocks of zeros.
void launch_packed_units(float *unit, size_t n, cudaStream_t s);

}  // namespace kvr
