// packed.cu -- the packed cache's entry points: documents held in 4 bits, their rows
// written and read back, and query rows that attend to them.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>

#include "packed.cuh"

using namespace kvr;

namespace {

static_assert(KVR_BLOCK == KVR_PAGE, "a block is a page");
constexpr int MAX_CAPACITY = 1 << 20;  // positions of a packed cache
constexpr int MAX_ROWS = 1 << 20, MAX_DOCS = 4096, MAX_BLOCKS = MAX_CAPACITY / KVR_PAGE;

kvr_status fail(kvr_status code, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return code;
}

#define KVR_TRY(expr)              \
  do {                             \
    kvr_status s__ = (expr);       \
    if (s__ != KVR_OK) return s__; \
  } while (0)

kvr_status use_device(const kvr_model *m) {
  const cudaError_t e = cudaSetDevice(m->device);
  return e == cudaSuccess ? KVR_OK : fail(KVR_E_CUDA, "cudaSetDevice: %s", cudaGetErrorString(e));
}

kvr_status launched(kvr_model *m, int kernels, const char *what) {
  m->launches += kernels;
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? KVR_OK : fail(KVR_E_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// Device or managed memory that `device` can use, on a 16-byte boundary.
kvr_status check_device_ptr(const kvr_model *m, const void *p, const char *name) {
  if (!p) return fail(KVR_E_INVAL, "NULL %s", name);
  if ((uintptr_t)p & 15) return fail(KVR_E_INVAL, "%s is not 16-byte aligned", name);
  cudaPointerAttributes a{};
  if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
    cudaGetLastError();
    return fail(KVR_E_INVAL, "%s is not device memory", name);
  }
  if (a.type == cudaMemoryTypeManaged || (a.type == cudaMemoryTypeDevice && a.device == m->device))
    return KVR_OK;
  return fail(KVR_E_INVAL, "%s is not memory of the model's device", name);
}

// Positions of a call (ascending) in segments of a page each; many scattered ones go to
// the model's readback scratch.
kvr_status rows_of(kvr_model *m, const int32_t *pos, int n, PackedRows &rows) {
  PackedList &r = rows.list;
  r.n = n;
  if (pos[n - 1] - pos[0] == n - 1) {
    r.first = pos[0];
    r.n_seg = pos[n - 1] / KVR_PAGE - pos[0] / KVR_PAGE + 1;
    return KVR_OK;
  }
  for (int i = 0, at = 0; i < n; ++i) {
    if (pos[i] / KVR_PAGE != pos[at] / KVR_PAGE) at = i;
    r.most = std::max(r.most, i - at + 1);
  }
  rows.inlined = n <= PACK_INLINE_POS;
  if (rows.inlined) {
    for (int i = 0; i < n; ++i)
      if (!i || pos[i] / KVR_PAGE != pos[i - 1] / KVR_PAGE) r.seg[r.n_seg++] = (uint16_t)i;
    r.seg[r.n_seg] = (uint16_t)n;
    memcpy(r.pos, pos, n * sizeof(int32_t));
    return KVR_OK;
  }
  std::vector<int32_t> all(pos, pos + n);
  for (int i = 0; i < n; ++i)
    if (!i || pos[i] / KVR_PAGE != pos[i - 1] / KVR_PAGE) all.push_back(i);
  r.n_seg = (int)all.size() - n;
  all.push_back(n);
  KVR_TRY(grow_device(m, m->read_scratch, m->read_scratch_bytes, all.size() * 4,
                      "readback scratch"));
  KVR_TRY(upload_words(m, m->read_scratch, all.data(), all.size()));
  r.pos_d = (const int32_t *)m->read_scratch;
  return KVR_OK;
}

kvr_status check_range(const kvr_model *m, const int32_t *positions, int n, int l0, int l1,
                       int end) {
  if (n < 0) return fail(KVR_E_RANGE, "negative number of positions");
  if (l0 < 0 || l1 > m->dims.L || l0 > l1)
    return fail(KVR_E_RANGE, "layers [%d, %d) outside [0, %d)", l0, l1, m->dims.L);
  if (n > 0 && !positions) return fail(KVR_E_INVAL, "NULL positions");
  for (int i = 0; i < n; ++i) {
    if (positions[i] < 0 || positions[i] >= end)
      return fail(KVR_E_RANGE, "position %d outside [0, %d)", positions[i], end);
    if (i && positions[i] <= positions[i - 1])
      return fail(KVR_E_RANGE, "positions not strictly increasing at %d", i);
  }
  return KVR_OK;
}

// ------------------------------------------------------------ query rows

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

kvr_status check_rows(const std::vector<kvr_packed *> &docs, const std::vector<int32_t> &doc_rows,
                      const int32_t *pos, size_t count) {
  size_t i = 0;
  for (size_t d = 0; d < docs.size(); ++d)
    for (int r = 0; r < doc_rows[d]; ++r, ++i) {
      if (pos[i] < -1 || pos[i] >= docs[d]->n)
        return fail(KVR_E_RANGE, "row %zu: position %d outside [-1, %d)", i, pos[i], docs[d]->n);
      if (r && pos[i] < pos[i - 1])
        return fail(KVR_E_RANGE, "row %zu: positions of a document descend", i);
    }
  return i == count ? KVR_OK : fail(KVR_E_RANGE, "row counts do not match");
}

// How tiles of `pages` pages each (times G KV heads) are dealt to the chip: warps of a
// CTA, pages of a part, parts of a cluster.
struct Deal {
  int warps, per, cluster;
  int parts(int np) const {
    const int n = std::max(1, (np + per - 1) / per);
    return (n + cluster - 1) / cluster * cluster;
  }
};

// The deal whose launch is modelled to end first, in units of 10 ns.  A wave of CTAs costs
// 2.8 us beside its rounds (a page for each of a CTA's warps), a round 1.5; a cluster's
// sums 1.4, a merge through memory 2.5 and 0.07 per cluster; clusters of 8 leave 7/20 of
// the SMs without a place.  Of 8179 launches of 220 calls (1 to 64 rows over 64 to 131072
// positions, up to 16 documents, both types) the deal taken is 3.4% slower than the fastest
// of its call on average, 18% at most (three rows over 1125 positions, 4 heads: 5.2 us, in
// clusters of 8 CTAs of 4 warps 4.4).  One token over 5000 positions, 4 KV heads: 8 CTAs
// of 12 warps as a cluster 6.3 us (merged through memory 8.0, with 4 warps 7.6); over
// 131072, 8 KV heads: 19 CTAs of 12 warps a head 30.7 (in clusters of 2 32.2); 16 documents
// of 8191: a CTA a document and head 30.5 (with 4 warps 33.2).
Deal deal(const kvr_model *m, const std::vector<std::pair<int, int>> &pages, int G) {
  const int many = m->dims.dtype == KVR_DTYPE_BF16 ? 12 : 8;
  int most = 1;
  for (const auto &x : pages) most = std::max(most, x.first);
  Deal best{};
  long long least = -1;
  for (int W : {many, 4}) {
    const int per_sm = packed_attn_ctas_per_sm(m->dims.dtype, W);
    for (int rounds = 1;; rounds += 1 + rounds / 12) {
      for (int cl = 1; cl <= PACK_CLUSTER; cl *= 2) {
        const Deal d{W, W * rounds, cl};
        if (cl > 1 && cl / 2 * d.per >= most) break;  // half the cluster would do
        long long ctas = 0;
        for (const auto &x : pages) ctas += (long long)d.parts(x.first) * x.second * G;
        const long long slots = std::max<long long>(
            cl, (long long)m->num_sms * per_sm * (cl == 8 ? 13 : 20) / 20);
        const long long waves = (ctas + slots - 1) / slots;
        const int parts = d.parts(most), nc = parts / cl, each = (most + parts - 1) / parts;
        if (nc > PACK_MERGE) continue;
        const int deep = std::max(1, (each + W - 1) / W);
        const long long t =
            waves * (280 + deep * 150) + (cl > 1 ? 140 : 0) + (nc > 1 ? 250 + 7 * nc : 0);
        if (least < 0 || t < least) least = t, best = d;
      }
      if (W * rounds >= most) break;
    }
  }
  return best;
}

// Whether the rows of a document at `pos` (ascending, >= 0) go by way of unpacked pages: one
// kernel widens the layer's blocks to pages of halves, and the tcgen05 attention takes a tile of
// 128 vectors at a time where the fused kernel takes 8.  Units are (page, tile of 8 vectors,
// KV head); where the other way is shorter was fitted to launches by both, of 8 to 4096 rows
// over 512 to 12345 positions.  One document (270 launches): the way taken is 0.3% slower than
// the other on average, 24% at most (40 rows spread over 12345 positions, 32 heads: 38.1 us
// by pages, 30.7 fused; over 5000, 28 heads, 20.6 and 15.5; the last 64 23.6 and 28.2; a
// chunk of 4096 rows over 12345 480 and 2813).  Several, with as many rows each, share the
// fused kernel's launch and are unpacked one after another (756 launches of 2, 4 and 8):
// 0.4% and 32% (eight times the last 96 rows over 2000 positions, 28 heads: 159 us by pages,
// 120 fused; two times 512 over 512, 32 heads, 31.0 and 54.2).
bool many_rows(const kvr_model *m, const int32_t *pos, int rows, size_t docs) {
  const Dims &dm = m->dims;
  if (dm.dtype != KVR_DTYPE_BF16 || rows < 1) return false;
  const int grp = dm.H / dm.G;
  long long units = 0;
  for (int v = 0; v < rows * grp; v += PACK_VEC)
    units += pos[std::min(rows * grp - 1, v + PACK_VEC - 1) / grp] / KVR_PAGE + 1;
  const long long n = pos[rows - 1] + 1;
  const long long least = docs == 1 ? (dm.dh == 128 ? 6600 + n * 2 / 5 : 5000 + n * 26 / 25)
                          : dm.dh == 128
                              ? 7500 + n * 11 / 10
                              : 7000 + n + 2000 * (long long)std::min<size_t>(docs, 8);
  return units * dm.G > least;
}

// The tables of rows at `pos`, built and sent.
kvr_status build_rows(kvr_rows *r, const int32_t *pos) {
  kvr_model *m = r->model;
  const Dims &dm = m->dims;
  const int grp = dm.H / dm.G, M = (int)r->pos.size(), D = (int)r->docs.size();
  std::vector<PackedPart> tiles;  // page1: all of the tile's
  std::vector<PackedRow> rows(M);
  std::vector<int> pages;
  std::vector<int32_t> tables;
  std::vector<kvr_rows::Many> many;
  int row0 = 0, most = 1, many_pages = 0;
  for (int d = 0; d < D; ++d) {
    const int R = r->doc_rows[d];
    const PackedView view = r->docs[d]->view();
    for (int i = row0; i < row0 + R; ++i) rows[i] = PackedRow{view, pos[i], 0};
    int few = R;  // rows that the fused kernel takes: the first ones
    {
      const int none = (int)(std::lower_bound(pos + row0, pos + row0 + R, 0) - (pos + row0));
      kvr_rows::Many x{d, row0 + none, tables.size(), {}};
      if (many_rows(m, pos + row0 + none, R - none, r->docs.size()) &&
          many_plan(m, pos + row0 + none, R - none, tables, x.plan)) {
        few = none;
        many.push_back(x);
        many_pages = std::max(many_pages, x.plan.pages);
        most = std::max(most, x.plan.pages);
      }
    }
    for (int v = 0; v < few * grp; v += PACK_VEC) {
      PackedPart t{};
      t.blocks = view.blocks;
      t.pages = view.pages;
      t.vec0 = row0 * grp + v;
      t.nvec = std::min(PACK_VEC, few * grp - v);
      const int last = pos[(t.vec0 + t.nvec - 1) / grp];  // positions ascend
      t.page1 = last < 0 ? 0 : last / KVR_PAGE + 1;
      t.tile = (int)tiles.size();
      tiles.push_back(t);
      pages.push_back(t.page1);
      most = std::max(most, t.page1);
    }
    row0 += R;
  }
  std::sort(pages.begin(), pages.end());
  std::vector<std::pair<int, int>> count;  // tiles of so many pages
  for (int np : pages) {
    if (count.empty() || count.back().first != np) count.push_back({np, 0});
    ++count.back().second;
  }
  const Deal dl = deal(m, count, dm.G);
  std::vector<PackedPart> parts;
  bool merged = false;
  for (const PackedPart &t : tiles) {
    PackedPart x = t;
    x.slot = (int)parts.size();
    x.n_parts = dl.parts(t.page1);
    merged = merged || x.n_parts > dl.cluster;
    for (x.part = 0; x.part < x.n_parts; ++x.part) {
      x.page0 = (int)((long long)t.page1 * x.part / x.n_parts);
      x.page1 = (int)((long long)t.page1 * (x.part + 1) / x.n_parts);
      parts.push_back(x);
    }
  }
  const size_t o_row = up256(parts.size() * sizeof(PackedPart)),
               o_pos = up256(o_row + M * sizeof(PackedRow)), o_many = up256(o_pos + M * 4ull),
               o_id = up256(o_many + tables.size() * 4), bytes = up256(o_id + many_pages * 4ull);
  std::vector<char> host(bytes);
  memcpy(host.data(), parts.data(), parts.size() * sizeof(PackedPart));
  memcpy(host.data() + o_row, rows.data(), M * sizeof(PackedRow));
  memcpy(host.data() + o_pos, pos, M * 4ull);
  memcpy(host.data() + o_many, tables.data(), tables.size() * 4);
  for (int i = 0; i < many_pages; ++i) ((int32_t *)(host.data() + o_id))[i] = i;
  r->sent = r->settled = false;
  r->lists.n = 0;
  KVR_TRY(grow_device(m, r->mem, r->mem_bytes, bytes, "query rows"));
  KVR_TRY(upload_words(m, r->mem, host.data(), bytes / 4));
  char *base = (char *)r->mem;
  r->parts_d = (PackedPart *)base;
  r->rows_d = (PackedRow *)(base + o_row);
  r->pos_d = (int32_t *)(base + o_pos);
  r->many_d = (int32_t *)(base + o_many);
  r->identity_d = (int32_t *)(base + o_id);
  r->many = std::move(many);
  r->n_parts = (int)parts.size();
  r->n_tiles = (int)tiles.size();
  r->max_pages = most;
  r->merged = merged;
  r->warps = dl.warps;
  r->cluster = dl.cluster;
  std::copy(pos, pos + M, r->pos.begin());
  r->sent = true;
  return KVR_OK;
}

// Room for the partial sums and arrival counts of a launch, where a tile has more than one
// cluster's to add.
kvr_status attn_workspace(kvr_model *m, PackedAttnArgs &a, long long parts, long long tiles,
                          bool merged) {
  if (!merged) return KVR_OK;
  const size_t sums = (size_t)(parts / a.cluster) * a.G,
               o = up256(sums * PACK_VEC * a.dh * sizeof(float)),
               ml = sums * PACK_CLUSTER * PACK_VEC * sizeof(float2),
               cb = (size_t)tiles * a.G * PACK_CLUSTER * sizeof(int);
  if (o + ml > m->pack_ws_bytes)
    KVR_TRY(grow_device(m, m->pack_ws, m->pack_ws_bytes, o + ml, "packed attention workspace"));
  if (cb > m->pack_count_bytes) {
    KVR_TRY(grow_device(m, m->pack_count, m->pack_count_bytes, cb, "packed attention counters"));
    if (cudaMemsetAsync(m->pack_count, 0, cb, m->stream) != cudaSuccess)
      return fail(KVR_E_CUDA, "packed attention counters");
  }
  a.ws_o = (float *)m->pack_ws;
  a.ws_ml = (float2 *)((char *)m->pack_ws + o);
  a.counters = (int *)m->pack_count;
  return KVR_OK;
}

// What the kernels of a call on rows take.
PackedAttnArgs kernel_args(const kvr_rows *r, int layer, const void *q, int ldq) {
  const kvr_model *m = r->model;
  const Dims &dm = m->dims;
  PackedAttnArgs a{};
  a.q = q;
  a.ldq = ldq;
  a.dtype = dm.dtype;
  a.H = dm.H, a.G = dm.G, a.grp = dm.H / dm.G, a.dh = dm.dh;
  a.layer = layer;
  a.scale = (float)(1.4426950408889634 / std::sqrt((double)dm.dh));
  a.pos = r->pos_d;
  a.rows = r->rows_d;
  a.parts = r->parts_d;
  a.n_parts = r->n_parts;
  a.warps = r->warps;
  a.cluster = r->cluster;
  a.settled = r->settled;
  a.n_rows = (int)r->pos.size();
  a.dev_flag = m->dev_flag;
  a.num_sms = m->num_sms;
  return a;
}

// The same after the checks common to the calls.
kvr_status rows_args(kvr_rows *r, int32_t layer, const void *q, int32_t ldq, PackedAttnArgs &a) {
  if (!r) return fail(KVR_E_INVAL, "NULL rows");
  kvr_model *m = r->model;
  const Dims &dm = m->dims;
  if (layer < 0 || layer >= dm.L) return fail(KVR_E_RANGE, "layer %d outside [0, %d)", layer, dm.L);
  for (const kvr_packed *d : r->docs) {
    if (!d) return fail(KVR_E_INVAL, "a document of these rows has been freed");
    if (d->poisoned) return fail(KVR_E_POISONED, "packed cache poisoned");
  }
  if (!r->sent) return fail(KVR_E_INVAL, "rows whose last move failed");
  if (ldq < dm.H * dm.dh || ldq * dm.es() % 16)
    return fail(KVR_E_INVAL, "row stride %d of q: at least %d, whole 16-byte pieces", ldq,
                dm.H * dm.dh);
  KVR_TRY(use_device(m));
  KVR_TRY(check_device_ptr(m, q, "q"));
  a = kernel_args(r, layer, q, ldq);
  return KVR_OK;
}

// Attention over all positions (a: rows_args').
kvr_status attend_all(kvr_rows *r, PackedAttnArgs &a, void *out) {
  kvr_model *m = r->model;
  const void *q = a.q;
  const int ldq = a.ldq, layer = a.layer;
  a.out = out;
  if (r->n_parts) {
    KVR_TRY(attn_workspace(m, a, r->n_parts, r->n_tiles, r->merged));
    if (const char *e = launch_packed_attention(a, m->stream))
      return fail(KVR_E_CUDA, "packed attention: %s", e);
    KVR_TRY(launched(m, 1, "packed attention"));
    r->settled = true;
  }
  const Dims &dm = m->dims;
  const size_t row_b = (size_t)dm.H * dm.dh * dm.es(),
               page_b = (size_t)2 * dm.G * KVR_PAGE * dm.dh * 2;
  for (const kvr_rows::Many &x : r->many) {
    KVR_TRY(grow_device(m, m->pack_pages, m->pack_pages_bytes, x.plan.pages * page_b,
                        "unpacked pages"));
    launch_packed_unpack(r->docs[x.doc]->view(), layer, x.plan.pages, m->pack_pages, r->settled,
                         m->stream);
    KVR_TRY(launched(m, 1, "unpack"));
    r->settled = true;
    KVR_TRY(many_attention(m, x.plan, (const int4 *)(r->many_d + x.table),
                           (const char *)q + (size_t)x.row0 * ldq * dm.es(), ldq,
                           r->pos_d + x.row0, m->pack_pages, r->identity_d,
                           (char *)out + x.row0 * row_b));
  }
  return KVR_OK;
}

// The blocks of each row.
kvr_status select_blocks(kvr_rows *r, PackedAttnArgs &a, int n_blocks, int32_t *blocks_out) {
  kvr_model *m = r->model;
  a.n_blocks = n_blocks;
  if (const char *e = launch_packed_select(a, r->max_pages, blocks_out, m->stream))
    return fail(KVR_E_CUDA, "block selection: %s", e);
  KVR_TRY(launched(m, 1, "block selection"));
  r->settled = true;
  return KVR_OK;
}

// Attention over listed blocks.  The deal is that of as many pages: over 350 launches of 1 to 64
// rows with lists of 1 to 64 blocks (both types, both head sizes) it is 3.2% slower than the
// fastest on average, 27% at most (40 rows of 64 blocks, fp32, 4 heads of 64: 15.6 us
// against 11.9); 40 rows of 24 blocks, 28 heads 12.6 (the fastest 12.6).
kvr_status attend_blocks(kvr_rows *r, PackedAttnArgs &a, const int32_t *blocks, int n_blocks,
                         void *out) {
  kvr_model *m = r->model;
  a.out = out;
  a.blocks = blocks;
  a.n_blocks = n_blocks;
  const long long tiles = (long long)a.n_rows * ((a.grp + PACK_VEC - 1) / PACK_VEC);
  if (tiles * n_blocks > 0x7FFFFFFF)
    return fail(KVR_E_UNSUPPORTED, "too many rows (%d) for %d blocks each", a.n_rows, n_blocks);
  auto &plan = r->lists;
  if (plan.n != n_blocks) {
    const Deal d = deal(m, {{n_blocks, (int)tiles}}, a.G);
    plan = {n_blocks, d.warps, std::min(d.per, packed_attn_max_blocks_per_part()), d.cluster};
  }
  const Deal dl{plan.warps, plan.per, plan.cluster};
  a.warps = dl.warps;
  a.cluster = dl.cluster;
  a.parts_per_row = dl.parts(n_blocks);
  KVR_TRY(attn_workspace(m, a, tiles * a.parts_per_row, tiles, a.parts_per_row > a.cluster));
  if (const char *e = launch_packed_attention(a, m->stream))
    return fail(KVR_E_CUDA, "block attention: %s", e);
  KVR_TRY(launched(m, 1, "block attention"));
  r->settled = true;
  return KVR_OK;
}

}  // namespace

namespace kvr {

kvr_status packed_rows_of(kvr_model *m, const int32_t *pos, int n, PackedRows &rows) {
  return rows_of(m, pos, n, rows);
}

kvr_status packed_pass_rows(kvr_packed *c, const int32_t *pos, int n, kvr_rows **out) {
  kvr_model *m = c->model;
  if (!m->pass_rows) {
    m->pass_rows = new kvr_rows();
    m->pass_rows->model = m;
    m->rows.push_back(m->pass_rows);
  }
  kvr_rows *r = m->pass_rows;
  r->docs.assign(1, c);
  r->doc_rows.assign(1, n);
  r->pos.assign(pos, pos + n);
  *out = r;
  return build_rows(r, r->pos.data());
}

kvr_status packed_attend(kvr_rows *r, int layer, const void *q, void *out, int n_blocks) {
  kvr_model *m = r->model;
  PackedAttnArgs a = kernel_args(r, layer, q, m->dims.H * m->dims.dh);
  if (!n_blocks) return attend_all(r, a, out);
  KVR_TRY(grow_device(m, m->sel_scratch, m->sel_scratch_bytes,
                      (size_t)a.n_rows * a.G * n_blocks * sizeof(int32_t), "selected blocks"));
  int32_t *blocks = (int32_t *)m->sel_scratch;
  KVR_TRY(select_blocks(r, a, n_blocks, blocks));
  return attend_blocks(r, a, blocks, n_blocks, out);
}

}  // namespace kvr

extern "C" {

kvr_status kvr_packed_create(kvr_model *m, int32_t capacity, kvr_packed **out) {
  kvr_packed *c = nullptr;
  return guarded([&]() -> kvr_status {
    if (!m || !out) return fail(KVR_E_INVAL, "NULL argument");
    *out = nullptr;
    if (capacity < 1 || capacity > MAX_CAPACITY)
      return fail(KVR_E_RANGE, "capacity %d outside [1, %d]", capacity, MAX_CAPACITY);
    KVR_TRY(use_device(m));
    const Dims &dm = m->dims;
    c = new kvr_packed();
    c->model = m;
    m->packed.push_back(c);
    c->cap = capacity;
    c->pages = (capacity + KVR_PAGE - 1) / KVR_PAGE;
    const size_t n = (size_t)dm.L * dm.G * c->pages, block_b = n * pack_block_bytes(dm.dh),
                 bound_b = n * 2 * dm.dh;
    c->blocks = (uint8_t *)dev_alloc(block_b);
    c->bounds = (int8_t *)dev_alloc(bound_b);
    c->unit = (float *)dev_alloc(n * sizeof(float));
    if (!c->blocks || !c->bounds || !c->unit) {
      kvr_packed_free(c);
      return fail(KVR_E_NOMEM, "packed cache of %d positions", capacity);
    }
    if (cudaMemsetAsync(c->blocks, 0, block_b, m->stream) != cudaSuccess ||
        cudaMemsetAsync(c->bounds, 0, bound_b, m->stream) != cudaSuccess) {
      kvr_packed_free(c);
      return fail(KVR_E_CUDA, "packed cache clear");
    }
    launch_packed_units(c->unit, n, m->stream);
    if (const kvr_status st = launched(m, 1, "packed cache clear")) {
      kvr_packed_free(c);
      return st;
    }
    *out = c;
    return KVR_OK;
  }, [&] { kvr_packed_free(c); });
}

void kvr_packed_free(kvr_packed *c) {
  if (!c) return;
  kvr_model *m = c->model;
  cudaSetDevice(m->device);
  flush_uploads(m);
  cudaStreamSynchronize(m->stream);
  m->packed.erase(std::remove(m->packed.begin(), m->packed.end(), c), m->packed.end());
  for (kvr_rows *r : m->rows)
    std::replace(r->docs.begin(), r->docs.end(), c, (kvr_packed *)nullptr);
  dev_free(c->tokens_d);
  dev_free(c->blocks);
  dev_free(c->bounds);
  dev_free(c->unit);
  delete c;
}

int32_t kvr_packed_len(const kvr_packed *c) { return c ? c->n : -1; }

kvr_status kvr_packed_write(kvr_packed *c, const int32_t *positions, int32_t n_pos, int32_t l0,
                            int32_t l1, const void *k, const void *v) {
  return guarded([&]() -> kvr_status {
    if (!c) return fail(KVR_E_INVAL, "NULL packed cache");
    if (c->poisoned) return fail(KVR_E_POISONED, "packed cache poisoned by an earlier CUDA error");
    kvr_model *m = c->model;
    KVR_TRY(check_range(m, positions, n_pos, l0, l1, c->cap));
    for (int i = 0, end = c->n; i < n_pos; ++i) {
      if (positions[i] > end)
        return fail(KVR_E_RANGE, "position %d leaves a gap after %d", positions[i], end);
      end = std::max(end, positions[i] + 1);
    }
    if (n_pos == 0 || l0 == l1) return KVR_OK;
    KVR_TRY(use_device(m));
    KVR_TRY(check_device_ptr(m, k, "k"));
    KVR_TRY(check_device_ptr(m, v, "v"));
    PackedRows rows;
    KVR_TRY(rows_of(m, positions, n_pos, rows));
    const int len = std::max(c->n, positions[n_pos - 1] + 1);
    int n = launch_packed_write(c->view(), m->dims.dtype, rows, len, l0, l1 - l0, k, v, m->num_sms,
                                m->stream);
    // the other layers hold zeros at the new positions: no write of theirs takes the bounds of
    // the block that the length ended in (those behind it are blocks of zeros)
    if (len > c->n && c->n % KVR_PAGE && l1 - l0 < m->dims.L) {
      launch_packed_bounds(c->view(), c->n / KVR_PAGE, len, m->dims.L, l0, l1, m->stream);
      ++n;
    }
    const kvr_status st = launched(m, n, "packed write");
    if (st)
      c->poisoned = true;
    else
      c->n = len;
    return st;
  });
}

kvr_status kvr_packed_read(const kvr_packed *c, const int32_t *positions, int32_t n_pos,
                           int32_t l0, int32_t l1, void *k_out, void *v_out) {
  return guarded([&]() -> kvr_status {
    if (!c) return fail(KVR_E_INVAL, "NULL packed cache");
    if (c->poisoned) return fail(KVR_E_POISONED, "packed cache poisoned");
    kvr_model *m = c->model;
    KVR_TRY(check_range(m, positions, n_pos, l0, l1, c->n));
    if (n_pos == 0 || l0 == l1) return KVR_OK;
    KVR_TRY(use_device(m));
    KVR_TRY(check_device_ptr(m, k_out, "k_out"));
    KVR_TRY(check_device_ptr(m, v_out, "v_out"));
    PackedRows rows;
    KVR_TRY(rows_of(m, positions, n_pos, rows));
    launch_packed_read(c->view(), m->dims.dtype, rows, l0, l1 - l0, k_out, v_out, m->stream);
    return launched(m, 1, "packed read");
  });
}

kvr_status kvr_packed_bounds(const kvr_packed *c, int32_t layer, int8_t *hi, int8_t *lo,
                             float *unit) {
  return guarded([&]() -> kvr_status {
    if (!c || !hi || !lo || !unit) return fail(KVR_E_INVAL, "NULL argument");
    kvr_model *m = c->model;
    const Dims &dm = m->dims;
    if (layer < 0 || layer >= dm.L)
      return fail(KVR_E_RANGE, "layer %d outside [0, %d)", layer, dm.L);
    KVR_TRY(use_device(m));
    KVR_TRY(synchronize(m));
    const int used = (c->n + KVR_PAGE - 1) / KVR_PAGE;
    const PackedView v = c->view();
    std::vector<int8_t> both((size_t)used * 2 * dm.dh);
    for (int g = 0; g < dm.G && used; ++g) {
      const size_t at = v.index(layer, g, 0);
      if (cudaMemcpy(both.data(), v.bounds + at * 2 * dm.dh, both.size(), cudaMemcpyDeviceToHost) !=
              cudaSuccess ||
          cudaMemcpy(unit + (size_t)g * used, v.unit + at, used * sizeof(float),
                     cudaMemcpyDeviceToHost) != cudaSuccess)
        return fail(KVR_E_CUDA, "bounds readback");
      for (int b = 0; b < used; ++b) {
        const int8_t *src = both.data() + (size_t)b * 2 * dm.dh;
        memcpy(hi + ((size_t)g * used + b) * dm.dh, src, dm.dh);
        memcpy(lo + ((size_t)g * used + b) * dm.dh, src + dm.dh, dm.dh);
      }
    }
    return KVR_OK;
  });
}

kvr_status kvr_rows_create(kvr_model *m, kvr_packed *const *docs, const int32_t *doc_rows,
                           int32_t n_docs, const int32_t *positions, kvr_rows **out) {
  kvr_rows *r = nullptr;
  return guarded([&]() -> kvr_status {
    if (!m || !docs || !doc_rows || !positions || !out) return fail(KVR_E_INVAL, "NULL argument");
    *out = nullptr;
    if (n_docs < 1 || n_docs > MAX_DOCS)
      return fail(KVR_E_RANGE, "n_docs=%d outside [1, %d]", n_docs, MAX_DOCS);
    long long M = 0;
    for (int d = 0; d < n_docs; ++d) {
      if (!docs[d] || docs[d]->model != m) return fail(KVR_E_INVAL, "document %d: bad handle", d);
      if (doc_rows[d] < 0) return fail(KVR_E_RANGE, "document %d: negative rows", d);
      M += doc_rows[d];
    }
    if (M < 1 || M > MAX_ROWS) return fail(KVR_E_RANGE, "%lld rows outside [1, %d]", M, MAX_ROWS);
    std::vector<kvr_packed *> dv(docs, docs + n_docs);
    std::vector<int32_t> rv(doc_rows, doc_rows + n_docs);
    KVR_TRY(check_rows(dv, rv, positions, (size_t)M));
    KVR_TRY(use_device(m));
    r = new kvr_rows();
    r->model = m;
    m->rows.push_back(r);
    r->docs = std::move(dv);
    r->doc_rows = std::move(rv);
    r->pos.resize(M);
    if (const kvr_status st = build_rows(r, positions)) {
      kvr_rows_free(r);
      return st;
    }
    *out = r;
    return KVR_OK;
  }, [&] { kvr_rows_free(r); });
}

kvr_status kvr_rows_move(kvr_rows *r, const int32_t *positions) {
  return guarded([&]() -> kvr_status {
    if (!r || !positions) return fail(KVR_E_INVAL, "NULL argument");
    for (const kvr_packed *d : r->docs)
      if (!d) return fail(KVR_E_INVAL, "a document of these rows has been freed");
    KVR_TRY(check_rows(r->docs, r->doc_rows, positions, r->pos.size()));
    KVR_TRY(use_device(r->model));
    return build_rows(r, positions);
  });
}

void kvr_rows_free(kvr_rows *r) {
  if (!r) return;
  kvr_model *m = r->model;
  cudaSetDevice(m->device);
  flush_uploads(m);
  cudaStreamSynchronize(m->stream);
  m->rows.erase(std::remove(m->rows.begin(), m->rows.end(), r), m->rows.end());
  if (m->pass_rows == r) m->pass_rows = nullptr;
  dev_free(r->mem);
  delete r;
}

kvr_status kvr_packed_attention(kvr_rows *r, int32_t layer, const void *q, int32_t ldq, void *out) {
  return guarded([&]() -> kvr_status {
    PackedAttnArgs a;
    KVR_TRY(rows_args(r, layer, q, ldq, a));
    kvr_model *m = r->model;
    KVR_TRY(check_device_ptr(m, out, "out"));
    return attend_all(r, a, out);
  });
}

kvr_status kvr_packed_select(kvr_rows *r, int32_t layer, const void *q, int32_t ldq,
                             int32_t n_blocks, int32_t *blocks_out) {
  return guarded([&]() -> kvr_status {
    PackedAttnArgs a;
    KVR_TRY(rows_args(r, layer, q, ldq, a));
    if (n_blocks < 1 || n_blocks > MAX_BLOCKS)
      return fail(KVR_E_RANGE, "n_blocks=%d outside [1, %d]", n_blocks, MAX_BLOCKS);
    kvr_model *m = r->model;
    KVR_TRY(check_device_ptr(m, blocks_out, "blocks_out"));
    return select_blocks(r, a, n_blocks, blocks_out);
  });
}

kvr_status kvr_packed_attention_blocks(kvr_rows *r, int32_t layer, const void *q, int32_t ldq,
                                       const int32_t *blocks, int32_t n_blocks, void *out) {
  return guarded([&]() -> kvr_status {
    PackedAttnArgs a;
    KVR_TRY(rows_args(r, layer, q, ldq, a));
    if (n_blocks < 1 || n_blocks > MAX_BLOCKS)
      return fail(KVR_E_RANGE, "n_blocks=%d outside [1, %d]", n_blocks, MAX_BLOCKS);
    kvr_model *m = r->model;
    KVR_TRY(check_device_ptr(m, out, "out"));
    KVR_TRY(check_device_ptr(m, blocks, "blocks"));
    return attend_blocks(r, a, blocks, n_blocks, out);
  });
}

}  // extern "C"
