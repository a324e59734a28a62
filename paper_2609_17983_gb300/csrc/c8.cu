// c8.cu -- the 8-bit cache's entry points: documents held in 8 bits, their rows written and read
// back, query rows that attend to them and weigh their entries, and the entries to keep.
#include <cmath>
#include <cstring>

#include "c8.cuh"
#include "entry.cuh"
#include "vec_deal.cuh"

namespace kvr {

kvr_status not_captured(const kvr_model *m, const char *what) {
  return capturing(m) ? fail(KVR_E_UNSUPPORTED, "%s while the model's stream is being captured", what)
                      : KVR_OK;
}

}  // namespace kvr

using namespace kvr;

namespace {

constexpr int MAX_CAPACITY = 1 << 20;  // entries of a cache
constexpr int MAX_ROWS = 1 << 20, MAX_DOCS = 4096;
// Scores of the tiles that are weighed by one launch (a tile of a long document may alone have
// more): half of L2, where the launch that sums them finds them.
constexpr long long SCORE_BYTES = 64 << 20;

// Scratch of at least `need` bytes.  What is outgrown is freed, or with the model once a graph may hold
// its address.  Growth at least doubles it, so that lengthening documents do not wait at every
// block, up to 256 MB at once where that leaves no outgrown memory behind.
kvr_status keep_device(kvr_model *m, void *&buf, size_t &have, size_t need, const char *what) {
  if (need <= have) return KVR_OK;
  KVR_TRY(not_captured(m, "scratch to be allocated (run the call once before)"));
  const size_t more = m->c8_captured ? have : std::min(have, (size_t)256 << 20);
  if (buf && m->c8_captured) {
    m->retired.push_back(buf);
  } else if (buf) {
    if (cudaStreamSynchronize(m->stream) != cudaSuccess)
      return fail(KVR_E_CUDA, "%s: %s", what, cudaGetErrorString(cudaGetLastError()));
    dev_free(buf);
  }
  const size_t size = std::max(need, have + more);
  buf = dev_alloc(size);
  have = buf ? size : 0;
  return buf ? KVR_OK : fail(KVR_E_NOMEM, "%s: %zu bytes", what, size);
}

// A kernel of these rows was launched: the next one follows it, not the tables' upload.  One that
// was captured does not lie in the stream between them.
void launched_behind_tables(kvr_c8_rows *r) {
  if (!r->settled) r->settled = !capturing(r->model);
}

int length(const kvr_c8 *c) { return *std::min_element(c->len.begin(), c->len.end()); }

kvr_status check_range(const kvr_c8 *c, const int32_t *entries, int n, int l0, int l1, int end) {
  const int L = c->model->dims.L;
  if (n < 0) return fail(KVR_E_RANGE, "negative number of entries");
  if (l0 < 0 || l1 > L || l0 > l1) return fail(KVR_E_RANGE, "layers [%d, %d) outside [0, %d)", l0, l1, L);
  if (n > 0 && !entries) return fail(KVR_E_INVAL, "NULL entries");
  for (int i = 0; i < n; ++i) {
    if (entries[i] < 0 || entries[i] >= end)
      return fail(KVR_E_RANGE, "entry %d outside [0, %d)", entries[i], end);
    if (i && entries[i] <= entries[i - 1])
      return fail(KVR_E_RANGE, "entries not strictly increasing at %d", i);
  }
  return KVR_OK;
}

kvr_status usable(const kvr_c8 *c) {
  if (!c) return fail(KVR_E_INVAL, "NULL cache");
  if (c->poisoned) return fail(KVR_E_POISONED, "cache poisoned by an earlier CUDA error");
  return KVR_OK;
}

// The shortest of layers [l0, l1).
int shortest(const kvr_c8 *c, int l0, int l1) {
  return l0 == l1 ? 0 : *std::min_element(c->len.begin() + l0, c->len.begin() + l1);
}

kvr_status check_first(const kvr_c8 *c, int n, int l0, int l1) {
  KVR_TRY(check_range(c, nullptr, 0, l0, l1, 0));
  if (n < 0 || (l0 < l1 && n > shortest(c, l0, l1)))
    return fail(KVR_E_RANGE, "the first %d entries of %d", n, shortest(c, l0, l1));
  return KVR_OK;
}

// The rows of a write into layers [l0, l1), a launch for each stretch of layers of one length.
kvr_status write_rows(kvr_c8 *c, const PackedRows &rows, int last, int l0, int l1,
                      const void *k, const void *v) {
  kvr_model *m = c->model;
  const Dims &dm = m->dims;
  kvr_status st = KVR_OK;
  for (int a = l0, b; a < l1 && !st; a = b) {
    for (b = a + 1; b < l1 && c->len[b] == c->len[a];) ++b;
    const size_t at = (size_t)(a - l0) * dm.G * dm.dh * dm.es();
    launch_c8_write(c->view(), dm.dtype, rows, c->len[a], c->shift, a, b - a, l1 - l0,
                    (const char *)k + at, (const char *)v + at, m->stream);
    st = launched(m, 1, "write in 8 bits");
    for (int l = a; l < b; ++l) c->len[l] = std::max(c->len[l], last + 1);
  }
  if (st) c->poisoned = true;
  return st;
}

// ------------------------------------------------------------ query rows

kvr_status check_rows(const std::vector<kvr_c8 *> &docs, const std::vector<int32_t> &doc_rows,
                      const int32_t *pos, size_t count) {
  size_t i = 0;
  for (size_t d = 0; d < docs.size(); ++d)
    for (int r = 0; r < doc_rows[d]; ++r, ++i) {
      if (pos[i] < -1 || pos[i] >= docs[d]->cap)
        return fail(KVR_E_RANGE, "row %zu: entry %d outside [-1, %d)", i, pos[i], docs[d]->cap);
      if (r && pos[i] < pos[i - 1])
        return fail(KVR_E_RANGE, "row %zu: entries of a document descend", i);
    }
  return i == count ? KVR_OK : fail(KVR_E_RANGE, "row counts do not match");
}

// The deal of tiles (deal_pages), by the costs of the 4-bit cache's kernel, whose pages cost as
// much beside one another: of all deals of 15 calls (1 to 40 rows over 300 to 131072 entries, 16
// documents of 8191, bf16 and fp32) the one taken is the fastest or within 4% of it (20 rows over
// 1000 entries, 6.95 against 6.68 us).
Deal deal(const kvr_model *m, const std::vector<std::pair<int, int>> &tiles) {
  const int dt = m->dims.dtype, many = c8_attn_warps(dt);
  return deal_pages(DealCost{280, 150, 140, 250, 7}, tiles, m->dims.G, m->num_sms, many,
                    c8_attn_ctas_per_sm(dt, many), c8_attn_ctas_per_sm(dt, 4));
}

// Tiles of at most 128 vectors of the attention straight from the codes: equal ones, their pages split
// so that the CTAs fill the chip once.
struct StraightTiles {
  int per, count, splits;  // rows of a tile, tiles, parts of their pages
};
StraightTiles straight_tiles(const kvr_model *m, int rows, int pages) {
  const Dims &dm = m->dims;
  StraightTiles t;
  const int most = 128 / (dm.H / dm.G), n = (rows + most - 1) / most;
  t.per = (rows + n - 1) / n;
  t.count = (rows + t.per - 1) / t.per;
  t.splits = std::max(1, std::min({m->num_sms / (t.count * dm.G), (pages + 1) / 2, 64}));
  while (t.splits > 1 && attn_tc_ws_floats(t.splits, t.count, dm.G, dm.dh) > m->attn_ws_floats)
    --t.splits;
  return t;
}

// Which kernels take the rows of a document at `pos` (ascending, >= 0): the fused one, the one
// straight from the codes, or the ones over pages of halves; those two share the sum of the
// weights. The way whose calls are modelled to end first, in us, `docs` documents sharing the fused
// kernel's launches; it is that of calls without weights, so that with them the output is the same.
// Of 430 calls (1 to 4096 rows, side by side or spread over 300 to 131072 entries, 4 and 7 heads a
// KV head of 128, 2 of 64) the way taken is 0.3% slower than the fastest on average, with weights
// 0.8%, 18% at most (512 rows over 2500 entries, 4 heads of 64: fused 15.7, straight 13.4, by pages
// 14.5), with weights 31% (8 rows over 40000, 32 heads: straight 69.3, fused 52.8).  40 rows spread
// over 5000 entries, 32 heads: fused 15.6, straight 18.3, by pages 22.6; the last 64 of 12345: 64,
// 22.6, 39; the last 4096 of 12345, 28 heads: straight 538, by pages 421.
enum Way { FUSED, STRAIGHT, PAGES };
Way way_of(const kvr_model *m, const int32_t *pos, int rows, size_t docs) {
  const Dims &dm = m->dims;
  const int grp = dm.H / dm.G;
  if (dm.dtype != KVR_DTYPE_BF16 || rows < 1 || grp > 128) return FUSED;
  const int pages = pos[rows - 1] / KVR_PAGE + 1;
  const StraightTiles t = straight_tiles(m, rows, pages);
  if (t.count > 60000) return FUSED;  // grid dimensions
  const double units = (double)vector_units(pos, rows, grp) * dm.G, d = dm.dh / 128.0,
               sms = m->num_sms;
  const double fused = 4.4 / docs + 1.4e-3 * units * (0.1 + 0.9 * d) + 0.116 * std::sqrt(pages);
  // straight: steps of two pages, of the longest CTA and on average of the SMs; CTAs of more than one wave
  double all = 0, longest = 0;
  for (int r = 0; r < rows; r += t.per) {
    const int n = pos[std::min(rows, r + t.per) - 1] / KVR_PAGE + 1;
    const int steps = ((n + t.splits - 1) / t.splits + 1) / 2;
    longest = std::max(longest, (double)steps);
    all += (double)steps * t.splits * dm.G / sms;
  }
  const double waves = t.count * (double)t.splits * dm.G / sms;
  const double straight = 7.75 + (waves <= 1 ? longest : all + longest / 2) * (0.75 + 0.23 * d) +
                          5.5 * std::max(0.0, waves - 1) + (t.splits > 1 ? 5.4 : 0.0);
  ManyPlan p;
  std::vector<int32_t> tables;
  double by_pages = 1e30;
  if (many_plan(m, pos, rows, tables, p))
    by_pages = 7.1 + 8.8e-3 * pages * dm.G * d + 0.1 * p.cost * (0.56 + 0.14 * d);
  return fused <= std::min(straight, by_pages) ? FUSED : straight <= by_pages ? STRAIGHT : PAGES;
}

// The tables of the attention straight from the codes.
void straight_plan(const kvr_model *m, const int32_t *pos, int rows, std::vector<int32_t> &tables,
                   ManyPlan &p) {
  p.rows = rows;
  p.pages = pos[rows - 1] / KVR_PAGE + 1;
  const StraightTiles t = straight_tiles(m, rows, p.pages);
  p.block_rows = t.per;
  p.n_blocks = t.count;
  p.splits = t.splits;
  for (int r = 0; r < rows; r += t.per) {
    const int k = std::min(t.per, rows - r);
    tables.insert(tables.end(), {r, k, pos[r + k - 1], 0});
  }
}

// The tables of rows at `pos`, built and sent.
kvr_status build_rows(kvr_c8_rows *r, const int32_t *pos) {
  kvr_model *m = r->model;
  const Dims &dm = m->dims;
  const int grp = dm.H / dm.G, M = (int)r->pos.size(), D = (int)r->docs.size();
  kvr_c8_rows::Plan p;
  std::vector<C8Part> parts;
  std::vector<C8Tile> tiles;
  std::vector<C8Doc> docs;
  std::vector<int32_t> tables;  // of many rows
  std::vector<int> tile_doc, pages;
  std::vector<bool> is_many(D);
  for (int d = 0, row0 = 0; d < D; row0 += r->doc_rows[d++]) {
    const int R = r->doc_rows[d];
    int few = R;  // rows that the fused kernel takes: the first ones
    const int none = (int)(std::lower_bound(pos + row0, pos + row0 + R, 0) - (pos + row0));
    kvr_c8_rows::Many y{d, row0 + none, false, tables.size(), {}, {}};
    const Way way = way_of(m, pos + row0 + none, R - none, r->docs.size());
    y.straight = way == STRAIGHT;
    if (y.straight) straight_plan(m, pos + row0 + none, R - none, tables, y.plan);
    if (y.straight ||
        (way == PAGES && many_plan(m, pos + row0 + none, R - none, tables, y.plan))) {
      few = none;
      is_many[d] = true;
      y.shape = c8_many_shape(R - none, grp, y.plan.pages, dm.G, m->num_sms);
      p.many.push_back(y);
      p.max_pages = std::max(p.max_pages, y.plan.pages);
    }
    for (int v = 0; v < few * grp; v += PACK_VEC) {
      C8Tile t{};
      t.vec0 = row0 * grp + v;
      t.nvec = std::min(PACK_VEC, few * grp - v);
      t.pages = (pos[(t.vec0 + t.nvec - 1) / grp] + KVR_PAGE) / KVR_PAGE;  // entries ascend
      tiles.push_back(t);
      tile_doc.push_back(d);
      pages.push_back(t.pages);
    }
  }
  std::sort(pages.begin(), pages.end());
  std::vector<std::pair<int, int>> count;  // tiles of so many pages
  for (int np : pages) {
    if (count.empty() || count.back().first != np) count.push_back({np, 0});
    ++count.back().second;
  }
  const Deal dl = deal(m, count);
  long long scores = 0;
  for (int i = 0; i < (int)tiles.size(); ++i) {
    C8Tile &t = tiles[i];
    const int d = tile_doc[i];
    const kvr_c8 *c = r->docs[d];
    const long long room = (long long)dm.G * t.pages * KVR_PAGE * (t.nvec > 4 ? PACK_VEC : 4);
    const int part0 = (int)parts.size(), doc0 = (int)docs.size();
    if (p.launches.empty() || (scores + room) * 4 > SCORE_BYTES) {
      p.launches.push_back({part0, part0, doc0, doc0, 0});
      scores = 0;
    }
    kvr_c8_rows::Launch &now = p.launches.back();
    t.scores = scores;
    scores += room;
    p.scores = std::max(p.scores, scores);
    const bool first = i == 0 || d != tile_doc[i - 1];
    // (rows of a many document that are left here see nothing and add nothing)
    if (!is_many[d]) {
      if (first || now.doc1 == now.doc0) {
        docs.push_back(C8Doc{c->weight, c->pages, i, i, first ? 1 : 0});
        p.doc_of.push_back(d);
        ++now.doc1;
      }
      docs.back().tile1 = i + 1;
      now.tiles = std::max(now.tiles, i + 1 - docs.back().tile0);
    }
    C8Part y{};
    y.blocks = c->blocks, y.power = c->power, y.pages = c->pages;
    y.vec0 = t.vec0, y.nvec = t.nvec;
    y.slot = part0, y.tile = i, y.np = t.pages, y.scores = t.scores;
    y.n_parts = dl.parts(t.pages);
    p.merged = p.merged || y.n_parts > dl.cluster;
    for (y.part = 0; y.part < y.n_parts; ++y.part) {
      y.page0 = (int)((long long)t.pages * y.part / y.n_parts);
      y.page1 = (int)((long long)t.pages * (y.part + 1) / y.n_parts);
      parts.push_back(y);
    }
    now.part1 = (int)parts.size();
  }
  p.n_parts = (int)parts.size();
  p.n_tiles = (int)tiles.size();
  p.warps = dl.warps;
  p.cluster = dl.cluster;
  const size_t o_tile = up256(parts.size() * sizeof(C8Part)),
               o_doc = up256(o_tile + tiles.size() * sizeof(C8Tile)),
               o_many = up256(o_doc + docs.size() * sizeof(C8Doc)),
               o_pos = up256(o_many + tables.size() * 4), o_id = up256(o_pos + M * 4ull),
               bytes = up256(o_id + p.max_pages * 4ull);
  std::vector<char> host(bytes);
  memcpy(host.data(), parts.data(), parts.size() * sizeof(C8Part));
  memcpy(host.data() + o_tile, tiles.data(), tiles.size() * sizeof(C8Tile));
  memcpy(host.data() + o_doc, docs.data(), docs.size() * sizeof(C8Doc));
  memcpy(host.data() + o_many, tables.data(), tables.size() * 4);
  memcpy(host.data() + o_pos, pos, M * 4ull);
  for (int i = 0; i < p.max_pages; ++i) ((int32_t *)(host.data() + o_id))[i] = i;
  r->sent = r->settled = false;
  KVR_TRY(grow_device(m, r->mem, r->mem_bytes, bytes, "query rows"));
  KVR_TRY(upload_words(m, r->mem, host.data(), bytes / 4));
  char *base = (char *)r->mem;
  p.parts_d = (C8Part *)base;
  p.tiles_d = (C8Tile *)(base + o_tile);
  p.docs_d = (C8Doc *)(base + o_doc);
  p.many_d = (int32_t *)(base + o_many);
  p.pos_d = (int32_t *)(base + o_pos);
  p.identity_d = (int32_t *)(base + o_id);
  r->plan = std::move(p);
  std::copy(pos, pos + M, r->pos.begin());
  r->sent = true;
  return KVR_OK;
}

// Room for the partial sums and arrival counts of a launch, where a tile has more than one
// cluster's to add.
kvr_status attn_workspace(kvr_model *m, const kvr_c8_rows::Plan &p, C8AttnArgs &a) {
  if (!p.merged) return KVR_OK;
  const size_t sums = (size_t)(p.n_parts / p.cluster) * a.G,
               o = up256(sums * PACK_VEC * a.dh * sizeof(float)),
               ml = sums * PACK_CLUSTER * PACK_VEC * sizeof(float2),
               cb = (size_t)p.n_tiles * a.G * PACK_CLUSTER * sizeof(int);
  KVR_TRY(keep_device(m, m->c8_ws, m->c8_ws_bytes, o + ml, "attention workspace"));
  if (cb > m->c8_count_bytes) {
    KVR_TRY(keep_device(m, m->c8_count, m->c8_count_bytes, cb, "attention counters"));
    if (cudaMemsetAsync(m->c8_count, 0, m->c8_count_bytes, m->stream) != cudaSuccess)
      return fail(KVR_E_CUDA, "attention counters");
  }
  a.ws_o = (float *)m->c8_ws;
  a.ws_ml = (float2 *)((char *)m->c8_ws + o);
  a.counters = (int *)m->c8_count;
  return KVR_OK;
}

// What the many rows of a document lay out in the pages' scratch: two sets of powers, the pages of halves,
// the vectors and what makes weights of their products, the runs' sums (those for weights alone).
struct ManyScratch {
  size_t powers, vectors, factors, last, partial, all;  // offsets from the second set of powers on
};
ManyScratch many_scratch(const Dims &dm, const kvr_c8_rows::Many &x, bool weigh) {
  const size_t pages_b = x.straight ? 0 : up256((size_t)x.plan.pages * 2 * dm.G * KVR_PAGE * dm.dh * 2),
               vec = (size_t)dm.G * x.shape.nv_pad;
  ManyScratch y;
  y.powers = up256(dm.G * sizeof(float2));
  y.vectors = 2 * y.powers + pages_b;
  y.factors = y.vectors + vec * dm.dh * 2;
  y.last = y.factors + vec * 12;
  y.partial = y.last + vec * 4;
  const size_t partial_b =
      x.shape.runs > 1 ? (size_t)x.shape.runs * dm.G * x.shape.keys * 4 : 0;
  y.all = weigh ? y.partial + partial_b : y.vectors;
  return y;
}

// The many rows of one document.  stats: [rows][H] of all rows, or null: without weights.
kvr_status attend_many(kvr_c8_rows *r, const kvr_c8_rows::Many &x, const C8AttnArgs &a, float2 *stats,
                       float decay) {
  kvr_model *m = r->model;
  const kvr_c8_rows::Plan &p = r->plan;
  const Dims &dm = m->dims;
  const kvr_c8 *c = r->docs[x.doc];
  const size_t vec = (size_t)dm.G * x.shape.nv_pad;
  const ManyScratch at = many_scratch(dm, x, stats != nullptr);
  char *base = (char *)m->c8_pages, *pages = base + 2 * at.powers;
  float2 *power = (float2 *)base;
  const void *q = (const char *)a.q + (size_t)x.row0 * a.ldq * dm.es();
  void *out = (char *)a.out + (size_t)x.row0 * dm.H * dm.dh * dm.es();
  const int4 *tables = (const int4 *)(p.many_d + x.table);
  const int32_t *pos = p.pos_d + x.row0;
  if (stats) stats += (size_t)x.row0 * dm.H;
  // for the weights
  float *key_power = (float *)(base + at.powers), *factor = (float *)(base + at.factors),
        *minus = factor + vec, *inverse = minus + vec;
  __half *vectors = (__half *)(base + at.vectors);
  int32_t *last = (int32_t *)(base + at.last);
  if (x.straight) {
    C8RowsArgs w{};
    w.cache = c->view();
    w.layer = a.layer, w.H = a.H, w.G = a.G, w.grp = a.grp, w.ldq = a.ldq, w.n_pages = x.plan.pages;
    w.scale = a.scale;
    w.q = (const __nv_bfloat16 *)q;
    w.pos = pos;
    w.blocks = tables;
    w.n_blocks = x.plan.n_blocks, w.n_splits = x.plan.splits;
    w.ws_o = m->attn_ws_o, w.ws_ml = m->attn_ws_ml;
    w.out = (__nv_bfloat16 *)out;
    w.page_power = power;
    if (stats) {
      w.vectors = vectors, w.factor = factor, w.key_power = key_power;
      w.weigh = {pos, minus, inverse, last, x.shape.nv_pad};
    }
    w.dev_flag = m->dev_flag;
    const char *e = launch_c8_rows(w, dm.dh, r->settled, m->stream);
    if (!e) {
      e = launch_attention_combine(tables, x.plan.n_blocks, x.plan.block_rows, x.plan.splits, dm,
                                   m->attn_ws_o, m->attn_ws_ml, out, m->stream, nullptr, 0, power,
                                   nullptr, &w.weigh);
    }
    if (e) return fail(KVR_E_CUDA, "attention in 8 bits: %s", e);
    KVR_TRY(launched(m, x.plan.splits > 1 ? 2 : 1, "attention in 8 bits"));
    launched_behind_tables(r);
  } else {
    launch_c8_unpack(c->view(), a.layer, x.plan.pages, pages, power, r->settled, m->stream);
    KVR_TRY(launched(m, 1, "blocks widened"));
    launched_behind_tables(r);
    KVR_TRY(many_attention(m, x.plan, tables, q, a.ldq, pos, pages, p.identity_d, out, power, stats));
  }
  if (!stats) return KVR_OK;
  C8ManyArgs w{};
  w.cache = c->view();
  w.layer = a.layer;
  w.rows = x.plan.rows, w.grp = a.grp, w.H = a.H, w.n_pages = x.plan.pages;
  w.n_tiles = x.shape.tiles, w.nv_pad = x.shape.nv_pad, w.keys = x.shape.keys;
  w.per = x.shape.per, w.runs = x.shape.runs, w.key_tiles = x.shape.key_tiles;
  w.scale = a.scale;
  w.pos = pos;
  w.stats = stats;
  w.key_power = key_power, w.vectors = vectors;
  w.factor = factor, w.minus = minus, w.inverse = inverse, w.last = last;
  w.partial = (float *)(base + at.partial);
  w.weight = c->weight + (size_t)a.layer * dm.G * c->pages * KVR_PAGE;
  w.len = c->len[a.layer];
  w.decay = decay;
  w.dev_flag = m->dev_flag;
  int n = 0;
  if (const char *e =
          launch_c8_weigh_many(w, x.straight ? nullptr : q, a.ldq, dm.dh, &n, m->stream))
    return fail(KVR_E_CUDA, "weights of entries: %s", e);
  return launched(m, n, "weights of entries");
}

// Attention of the rows; weigh: their weights are added to the entries'.
kvr_status attend(kvr_c8_rows *r, int layer, const void *q, int ldq, bool weigh, float decay,
                  void *out) {
  kvr_model *m = r->model;
  const Dims &dm = m->dims;
  const kvr_c8_rows::Plan &p = r->plan;
  C8AttnArgs a{};
  a.q = q, a.out = out, a.ldq = ldq;
  a.dtype = dm.dtype, a.H = dm.H, a.G = dm.G, a.grp = dm.H / dm.G, a.dh = dm.dh;
  a.layer = layer;
  a.scale = (float)(1.4426950408889634 / std::sqrt((double)dm.dh));
  a.pos = p.pos_d;
  a.warps = p.warps, a.cluster = p.cluster;
  a.dev_flag = m->dev_flag;
  KVR_TRY(attn_workspace(m, p, a));
  float2 *stats = nullptr;
  if (weigh) {
    const size_t stats_b = up256(r->pos.size() * dm.H * sizeof(float2));
    KVR_TRY(keep_device(m, m->c8_scores, m->c8_scores_bytes, stats_b + p.scores * 4,
                        "attention scores"));
    stats = a.stats = (float2 *)m->c8_scores;
    a.scores = (float *)((char *)m->c8_scores + stats_b);
  }
  // all scratch is there before the first launch: a call that has to be refused leaves nothing behind
  size_t many = 0;
  for (const auto &x : p.many) many = std::max(many, many_scratch(dm, x, weigh).all);
  KVR_TRY(keep_device(m, m->c8_pages, m->c8_pages_bytes, many, "pages of halves"));
  std::vector<int> len;
  for (const auto &x : p.launches) {
    a.settled = r->settled;
    a.parts = p.parts_d + x.part0;
    a.n_parts = x.part1 - x.part0;
    if (!weigh) a.parts = p.parts_d, a.n_parts = p.n_parts;  // all at once
    if (const char *e = launch_c8_attention(a, m->stream))
      return fail(KVR_E_CUDA, "attention in 8 bits: %s", e);
    KVR_TRY(launched(m, 1, "attention in 8 bits"));
    launched_behind_tables(r);
    if (!weigh) break;
    len.clear();
    for (int i = x.doc0; i < x.doc1; ++i) len.push_back(r->docs[p.doc_of[i]]->len[layer]);
    const int n = launch_c8_weigh(a, p.tiles_d, p.docs_d + x.doc0, x.doc1 - x.doc0, len.data(),
                                  x.tiles, decay, m->stream);
    KVR_TRY(launched(m, n, "weights of entries"));
  }
  for (const auto &x : p.many) KVR_TRY(attend_many(r, x, a, stats, decay));
  return KVR_OK;
}

kvr_status attention_call(kvr_c8_rows *r, int32_t layer, const void *q, int32_t ldq, bool weigh,
                          float decay, void *out) {
  if (!r) return fail(KVR_E_INVAL, "NULL rows");
  kvr_model *m = r->model;
  const Dims &dm = m->dims;
  if (layer < 0 || layer >= dm.L) return fail(KVR_E_RANGE, "layer %d outside [0, %d)", layer, dm.L);
  size_t row = 0;
  for (size_t d = 0; d < r->docs.size(); ++d) {
    const kvr_c8 *c = r->docs[d];
    if (!c) return fail(KVR_E_INVAL, "a document of these rows has been freed");
    KVR_TRY(usable(c));
    row += r->doc_rows[d];
    if (r->doc_rows[d] && r->pos[row - 1] >= c->len[layer])
      return fail(KVR_E_RANGE, "document %zu: a row at entry %d, layer %d holds %d", d,
                  r->pos[row - 1], layer, c->len[layer]);
  }
  if (!r->sent) return fail(KVR_E_INVAL, "rows whose last move failed");
  if (ldq < dm.H * dm.dh || ldq * dm.es() % 16)
    return fail(KVR_E_INVAL, "row stride %d of q: at least %d, whole 16-byte pieces", ldq,
                dm.H * dm.dh);
  KVR_TRY(use_device(m));
  KVR_TRY(check_device_ptr(m, q, "q"));
  KVR_TRY(check_device_ptr(m, out, "out"));
  if (!m->c8_captured) m->c8_captured = capturing(m);  // (0.03 us)
  return attend(r, layer, q, ldq, weigh, decay, out);
}

void free_rows_of(kvr_model *m, const kvr_c8 *c) {
  for (kvr_c8_rows *r : m->c8_rows)
    std::replace(r->docs.begin(), r->docs.end(), const_cast<kvr_c8 *>(c), (kvr_c8 *)nullptr);
}

}  // namespace

namespace kvr {

kvr_status c8_write_layers(kvr_c8 *c, const PackedRows &rows, int last, int l0, int l1,
                           const void *k, const void *v) {
  return write_rows(c, rows, last, l0, l1, k, v);
}

kvr_status c8_pass_rows(kvr_c8 *c, const int32_t *entries, int n, kvr_c8_rows **out) {
  kvr_model *m = c->model;
  if (!m->c8_pass_rows) {
    m->c8_pass_rows = new kvr_c8_rows();
    m->c8_pass_rows->model = m;
    m->c8_rows.push_back(m->c8_pass_rows);
  }
  kvr_c8_rows *r = m->c8_pass_rows;
  r->docs.assign(1, c);
  r->doc_rows.assign(1, n);
  r->pos.assign(entries, entries + n);
  *out = r;
  return build_rows(r, r->pos.data());
}

kvr_status c8_attend(kvr_c8_rows *r, int layer, const void *q, void *out, float decay) {
  const Dims &dm = r->model->dims;
  return attend(r, layer, q, dm.H * dm.dh, decay >= 0.f, decay, out);
}

}  // namespace kvr

extern "C" {

kvr_status kvr_c8_create(kvr_model *m, int32_t capacity, kvr_c8 **out) {
  kvr_c8 *c = nullptr;
  return guarded([&]() -> kvr_status {
    if (!m || !out) return fail(KVR_E_INVAL, "NULL argument");
    *out = nullptr;
    if (capacity < 1 || capacity > MAX_CAPACITY)
      return fail(KVR_E_RANGE, "capacity %d outside [1, %d]", capacity, MAX_CAPACITY);
    KVR_TRY(use_device(m));
    KVR_TRY(not_captured(m, "a cache created"));
    const Dims &dm = m->dims;
    c = new kvr_c8();
    c->model = m;
    m->c8.push_back(c);
    c->cap = capacity;
    c->pages = (capacity + KVR_PAGE - 1) / KVR_PAGE;
    c->len.assign(dm.L, 0);
    const size_t n = (size_t)dm.L * dm.G * c->pages;
    c->blocks = (uint8_t *)dev_alloc(n * c8_block_bytes(dm.dh));
    c->power = (float2 *)dev_alloc(n * sizeof(float2));
    c->number = (int32_t *)dev_alloc(n * KVR_PAGE * sizeof(int32_t));
    c->weight = (float *)dev_alloc(n * KVR_PAGE * sizeof(float));
    kvr_status st = KVR_OK;
    if (!c->blocks || !c->power || !c->number || !c->weight)
      st = fail(KVR_E_NOMEM, "cache of %d entries in 8 bits", capacity);
    // V's codes are finite from the start: entries behind the last take part with a weight of zero
    if (!st && cudaMemsetAsync(c->blocks, 0, n * c8_block_bytes(dm.dh), m->stream) != cudaSuccess)
      st = fail(KVR_E_CUDA, "cache clear");
    if (!st) {
      launch_c8_clear(c->view(), n, m->stream);
      st = launched(m, 1, "cache clear");
    }
    if (st) {
      kvr_c8_free(c);
      return st;
    }
    *out = c;
    return KVR_OK;
  }, [&] { kvr_c8_free(c); });
}

void kvr_c8_free(kvr_c8 *c) {
  if (!c) return;
  kvr_model *m = c->model;
  cudaSetDevice(m->device);
  flush_uploads(m);
  cudaStreamSynchronize(m->stream);
  m->c8.erase(std::remove(m->c8.begin(), m->c8.end(), c), m->c8.end());
  free_rows_of(m, c);
  dev_free(c->tokens_d);
  dev_free(c->blocks);
  dev_free(c->power);
  dev_free(c->number);
  dev_free(c->weight);
  delete c;
}

int32_t kvr_c8_len(const kvr_c8 *c) { return c ? length(c) : -1; }

kvr_status kvr_c8_write(kvr_c8 *c, const int32_t *entries, int32_t n, int32_t l0, int32_t l1,
                        const void *k, const void *v) {
  return guarded([&]() -> kvr_status {
    KVR_TRY(usable(c));
    kvr_model *m = c->model;
    KVR_TRY(check_range(c, entries, n, l0, l1, c->cap));
    for (int i = 0, end = shortest(c, l0, l1); i < n; ++i) {
      if (l0 < l1 && entries[i] > end)
        return fail(KVR_E_RANGE, "entry %d leaves a gap after %d", entries[i], end);
      end = std::max(end, entries[i] + 1);
    }
    if (n == 0 || l0 == l1) return KVR_OK;
    KVR_TRY(use_device(m));
    KVR_TRY(not_captured(m, "entries written"));
    KVR_TRY(check_device_ptr(m, k, "k"));
    KVR_TRY(check_device_ptr(m, v, "v"));
    PackedRows rows;
    KVR_TRY(packed_rows_of(m, entries, n, rows));
    return write_rows(c, rows, entries[n - 1], l0, l1, k, v);
  });
}

kvr_status kvr_c8_read(const kvr_c8 *c, const int32_t *entries, int32_t n, int32_t l0, int32_t l1,
                       void *k_out, void *v_out) {
  return guarded([&]() -> kvr_status {
    KVR_TRY(usable(c));
    kvr_model *m = c->model;
    KVR_TRY(check_range(c, entries, n, l0, l1, MAX_CAPACITY));
    if (n == 0 || l0 == l1) return KVR_OK;
    const int len = shortest(c, l0, l1);
    if (entries[n - 1] >= len)
      return fail(KVR_E_RANGE, "entry %d outside [0, %d)", entries[n - 1], len);
    KVR_TRY(use_device(m));
    KVR_TRY(check_device_ptr(m, k_out, "k_out"));
    KVR_TRY(check_device_ptr(m, v_out, "v_out"));
    if (n > PACK_INLINE_POS && entries[n - 1] - entries[0] != n - 1)
      KVR_TRY(not_captured(m, "a list of entries sent"));
    PackedRows rows;
    KVR_TRY(packed_rows_of(m, entries, n, rows));
    launch_c8_read(c->view(), m->dims.dtype, rows, l0, l1 - l0, k_out, v_out, m->stream);
    return launched(m, 1, "read of 8 bits");
  });
}

kvr_status kvr_c8_entries(const kvr_c8 *c, int32_t n, int32_t l0, int32_t l1,
                          int32_t *number_out, float *weight_out) {
  return guarded([&]() -> kvr_status {
    KVR_TRY(usable(c));
    kvr_model *m = c->model;
    KVR_TRY(check_first(c, n, l0, l1));
    if (!n || l0 == l1 || (!number_out && !weight_out)) return KVR_OK;
    KVR_TRY(use_device(m));
    if (number_out) KVR_TRY(check_device_ptr(m, number_out, "number_out", 4));
    if (weight_out) KVR_TRY(check_device_ptr(m, weight_out, "weight_out", 4));
    launch_c8_entries(c->view(), n, l0, l1 - l0, number_out, weight_out, m->stream);
    return launched(m, 1, "numbers and weights");
  });
}

kvr_status kvr_c8_set_weights(kvr_c8 *c, int32_t n, int32_t l0, int32_t l1, const float *weight) {
  return guarded([&]() -> kvr_status {
    KVR_TRY(usable(c));
    kvr_model *m = c->model;
    KVR_TRY(check_first(c, n, l0, l1));
    if (!n || l0 == l1) return KVR_OK;
    KVR_TRY(use_device(m));
    KVR_TRY(check_device_ptr(m, weight, "weight", 4));
    launch_c8_set_weights(c->view(), n, l0, l1 - l0, weight, m->stream);
    return launched(m, 1, "weights set");
  });
}

kvr_status kvr_c8_choose(const kvr_c8 *c, int32_t keep, int32_t first, int32_t recent,
                         int32_t *kept_out) {
  return guarded([&]() -> kvr_status {
    KVR_TRY(usable(c));
    kvr_model *m = c->model;
    const int len = c->common_length();
    if (len < 0) return fail(KVR_E_INVAL, "layers of different lengths");
    if (keep < 0 || keep > len || first < 0 || recent < 0 || (long long)first + recent > keep)
      return fail(KVR_E_RANGE, "%d of %d entries, the first %d and the last %d among them", keep, len,
                  first, recent);
    if (!keep) return KVR_OK;
    KVR_TRY(use_device(m));
    KVR_TRY(check_device_ptr(m, kept_out, "kept_out", 4));
    if (const char *e = launch_c8_choose(c->view(), len, m->dims.L, keep, first, recent, kept_out,
                                         m->stream))
      return fail(KVR_E_CUDA, "choice of entries: %s", e);
    return launched(m, 1, "choice of entries");
  });
}

kvr_status kvr_c8_keep(kvr_c8 *c, const int32_t *kept, int32_t n, kvr_c8 *into) {
  return guarded([&]() -> kvr_status {
    KVR_TRY(usable(c));
    kvr_c8 *to = into ? into : c;
    KVR_TRY(usable(to));
    kvr_model *m = c->model;
    if (to->model != m) return fail(KVR_E_INVAL, "caches of different models");
    const int len = c->common_length();
    if (len < 0) return fail(KVR_E_INVAL, "layers of different lengths");
    if (n < 0 || n > len) return fail(KVR_E_RANGE, "%d of %d entries", n, len);
    if (n > to->cap) return fail(KVR_E_RANGE, "%d entries into a cache of %d", n, to->cap);
    KVR_TRY(use_device(m));
    KVR_TRY(not_captured(m, "entries dropped"));
    if (n) KVR_TRY(check_device_ptr(m, kept, "kept", 4));
    if (n) {
      const char *e = launch_c8_keep(c->view(), to->view(), len, m->dims.L, kept, n, m->num_sms,
                                     m->stream);
      const kvr_status st = e ? fail(KVR_E_CUDA, "entries kept: %s", e) : launched(m, 1, "entries kept");
      if (st) {
        to->poisoned = true;
        return st;
      }
    }
    to->shift = c->shift + len - n;
    to->len.assign(m->dims.L, n);
    if (to != c && to->tokens_d) {  // entries alone: it is no longer the document that it was
      to->tokens_h.clear();
      flush_uploads(m);
      cudaStreamSynchronize(m->stream);
      dev_free(to->tokens_d);
      to->tokens_d = nullptr;
    }
    return KVR_OK;
  });
}

kvr_status kvr_c8_rows_create(kvr_model *m, kvr_c8 *const *docs, const int32_t *doc_rows,
                              int32_t n_docs, const int32_t *entries, kvr_c8_rows **out) {
  kvr_c8_rows *r = nullptr;
  return guarded([&]() -> kvr_status {
    if (!m || !docs || !doc_rows || !entries || !out) return fail(KVR_E_INVAL, "NULL argument");
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
    std::vector<kvr_c8 *> dv(docs, docs + n_docs);
    {  // two sets of rows of one document would add to the same weights
      std::vector<kvr_c8 *> sorted = dv;
      std::sort(sorted.begin(), sorted.end());
      if (std::adjacent_find(sorted.begin(), sorted.end()) != sorted.end())
        return fail(KVR_E_INVAL, "a document listed twice");
    }
    std::vector<int32_t> rv(doc_rows, doc_rows + n_docs);
    KVR_TRY(check_rows(dv, rv, entries, (size_t)M));
    KVR_TRY(use_device(m));
    KVR_TRY(not_captured(m, "rows created"));
    r = new kvr_c8_rows();
    r->model = m;
    m->c8_rows.push_back(r);
    r->docs = std::move(dv);
    r->doc_rows = std::move(rv);
    r->pos.resize(M);
    if (const kvr_status st = build_rows(r, entries)) {
      kvr_c8_rows_free(r);
      return st;
    }
    *out = r;
    return KVR_OK;
  }, [&] { kvr_c8_rows_free(r); });
}

kvr_status kvr_c8_rows_move(kvr_c8_rows *r, const int32_t *entries) {
  return guarded([&]() -> kvr_status {
    if (!r || !entries) return fail(KVR_E_INVAL, "NULL argument");
    for (const kvr_c8 *d : r->docs)
      if (!d) return fail(KVR_E_INVAL, "a document of these rows has been freed");
    KVR_TRY(check_rows(r->docs, r->doc_rows, entries, r->pos.size()));
    KVR_TRY(use_device(r->model));
    KVR_TRY(not_captured(r->model, "rows moved"));
    return build_rows(r, entries);
  });
}

void kvr_c8_rows_free(kvr_c8_rows *r) {
  if (!r) return;
  kvr_model *m = r->model;
  cudaSetDevice(m->device);
  flush_uploads(m);
  cudaStreamSynchronize(m->stream);
  m->c8_rows.erase(std::remove(m->c8_rows.begin(), m->c8_rows.end(), r), m->c8_rows.end());
  if (m->c8_pass_rows == r) m->c8_pass_rows = nullptr;
  dev_free(r->mem);
  delete r;
}

kvr_status kvr_c8_attention(kvr_c8_rows *r, int32_t layer, const void *q, int32_t ldq, void *out) {
  return guarded([&] { return attention_call(r, layer, q, ldq, false, 0.f, out); });
}

kvr_status kvr_c8_attention_weigh(kvr_c8_rows *r, int32_t layer, const void *q, int32_t ldq,
                                  float decay, void *out) {
  return guarded([&]() -> kvr_status {
    if (!(decay >= 0.f && decay <= 1.f))
      return fail(KVR_E_RANGE, "decay %g outside [0, 1]", (double)decay);
    return attention_call(r, layer, q, ldq, true, decay, out);
  });
}

}  // extern "C"
