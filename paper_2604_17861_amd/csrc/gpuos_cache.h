// gpuos_cache.h -- cache operators (gpuos_cache_task): what their kernels are given and, for the host, the check of a
// descriptor and its packing.
#pragma once
#include "gpuos_model.h"

namespace gpuos {

enum CacheFormat : uint32_t { CF_E2M1 = 0, CF_I8 = 1, CF_E4M3 = 2 };

// A cache of keys or of values: where it lies, what a page, a place and a head are apart (bytes; floats for the scales).
struct CachePart {
  uint64_t cache, scales;
  uint32_t cs[3], ss[4];           // page, place, head (, group)
};
// Queries, keys or values: where the rows are, and where they go: the rotated rows, or a cache and its scales.
struct AppendSide {
  uint64_t x, to, scales;
  uint32_t xs[4], ts[4], ss[4];    // strides: B, S, H, D; the same, or page, place, head (bytes); page, place, head, group
  uint32_t heads, blocks;          // heads, and blocks of them
  uint32_t items, chunks;
  Div by_blocks;
};
struct AppendArgs {
  AppendSide side[3];
  uint64_t table, positions, slots;
  uint32_t ps[2], ls[2], ts;                         // strides of positions, slots: B, S; of the table's rows
  uint32_t seq, d, half, places, pages, page, group;
  Div by_seq, by_page;
  uint32_t dtype, format;
  uint32_t vec, pairs;                               // rows in vectors (the rules are at the packing); neighbours are rotated together
};
struct AttendArgs {
  uint64_t q, out, table, lengths, part, stats;      // part, stats: the pieces' sums [pieces, rows, D] and [pieces, rows, 2]
  CachePart kv[2];
  uint32_t qs[4], os[4], ps[2], ls;                  // strides: B, S, H, D; of the page table, the lengths
  uint32_t b, s, hq, hk, per, d, pages, page, group, longest, window;      // per: heads of queries that share one of keys
  uint32_t rows, tiles, pieces;                      // rows: queries of a head of keys, per * S; tiles of them, and of parts of results; pieces of a sequence
  uint32_t by_fours;                                 // scales of 32 elements each, side by side: read in fours
  uint32_t by_head, heads;                           // a wavefront has a head of its own: heads of keys in fours (else heads)
  uint32_t lg_parts;                                 // parts of a result that are a workgroup each: 1 or 2
  uint32_t joined;                                   // a second launch makes the results out of the pieces' sums
  uint32_t blocks, inner;                            // workgroups, and how many that follow each other go to one die
  Div by_page, by_per, by_tiles, by_inner, by_pieces, by_rows, by_heads, by_hk, by_group;
  uint32_t dtype;
  float scale;                                       // of the scores, in powers of two
};

constexpr uint32_t kAppendBlock = 2;       // heads of an item
constexpr uint32_t kTileRows = 16;         // queries of a tile: a side of a matrix instruction's result
constexpr uint32_t kJoinThreads = 512;     // a workgroup of the second launch: a wavefront a query, or all of them
constexpr int64_t kJoinedMost = (1 << 26) - 8;      // heads of queries that it takes, eight a workgroup: a grid of fewer than 2^32 threads
constexpr uint32_t kPiecesMost = 256;      // (one sequence of 131,072 rows, 8 heads, in 128 / 256 / 384: 61, 44, 48 us, and 5.8, 7.1, 7.5 for joining)

// Elements of a head that the kernel of a head's d has room for.
constexpr uint32_t attend_room(uint32_t d, uint32_t dt) { return d == 64u && dt != GPUOS_F32 ? 64u : (d <= 128u ? 128u : 256u); }
// LDS: the queries' parts; for each wavefront a slab, where its rows lie, their scales; or, in their place, sums to be joined.
// Dynamic, because the compiler goes by what it knows of LDS when it chooses how many registers to take: with 45 KB it took 168, and a
// workgroup has to fit into the 128 (and the 69,808 bytes) that a worker of three workgroups a compute unit leaves.
constexpr uint32_t kSlab = 4096;           // bytes of codes that a wavefront has in LDS: 64 rows by 64
constexpr uint32_t attend_wave_lds(uint32_t dp, bool multi) { return kSlab + 1024u + (multi ? dp / 32u : 1u) * 512u; }
constexpr uint32_t attend_q_lds(uint32_t dp, uint32_t dt) { return (dt == GPUOS_BF16 ? 1u : (dt == GPUOS_F16 ? 2u : 3u)) * (dp / 32u) * 1024u; }
constexpr uint32_t attend_lds(uint32_t dp, uint32_t dt, bool multi, bool by_head) {
  const uint32_t loop = attend_q_lds(dp, dt) * (by_head ? 4u : 1u) + 4u * attend_wave_lds(dp, multi), join = 2u * 16u * (dp < 128u ? dp : 128u) * 4u + 512u;
  return loop > join ? loop : join;
}
constexpr uint32_t kLdsMost = 65536;
static_assert(attend_lds(256, GPUOS_F32, true, false) <= kLdsMost, "what a launch may ask for");

int launch_append(const AppendArgs& a, void* stream);       // gpuos_cache.hip
int launch_attend(const AttendArgs& a, uint32_t format, void* stream);

// Checks and packs one descriptor.
class CachePack : ModelPack {
 public:
  static constexpr uint32_t kHead = 256;   // elements of a head that attention takes
  static constexpr int64_t kRowsMost = 1 << 30;      // rows of a sequence: what a place is computed from stays within 32 bits
  static constexpr uint64_t kBlocksMost = 14000000;      // workgroups of a launch: a grid, an eighth larger, has fewer than 2^32 threads

  static int append(const gpuos_cache_task& t, AppendArgs* a, bool* empty) {
    memset(a, 0, sizeof(*a));
    if (t.op != GPUOS_CACHE_APPEND || (t.flags & ~GPUOS_FLAG_PAIRS)) return GPUOS_E_INVAL;
    if (!in_range(t, 10)) return GPUOS_E_INVAL;
    const int64_t *z = t.size, b = z[0], s = z[1], hq = z[2], hk = z[3], d = z[4], rot = z[5], places = z[6], pages = z[7], page = z[8], groups = z[9];
    if (!fits(b, s, hq + 2 * hk, d) || d < 1 || d > (int64_t)kModelRow || rot > d || rot % 2 != 0) return GPUOS_E_INVAL;
    const gpuos_model_operand *q = &t.operand[0], *k = &t.operand[1], *v = &t.operand[2], *table = &t.operand[3], *pos = &t.operand[4], *slots = &t.operand[5],
                              *out = &t.operand[6];
    const bool some = b * s != 0, keys = some && hk != 0, queries = some && hq != 0;
    *empty = !keys && !queries;
    const int64_t qz[4] = {b, s, hq, d}, kz[4] = {b, s, hk, d}, tz[2] = {places, rot};
    if ((keys && (!k->ptr || !v->ptr || !slots->ptr)) || (queries && (!q->ptr || !out->ptr))) return GPUOS_E_INVAL;
    const uint32_t dt = k->dtype;
    if (!is_float(dt) || v->dtype != dt || (hq != 0 && (q->dtype != dt || out->dtype != dt))) return GPUOS_E_INVAL;
    AppendSide &sq = a->side[0], &sk = a->side[1], &sv = a->side[2];
    if (hq != 0 && (!operand(*q, 4, qz, false, false, sq.xs) || !operand(*out, 4, qz, true, false, sq.ts))) return GPUOS_E_INVAL;
    if (!operand(*k, 4, kz, false, false, sk.xs) || !operand(*v, 4, kz, false, false, sv.xs)) return GPUOS_E_INVAL;
    if (slots->dtype != GPUOS_I32 || !operand(*slots, 2, kz, false, false, a->ls)) return GPUOS_E_INVAL;
    uint32_t ts[2] = {0, 0};
    if (rot > 0) {
      if (places < 1 || !table->ptr || table->dtype != GPUOS_F32 || !operand(*table, 2, tz, false, true, ts)) return GPUOS_E_INVAL;
      if (pos->ptr && (pos->dtype != GPUOS_I32 || !operand(*pos, 2, kz, false, false, a->ps))) return GPUOS_E_INVAL;
    }
    CachePart kv[2];
    const int rc = caches(t, 7, hk, d, pages, page, groups, true, keys && pages != 0, 8, kv, &a->format);
    if (rc != GPUOS_OK) return rc;
    sq.x = (uint64_t)q->ptr; sk.x = (uint64_t)k->ptr; sv.x = (uint64_t)v->ptr;
    sq.to = (uint64_t)out->ptr;
    for (int c = 0; c < 2; ++c) {
      AppendSide& side = a->side[1 + c];
      side.to = kv[c].cache;
      side.scales = kv[c].scales;
      for (int i = 0; i < 3; ++i) side.ts[i] = kv[c].cs[i];
      for (int i = 0; i < 4; ++i) side.ss[i] = kv[c].ss[i];
    }
    a->table = rot > 0 ? (uint64_t)table->ptr : 0;
    a->positions = rot > 0 ? (uint64_t)pos->ptr : 0;
    a->slots = (uint64_t)slots->ptr;
    a->ts = ts[0];
    a->seq = (uint32_t)s; a->d = (uint32_t)d;
    a->half = (uint32_t)(rot / 2); a->places = (uint32_t)places;
    a->pages = (uint32_t)pages; a->page = (uint32_t)page; a->group = (uint32_t)(d / groups);
    a->dtype = dt;
    a->pairs = (t.flags & GPUOS_FLAG_PAIRS) ? 1u : 0u;
    if (*empty) return GPUOS_OK;
    a->by_seq = make_div(a->seq);
    a->by_page = make_div(a->page);
    // Vectors: a lane takes eight elements that are all rotated by the same half of the pairs, or not rotated.
    const bool dense = (hq == 0 || (sq.xs[3] == 1 && sq.ts[3] == 1)) && (hk == 0 || (sk.xs[3] == 1 && sv.xs[3] == 1));
    a->vec = dense && d % 8 == 0 && (a->pairs ? rot : rot / 2) % 8 == 0 ? 1u : 0u;
    const uint32_t block = a->vec ? kAppendBlock : 1;
    uint32_t lanes = 1;
    while (lanes < (a->d + 7) / 8) lanes *= 2;
    const uint32_t pass = kThreads / lanes;
    for (int c = 0; c < 3; ++c) {
      AppendSide& side = a->side[c];
      side.heads = (uint32_t)(c == 0 ? hq : hk);
      side.blocks = (side.heads + block - 1) / block;
      side.by_blocks = make_div(side.blocks);
      side.items = (uint32_t)(b * s) * side.blocks;
      const uint64_t passes = ((uint64_t)side.items + pass - 1) / pass;
      side.chunks = passes < 65536 ? (uint32_t)passes : 65536u;
    }
    return GPUOS_OK;
  }

  // *bytes: what the pieces' sums take, 0 if there is one piece; by sizes alone, so that of the two ways to share out the heads (by_head) the one that
  // has more pieces, whichever strides and dtypes choose
  static int attend(const gpuos_cache_task& t, AttendArgs* a, uint32_t* format, uint64_t* bytes, bool* empty) {
    memset(a, 0, sizeof(*a));
    *bytes = 0;
    if (t.op != GPUOS_CACHE_ATTENTION || t.flags != 0 || !in_range(t, 11)) return GPUOS_E_INVAL;
    const int64_t *z = t.size, b = z[0], s = z[1], hq = z[2], hk = z[3], d = z[4], pages = z[5], page = z[6], groups = z[7], width = z[8], longest = z[9], window = z[10];
    if (!fits(b, s, hq, d) || d < 8 || d > (int64_t)kHead || d % 8 != 0) return GPUOS_E_INVAL;
    *empty = b * s * hq == 0;
    if (hk < 1 || hq % hk != 0 || hk > kMost / (b > 0 ? b : 1)) return GPUOS_E_INVAL;
    if (!*empty && pages < 1) return GPUOS_E_INVAL;
    const gpuos_model_operand *q = &t.operand[0], *table = &t.operand[5], *lengths = &t.operand[6], *out = &t.operand[7];
    const int64_t qz[4] = {b, s, hq, d}, pz[2] = {b, width};
    if (!*empty && (!q->ptr || !out->ptr || (longest != 0 && !table->ptr))) return GPUOS_E_INVAL;
    if (!is_float(q->dtype) || out->dtype != q->dtype || !operand(*q, 4, qz, false, false, a->qs) || !operand(*out, 4, qz, true, false, a->os)) return GPUOS_E_INVAL;
    if (table->dtype != GPUOS_I32 || !operand(*table, 2, pz, false, false, a->ps)) return GPUOS_E_INVAL;
    if (lengths->ptr && (lengths->dtype != GPUOS_I32 || !operand(*lengths, 1, pz, false, false, &a->ls))) return GPUOS_E_INVAL;
    const int rc = caches(t, 1, hk, d, pages, page, groups, false, !*empty, 32, a->kv, format);
    if (rc != GPUOS_OK) return rc;
    if (longest > width * page || longest > kRowsMost) return GPUOS_E_INVAL;      // the table names every row there may be
    if (!(t.alpha == t.alpha)) return GPUOS_E_INVAL;
    a->q = (uint64_t)q->ptr; a->out = (uint64_t)out->ptr; a->table = (uint64_t)table->ptr; a->lengths = (uint64_t)lengths->ptr;
    a->b = (uint32_t)b; a->s = (uint32_t)s; a->hq = (uint32_t)hq; a->hk = (uint32_t)hk; a->per = (uint32_t)(hq / hk); a->d = (uint32_t)d;
    a->pages = (uint32_t)pages; a->page = (uint32_t)page; a->group = (uint32_t)(d / groups); a->longest = (uint32_t)longest; a->window = window >= longest ? 0u : (uint32_t)window;      // (one that cuts nothing off is none)
    a->dtype = q->dtype;
    a->scale = t.alpha * 1.44269504088896340736f;
    if (*empty) return GPUOS_OK;
    a->rows = a->per * a->s;
    a->lg_parts = d > 128 ? 1u : 0u;
    a->tiles = ((a->rows + kTileRows - 1) / kTileRows) << a->lg_parts;
    // what a tile of queries sees, at most
    const int64_t seen = a->window != 0 && window + s - 1 < longest ? window + s - 1 : longest;
    a->by_fours = a->group == 32 && a->kv[0].ss[3] == 1 && a->kv[1].ss[3] == 1 ? 1u : 0u;
    // Four heads of a row that lie together are read together, by a wavefront each, if their queries fit into LDS; else a workgroup has a head, and its
    // wavefronts every fourth 64 rows.  64 sequences of 4,096 rows of 8 heads of 128, int8: 134 and 162 us, 4 bits 75 and 80.  (Short ones are cut into
    // rows all the same: with a head each a wavefront has more of them behind each other.)  Pages of one place, whose stride stands for 0, count as heads apart;
    // the limit of 3 heads is not measured (of 5, three wavefronts of eight have none).
    const bool few = hk >= 3 && seen > 512 && a->rows <= 2 * kTileRows;
    a->by_head = few && a->kv[0].cs[2] < a->kv[0].cs[1] && attend_lds(attend_room(a->d, q->dtype), q->dtype, groups > 1, true) <= kLdsMost ? 1u : 0u;
    a->heads = a->by_head ? (a->hk + 3) / 4 : a->hk;
    const uint64_t pairs = (uint64_t)b * a->heads * a->tiles;
    a->pieces = pieces(pairs, (uint64_t)seen, a->by_head ? 128 : 512);
    const uint32_t most = few ? pieces((uint64_t)b * ((a->hk + 3) / 4) * a->tiles, (uint64_t)seen, 128) : a->pieces;
    if (pairs * a->pieces > kBlocksMost) return GPUOS_E_INVAL;
    a->blocks = (uint32_t)(pairs * a->pieces);
    // All heads of a piece of a sequence go to one die, if the dies then have about as much to do; else all queries of a head; else each workgroup to the
    // next.  (By the first rule alone 1,024 queries of one sequence were all on one die: 825 us, so 130.)
    const uint32_t inners[2] = {a->heads * a->tiles, a->tiles};
    a->inner = 1;
    for (uint32_t n : inners) {
      const uint32_t outer = a->blocks / n;
      if ((outer + 7) / 8 * 8 * 8 <= outer * 9) { a->inner = n; break; }
    }
    a->by_page = make_div(a->page);
    a->by_per = make_div(a->per);
    a->by_group = make_div(a->group);
    a->by_tiles = make_div(a->tiles);
    a->by_inner = make_div(a->inner);
    a->by_pieces = make_div(a->pieces);
    a->by_rows = make_div(a->rows);
    a->by_heads = make_div(a->heads);
    a->by_hk = make_div(a->hk);
    if (most > 1) *bytes = (uint64_t)most * GPUOS_CACHE_SUMS_BYTES((uint64_t)b, s, hq, d);
    // In place two workgroups that have a query's parts would read it and store over it: the second launch stores, as it does for pieces.
    // (1,024 queries of 32 heads of 256 over 4,096 rows 321 us, in place 332; 256 sequences of 300 rows 48 and 52.)
    a->joined = a->pieces > 1 || (a->lg_parts != 0 && a->out == a->q) ? 1u : 0u;
    if (a->joined && b * s * hq > kJoinedMost) return GPUOS_E_INVAL;
    return GPUOS_OK;
  }

  // Pieces that a sequence's rows are cut into, each a workgroup's, of 512 rows at least, of 128 where a wavefront has a head (one sequence of 301 rows: 9.0 us,
  // in two pieces 6.5 and 3.7 for joining), for 768 workgroups (three a compute unit); a second launch joins them.
  // 64 sequences of 2,048 to 4,096 rows of 8 heads of 128, 4 bits, in 512 / 768 / 1,024 / 1,536 workgroups: 56, 55, 56, 62 us (with pieces
  // of one length for all sequences, so more of them for the longer ones, 67).
  static uint32_t pieces(uint64_t pairs, uint64_t seen, uint64_t least) {
    uint64_t n = (768 + pairs - 1) / pairs;
    const uint64_t most = (seen + least - 1) / least;
    if (n > most) n = most;
    if (n > kPiecesMost) n = kPiecesMost;
    return n < 1 ? 1u : (uint32_t)n;
  }

 private:
  static bool in_range(const gpuos_cache_task& t, int n) {
    for (int k = 0; k < n; ++k)
      if (t.size[k] < 0 || t.size[k] > kMost) return false;
    return true;
  }
  static bool fits(int64_t b, int64_t s, int64_t h, int64_t d) { return b * s <= kMost && h <= kMost && (b * s == 0 || h <= kMost / (b * s)) && d <= kMost; }
  // keys' cache and scales, values' cache and scales: operands `first` to first + 3
  static int caches(const gpuos_cache_task& t, int first, int64_t hk, int64_t d, int64_t pages, int64_t page, int64_t groups, bool out, bool used, int64_t least,
                    CachePart* kv, uint32_t* format) {
    if (groups < 1 || d % groups != 0 || page < 1 || pages > kMost / page) return GPUOS_E_INVAL;
    const int64_t group = d / groups;
    if (groups > 1 && (group < least || (group & (group - 1)) != 0)) return GPUOS_E_INVAL;
    const uint32_t dt = t.operand[first].dtype;
    if (dt != GPUOS_I8 && dt != GPUOS_E4M3 && dt != GPUOS_E2M1) return GPUOS_E_INVAL;
    if (dt == GPUOS_E2M1 && d % 2 != 0) return GPUOS_E_INVAL;
    *format = dt == GPUOS_E2M1 ? CF_E2M1 : (dt == GPUOS_I8 ? CF_I8 : CF_E4M3);
    const int64_t cz[4] = {pages, page, hk, dt == GPUOS_E2M1 ? d / 2 : d}, sz[4] = {pages, page, hk, groups};
    for (int k = 0; k < 2; ++k) {
      gpuos_model_operand cache = t.operand[first + 2 * k];
      const gpuos_model_operand& scales = t.operand[first + 2 * k + 1];
      uint32_t cs[4];
      if (cache.dtype != dt || scales.dtype != GPUOS_F32 || (used && (!cache.ptr || !scales.ptr))) return GPUOS_E_INVAL;
      cache.dtype = GPUOS_I8;                        // (bytes, as far as strides go)
      if (!operand(cache, 4, cz, out, true, cs) || !operand(scales, 4, sz, out, false, kv[k].ss)) return GPUOS_E_INVAL;
      for (int i = 0; i < 3; ++i) kv[k].cs[i] = cs[i];
      kv[k].cache = (uint64_t)cache.ptr;
      kv[k].scales = (uint64_t)scales.ptr;
    }
    return GPUOS_OK;
  }
};

}  // namespace gpuos
