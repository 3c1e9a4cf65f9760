// gpuos_model.h -- model operators (gpuos_model_task): their bodies of the 256-byte ring record and, for
// the host, the check of a descriptor and its packing.  Shared by the host runtime, the worker's
// executors and the kernels of gpuos_launch_model.
#pragma once
#include <stddef.h>
#include <stdint.h>
#include <string.h>

#include <initializer_list>

#include "../../include/gpuos.h"
#include "gpuos_internal.h"

namespace gpuos {

// n / d for n < 2^31 by a multiplication: (n * mul) >> shift, mul = floor(2^(31 + l) / d) + 1 with
// l = ceil(log2 d).  (mul * d exceeds 2^(31 + l) by at most d <= 2^l, so the product is off by less than n / 2^31 < 1 in
// units of 1 / d.)  {1, 0} divides by one, {0, 0} by more than any n.
struct Div { uint32_t mul, shift; };
inline Div make_div(uint32_t d) {
  uint32_t l = 0;
  while ((1ull << l) < d) ++l;
  return d <= 1 ? Div{1u, 0u} : Div{(uint32_t)((1ull << (31 + l)) / d + 1), 31 + l};
}
GPUOS_HD inline uint32_t divided(uint32_t n, Div d) { return (uint32_t)(((uint64_t)n * d.mul) >> d.shift); }

// What every record begins with (the words of Record that a model operator has a use for), then a body of its own.
// The pieces that the dispatcher fills in and the check word lie where they do in Record.
struct ModelHead {
  uint16_t op_id;
  uint8_t  path;                   // PATH_MODEL
  uint8_t  vec;                    // 1: rows in vectors (the rules are at the packing)
  uint8_t  flags;                  // MF_*
  uint8_t  dtype[4];               // x, out, and per operator
  uint8_t  rflags;
  uint8_t  block;                  // heads of a token that an item has
  uint8_t  pad0[2];
  uint8_t  sel;
  uint8_t  pad1[2];
  uint32_t impl, version;
  int32_t  status;
  uint32_t nchunks;
  uint32_t chunk;                  // items (blocks of heads, segments of rows) in a chunk, at most
  uint32_t items;                  // ... and in all
  uint32_t d;                      // elements of a row
  float    alpha;
  uint16_t dep[3];
  uint16_t run;
  uint64_t ticket;
};
static_assert(sizeof(ModelHead) == 64 && offsetof(ModelHead, rflags) == offsetof(Record, rflags) && offsetof(ModelHead, sel) == offsetof(Record, sel) &&
              offsetof(ModelHead, impl) == offsetof(Record, impl) && offsetof(ModelHead, nchunks) == offsetof(Record, nchunks) &&
              offsetof(ModelHead, chunk) == offsetof(Record, chunk) && offsetof(ModelHead, items) == offsetof(Record, numel) &&
              offsetof(ModelHead, dep) == offsetof(Record, dep) && offsetof(ModelHead, run) == offsetof(Record, run) &&
              offsetof(ModelHead, ticket) == offsetof(Record, ticket) && offsetof(ModelHead, path) == offsetof(Record, path), "the words the dispatcher and the worker read");
enum ModelFlag : uint8_t { MF_PAIRS = 1, MF_LINES = 2 };      // neighbours are pairs; what a store of a wavefront writes of an output row is whole blocks of 64 bytes

struct alignas(16) RopeRecord {    // NORM_ROPE, NORM_ROPE_GRAD, GAMMA_SUM
  ModelHead h;                     // dtype: x, out, gamma, dout
  uint64_t x, gamma, table, positions, out, dout, partial;
  uint32_t xs[4], os[4], zs[4];    // strides of x, out, dout: B, S, H, D
  uint32_t gs, ts, ps[2], cs;      // of gamma, the table's rows, positions, the partial sums' rows
  uint32_t half, places;           // R / 2, rows of the table
  uint32_t seq, heads;             // S, H
  Div by_seq;
  uint32_t pad0;
  uint32_t unused[2];              // (t_dequeue)
  Div by_blocks;
  uint32_t blocks;                 // of heads
  uint32_t spare[4];
  uint32_t check;
};
struct alignas(16) CacheRecord {   // CACHE_STORE, CACHE_LOAD
  ModelHead h;                     // dtype: x or out, cache
  uint64_t x, cache, scales, slots, lengths;       // x: the rows outside the cache; slots: or the page table
  uint32_t xs[4], cs[3], ss[4];    // strides of x: B, S, H, D; of the cache: page, place, head; of the scales: page, place, head, group
  uint32_t ps[2], ls;              // of slots (or the table), lengths
  uint32_t pages, page, group;
  uint32_t heads, blocks;
  Div by_blocks;
  uint32_t pad0[7];
  uint32_t unused[2];              // (t_dequeue)
  uint32_t seq;
  Div by_seq, by_page, by_group;   // (by_group: CACHE_LOAD element by element)
  uint32_t check;
};
struct alignas(16) PenaltyRecord { // LOGIT_PENALTY
  ModelHead h;                     // dtype: x, out, bias; d = V
  uint64_t x, out, history, prompts, params, bias, allowed;
  uint32_t xs[2], os[2], hs[2], ps, ms[2], bs[2], as[2];     // strides: B, last (prompts: B)
  uint32_t n;                      // N
  uint32_t seg;                    // elements of a segment
  Div by_segs;                     // segments of a row
  uint32_t segs;
  uint32_t pad0[6];
  uint32_t unused[2];              // (t_dequeue)
  uint32_t spare[7];
  uint32_t check;
};
union alignas(16) ModelRecord {
  ModelHead h;
  RopeRecord rope;
  CacheRecord cache;
  PenaltyRecord penalty;
  Record ring;
};
static_assert(sizeof(RopeRecord) == 256 && sizeof(CacheRecord) == 256 && sizeof(PenaltyRecord) == 256 && sizeof(ModelRecord) == 256, "ring record");
static_assert(offsetof(RopeRecord, unused) == offsetof(Record, t_dequeue) && offsetof(CacheRecord, unused) == offsetof(Record, t_dequeue) &&
              offsetof(PenaltyRecord, unused) == offsetof(Record, t_dequeue) && offsetof(RopeRecord, check) == offsetof(Record, check) &&
              offsetof(CacheRecord, check) == offsetof(Record, check) && offsetof(PenaltyRecord, check) == offsetof(Record, check), "the words the dispatcher writes");

constexpr uint32_t kModelRow = 512;          // elements of a head, at most: 64 lanes of eight
constexpr uint32_t kModelParts = 1024;       // shares of the gradient of gamma, at most (a unit names its chunk in ten bits)
// Lanes that a row of vectors takes: a lane has four pairs, or eight elements that are not rotated (neighbours: eight elements).
GPUOS_HD inline uint32_t rope_units(uint32_t d, uint32_t half, bool pairs) { return pairs ? (d + 7u) / 8u : (half + 3u) / 4u + (d - 2u * half + 7u) / 8u; }
// Heads of an item that goes in vectors.  More of them share a token's position, slot and page and have more on their way at once, but the
// code grows with them and a short call waits for it: 2, 4 and 8 heads (the gradient: 1, 2 and 4) take, for 16 heads of one token
// and for 327,680 of 128 bf16, norm and rotation 3.6, 4.3, 6.0 and 38.3, 36.9, 35.0 us, the gradient (262,144 heads) 4.2, 4.8, 6.0 and 56.1, 50.3, 49.2;
// storing 2.4, 3.0, 4.7 and 19.2, 19.8, 22.7 (262,144 heads), reading back 2.2, 2.5, 3.1 and 179, 159, 157 (2,097,152 heads).
constexpr uint32_t kRopeBlock = 4, kGradBlock = 2, kStoreBlock = 2, kLoadBlock = 4;
// In the ring, whose workgroups do not make up for each other's waits: twice as many of the cache's (744 MB read back 193 -> 168 us, 100 MB stored
// 52 -> 49, a token's the same); of rotations they made a token 17 us of 14, and 172 MB 64 of 69.
constexpr uint32_t kRingStoreBlock = 4, kRingLoadBlock = 8;
constexpr uint32_t kModelLaunch = 8;         // tasks of one launch: their records are kernel arguments, 2 KB of the 4 KB there may be

// What gpuos_launch_model hands a kernel: tasks of one variant.  (A block's second index is its task's place here: its
// record is then one trip to memory away, with a table of first blocks it was two.)
struct alignas(16) ModelLaunch {
  ModelRecord rec[kModelLaunch];
};
int hip_status(int e, const char* what);     // GPUOS_OK, or GPUOS_E_HIP with gpuos_last_hip_error() set (gpuos_runtime.cpp)
int launch_model(const ModelLaunch& l, uint32_t variant, uint32_t chunks, uint32_t tasks, void* stream);      // gpuos_model.hip

inline bool impl_is_model(uint32_t impl) { return impl >= GPUOS_IMPL_NORM_ROPE && impl <= GPUOS_IMPL_LOGIT_PENALTY; }
inline int model_arity(uint32_t impl) {
  switch (impl) {
    case GPUOS_IMPL_NORM_ROPE: case GPUOS_IMPL_CACHE_LOAD: return 5;
    case GPUOS_IMPL_NORM_ROPE_GRAD: case GPUOS_IMPL_LOGIT_PENALTY: return 7;
    case GPUOS_IMPL_GAMMA_SUM: return 2;
    case GPUOS_IMPL_CACHE_STORE: return 4;
    default: return -1;
  }
}

// The executors of the operators, one after the other: rows in vectors by dtype (rotations: halves, then neighbours), then element by
// element.  A kernel and a function of the worker each, so that none has the registers of another.
enum ModelVariant : uint32_t { MV_ROPE = 0, MV_GRAD = 7, MV_SUM = 14, MV_STORE = 15, MV_LOAD = 19, MV_PENALTY = 23, MV_COUNT = 27 };
GPUOS_HD inline uint32_t model_variant(uint32_t impl, uint32_t vec, uint32_t dtype, uint32_t flags) {
  if (impl == GPUOS_IMPL_GAMMA_SUM) return MV_SUM;
  if (impl <= GPUOS_IMPL_NORM_ROPE_GRAD) return (impl == GPUOS_IMPL_NORM_ROPE ? MV_ROPE : MV_GRAD) + (vec == 0 ? 6u : dtype + ((flags & MF_PAIRS) ? 3u : 0u));
  return (impl == GPUOS_IMPL_CACHE_STORE ? MV_STORE : (impl == GPUOS_IMPL_CACHE_LOAD ? MV_LOAD : MV_PENALTY)) + (vec == 0 ? 3u : dtype);
}

// How a task is cut: chunks of at least so many bytes, at most so many; and whether vectors have to be aligned (the worker's accesses of
// 8 bytes go by atomic loads and stores, a kernel's by ordinary ones, which gfx950 takes at any address of an element).
// Of the passes that a workgroup makes over all items, chunk c makes every nchunks-th from the c-th on, so that what is worked on at a
// time lies together in memory: 2,097,152 heads read back in 2,048 chunks of passes that follow each other took 159 us, in 4,096 148, in
// 16,384, a pass each, 124.
struct ModelCut { uint32_t least_bytes, most; bool aligned; uint32_t store_block, load_block; };
constexpr ModelCut kRingCut{16384, kMaxChunksPerTask, true, kRingStoreBlock, kRingLoadBlock};       // a unit costs the dispatcher 12 ns and the worker about a microsecond
constexpr ModelCut kLaunchCut{4096, 65536, false, kStoreBlock, kLoadBlock};

// Checks and packs one descriptor.
class ModelPack {
 public:
  // GPUOS_OK, or why not; *r holds something only if GPUOS_OK
  static int pack(const gpuos_model_task& t, uint32_t impl, ModelRecord* r, ModelCut cut) {
    memset(r, 0, sizeof(*r));
    ModelHead& h = r->h;
    h.op_id = t.op_id;
    h.impl = impl;
    h.alpha = t.alpha;
    for (int k = 0; k < 3; ++k) h.dep[k] = t.dep[k];
    if (t.flags & ~(GPUOS_FLAG_FENCE | GPUOS_FLAG_PAIRS)) return GPUOS_E_INVAL;
    if (t.flags & GPUOS_FLAG_FENCE) h.rflags = RF_FENCE;
    if (impl == GPUOS_IMPL_FAIL) {                   // executes nothing; one unit reports it
      h.path = PATH_NOP;
      h.nchunks = 1;
      return GPUOS_OK;
    }
    if (!impl_is_model(impl)) return GPUOS_E_BADOP;
    if (t.n_operands != model_arity(impl)) return GPUOS_E_INVAL;
    const bool rope = impl == GPUOS_IMPL_NORM_ROPE || impl == GPUOS_IMPL_NORM_ROPE_GRAD;
    if ((t.flags & GPUOS_FLAG_PAIRS) && !rope) return GPUOS_E_INVAL;
    if (t.flags & GPUOS_FLAG_PAIRS) h.flags = MF_PAIRS;
    h.path = PATH_MODEL;
    int rc;
    if (rope) rc = pack_rope(t, r->rope, impl == GPUOS_IMPL_NORM_ROPE_GRAD, cut);
    else if (impl == GPUOS_IMPL_GAMMA_SUM) rc = pack_sum(t, r->rope, cut);
    else if (impl == GPUOS_IMPL_LOGIT_PENALTY) rc = pack_penalty(t, r->penalty, cut);
    else rc = pack_cache(t, r->cache, impl == GPUOS_IMPL_CACHE_STORE, cut);
    if (rc == GPUOS_OK && h.items == 0) {
      h.path = PATH_NOP;
      h.nchunks = 1;
    }
    return rc;
  }

 protected:
  static constexpr int64_t kMost = 2147483647LL;     // rows, and elements of one dim
  static constexpr int64_t kExtent = 1LL << 46;      // elements from an operand's first to its last
  static uint32_t size_of(uint32_t dt) { return dt >= GPUOS_I8 ? 1u : (dt == GPUOS_F32 || dt == GPUOS_I32 ? 4u : 2u); }
  static bool is_float(uint32_t dt) { return dt <= GPUOS_BF16; }

  // (What has no elements may have no address: a task without rows, a cache without pages.)
  // An operand of nd dims: its strides (0 where the dim has one element), or false.  `out`: no two elements share memory as far as
  // strides of 0 go; `dense`: the last dim's stride is 1.
  static bool operand(const gpuos_model_operand& o, int nd, const int64_t* size, bool out, bool dense, uint32_t* st) {
    if (o.dtype > GPUOS_E4M3 || (uint64_t)o.ptr % size_of(o.dtype) != 0) return false;
    int64_t extent = 0;
    bool empty = false;
    for (int d = 0; d < nd; ++d) empty = empty || size[d] == 0;
    for (int d = 0; d < nd; ++d) {
      const int64_t s = o.stride[d];
      if (s < 0 || s > 0xffffffffLL) return false;
      if (out && s == 0 && size[d] > 1 && !empty) return false;
      if (dense && d == nd - 1 && s != 1 && size[d] > 1) return false;
      if (size[d] > 1) {
        if (s > (kExtent - extent) / (size[d] - 1)) return false;      // (compared before it is added: one dim's part may be close to 2^63)
        extent += (size[d] - 1) * s;
      }
      st[d] = size[d] > 1 ? (uint32_t)s : 0u;
    }
    return true;
  }
  static bool sizes(const gpuos_model_task& t, int n) {
    for (int k = 0; k < n; ++k)
      if (t.size[k] < 0 || t.size[k] > kMost) return false;
    return true;
  }
  // whether rows may be read `unit` elements at a time: the last dim's stride is 1 and, if they have to be aligned, every row begins on 8 bytes
  static bool vectors(ModelCut cut, uint64_t ptr, uint32_t es, const uint32_t* st, int outer, bool last_dense) {
    bool ok = last_dense;
    if (!cut.aligned) return ok;
    ok = ok && ptr % 8 == 0;
    for (int d = 0; d < outer; ++d) ok = ok && (uint64_t)st[d] * es % 8 == 0;
    return ok;
  }
  // The heads of a token in blocks of `block`.
  template <class RECORD> static void in_blocks(RECORD& r, uint64_t tokens, uint32_t block) {
    r.h.block = (uint8_t)block;
    r.blocks = (r.heads + block - 1) / block;
    r.by_blocks = make_div(r.blocks);
    r.h.items = (uint32_t)(tokens * r.blocks);
  }
  // whether the rows of an output begin on blocks of 64 bytes, and parts of so many elements are whole blocks
  static bool lines(uint64_t ptr, uint32_t es, const uint32_t* st, int outer, uint32_t part) {
    bool ok = ptr % 64 == 0 && (uint64_t)part * es % 64 == 0;
    for (int d = 0; d < outer; ++d) ok = ok && (uint64_t)st[d] * es % 64 == 0;
    return ok;
  }
  // Items in chunks, `pass` of them at a time.
  static void cut_items(ModelHead& h, ModelCut cut, uint64_t item_bytes, uint32_t pass) {
    const uint64_t passes = ((uint64_t)h.items + pass - 1) / pass, pass_bytes = item_bytes * pass;
    uint64_t per = (cut.least_bytes + pass_bytes - 1) / pass_bytes;
    const uint64_t even = (passes + cut.most - 1) / cut.most;
    if (per < even) per = even;
    h.nchunks = passes == 0 ? 1u : (uint32_t)((passes + per - 1) / per);
    set_most(h, passes, pass);
  }
  static void set_most(ModelHead& h, uint64_t passes, uint32_t pass) {
    const uint64_t most = (passes + h.nchunks - 1) / h.nchunks * pass;
    h.chunk = most < h.items ? (uint32_t)most : h.items;
  }
  // rows that the workgroup's 256 lanes take at once, `lanes` of them each
  static uint32_t rows_at_once(uint32_t lanes) {
    uint32_t p = 1;
    while (p < lanes && p < 64) p *= 2;
    return kThreads / p;
  }

  // B and S as one dim where every operand allows it: the rows then need no division by S (true).
  template <class... ST> static bool join(uint32_t b, uint32_t& seq, ST*... st) {
    const uint32_t s = seq;
    bool ok = true;
    (void)std::initializer_list<int>{(ok = ok && (b <= 1 || (s <= 1 ? true : (uint64_t)st[0] == (uint64_t)st[1] * s)), 0)...};
    if (!ok) return false;
    if (s <= 1 && b > 1) (void)std::initializer_list<int>{(st[1] = st[0], 0)...};
    seq = b * s;
    return true;
  }

  static int pack_rope(const gpuos_model_task& t, RopeRecord& r, bool grad, ModelCut cut) {
    if (!sizes(t, grad ? 7 : 6)) return GPUOS_E_INVAL;
    const int64_t *z = t.size, d = z[3], rot = z[4], places = z[5];
    if (d < 1 || d > (int64_t)kModelRow || rot > d || rot % 2 != 0) return GPUOS_E_INVAL;
    const int64_t tokens = z[0] * z[1];
    if (tokens > kMost || tokens * z[2] > kMost) return GPUOS_E_INVAL;
    const gpuos_model_operand *x = &t.operand[0], *gamma = &t.operand[1], *table = &t.operand[2], *pos = &t.operand[3], *out = &t.operand[4];
    const gpuos_model_operand *dz = &t.operand[grad ? 5 : 0], *part = grad ? &t.operand[6] : nullptr;
    const int64_t xz[4] = {z[0], z[1], z[2], d}, gz[1] = {d}, tz[2] = {places, rot};
    const bool rows = tokens * z[2] != 0;
    if ((rows && (!x->ptr || !out->ptr || !dz->ptr)) || !is_float(x->dtype) || !is_float(out->dtype) || !is_float(dz->dtype)) return GPUOS_E_INVAL;
    if (!operand(*x, 4, xz, false, false, r.xs) || !operand(*out, 4, xz, true, false, r.os) || !operand(*dz, 4, xz, false, false, r.zs)) return GPUOS_E_INVAL;
    if (gamma->ptr && (!is_float(gamma->dtype) || !operand(*gamma, 1, gz, false, false, &r.gs))) return GPUOS_E_INVAL;
    uint32_t ts[2] = {0, 0};
    if (rot > 0) {
      if (places < 1 || !table->ptr || table->dtype != GPUOS_F32 || !operand(*table, 2, tz, false, true, ts)) return GPUOS_E_INVAL;
      if (pos->ptr && (pos->dtype != GPUOS_I32 || !operand(*pos, 2, xz, false, false, r.ps))) return GPUOS_E_INVAL;
    }
    r.h.dtype[0] = x->dtype; r.h.dtype[1] = out->dtype; r.h.dtype[2] = gamma->dtype; r.h.dtype[3] = dz->dtype;
    r.x = (uint64_t)x->ptr; r.out = (uint64_t)out->ptr; r.gamma = (uint64_t)gamma->ptr; r.dout = (uint64_t)dz->ptr;
    r.table = rot > 0 ? (uint64_t)table->ptr : 0;
    r.positions = rot > 0 ? (uint64_t)pos->ptr : 0;
    r.ts = ts[0];
    r.half = (uint32_t)(rot / 2);
    r.places = (uint32_t)places;
    r.heads = (uint32_t)z[2];
    r.seq = (uint32_t)z[1];
    r.h.d = (uint32_t)d;
    // (a position that is the index in S needs S by itself)
    const bool joined = (rot == 0 || pos->ptr) && join((uint32_t)z[0], r.seq, r.xs, r.os, r.zs, r.ps);
    r.by_seq = joined ? Div{0, 0} : make_div(r.seq);
    // Vectors: a lane takes four elements twice, by windows that stay in their part of the row: so a part is nothing or four elements
    // (neighbours: the row eight, of an even number), and all operands are of one dtype.  Where vectors have to be aligned the parts are whole
    // numbers of windows.
    const uint32_t es = size_of(x->dtype), rest = (uint32_t)d - 2u * r.half;
    const bool last = d == 1 || (r.xs[3] == 1 && r.os[3] == 1 && r.zs[3] == 1), pairs = (t.flags & GPUOS_FLAG_PAIRS) != 0;
    const bool parts = pairs ? d >= 8 && d % 2 == 0 : (r.half == 0 || r.half >= 4) && (rest == 0 || rest >= 4);
    if (x->dtype == out->dtype && x->dtype == dz->dtype && parts && rope_units((uint32_t)d, r.half, pairs) <= 64 &&
        (!cut.aligned || (d % 8 == 0 && r.half % 4 == 0)) && vectors(cut, r.x, es, r.xs, 3, last) && vectors(cut, r.out, es, r.os, 3, last) &&
        vectors(cut, r.dout, es, r.zs, 3, last) && vectors(cut, r.table, 4, &r.ts, 1, true))
      r.h.vec = 1;
    // (halves: a wavefront stores either by itself, and of what is not rotated every second four)
    if (lines(r.out, es, r.os, 3, (uint32_t)d) && (pairs || (rest == 0 && (uint64_t)r.half * es % 64 == 0))) r.h.flags |= MF_LINES;
    in_blocks(r, (uint64_t)tokens, r.h.vec ? (grad ? kGradBlock : kRopeBlock) : 1);
    const uint32_t pass = rows_at_once(r.h.vec ? rope_units((uint32_t)d, r.half, pairs) : (uint32_t)(d + 1) / 2);
    cut_items(r.h, cut, (uint64_t)d * es * (grad ? 3 : 2) * r.h.block, pass);
    if (grad && part->ptr) {
      const int64_t parts = z[6], cz[2] = {d, parts};
      uint32_t cs[2];
      if (parts < 1 || parts > (int64_t)kModelParts || part->dtype != GPUOS_F32 || !operand(*part, 2, cz, true, true, cs)) return GPUOS_E_INVAL;
      if (d > 1 && (int64_t)cs[0] < parts) return GPUOS_E_INVAL;
      r.partial = (uint64_t)part->ptr;
      r.cs = cs[0];
      r.h.nchunks = (uint32_t)parts;                 // every column is written, also of shares with no rows
      set_most(r.h, ((uint64_t)r.h.items + pass - 1) / pass, pass);
      if (r.h.items == 0) {                           // (not an empty task: see pack)
        r.h.vec = 0;
        r.h.items = kNoRows;
      }
    }
    return GPUOS_OK;
  }

  static int pack_sum(const gpuos_model_task& t, RopeRecord& r, ModelCut cut) {
    if (!sizes(t, 2)) return GPUOS_E_INVAL;
    const gpuos_model_operand &part = t.operand[0], &out = t.operand[1];
    uint32_t cs[2];
    if ((!part.ptr && t.size[1] != 0 && t.size[0] != 0) || (!out.ptr && t.size[0] != 0) || part.dtype != GPUOS_F32 || !is_float(out.dtype)) return GPUOS_E_INVAL;
    if (!operand(part, 2, t.size, false, true, cs) || !operand(out, 1, t.size, true, false, r.os)) return GPUOS_E_INVAL;
    r.partial = (uint64_t)part.ptr;
    r.out = (uint64_t)out.ptr;
    r.cs = cs[0];
    r.h.dtype[1] = out.dtype;
    r.h.items = (uint32_t)t.size[0];
    r.h.d = (uint32_t)t.size[1];
    // (a row is a wait for memory and two barriers however short it is: 128 rows of one share each by one workgroup take 49 us, by one each 4)
    cut_items(r.h, cut, r.h.d < 1024 ? 4096u : 4ull * r.h.d, 1);
    return GPUOS_OK;
  }

  static int pack_cache(const gpuos_model_task& t, CacheRecord& r, bool store, ModelCut cut) {
    if (!sizes(t, store ? 7 : 8)) return GPUOS_E_INVAL;
    const int64_t *z = t.size, d = z[3], pages = z[4], page = z[5], groups = z[6];
    const int64_t tokens = z[0] * z[1];
    if (tokens > kMost || tokens * z[2] > kMost || d < 1 || d > (int64_t)kModelRow || groups < 1 || d % groups != 0) return GPUOS_E_INVAL;
    if (page < 1 || pages * page > kMost) return GPUOS_E_INVAL;
    const int64_t group = d / groups;
    if (groups > 1 && (group < 8 || (group & (group - 1)) != 0)) return GPUOS_E_INVAL;
    const gpuos_model_operand &x = t.operand[store ? 0 : 4], &cache = t.operand[store ? 2 : 0], &scales = t.operand[store ? 3 : 1];
    const gpuos_model_operand &slots = t.operand[store ? 1 : 2], &lengths = t.operand[3];
    const int64_t xz[4] = {z[0], z[1], z[2], d}, cz[4] = {pages, page, z[2], d}, sz[4] = {pages, page, z[2], groups};
    const int64_t pz[2] = {z[0], store ? z[1] : z[7]};
    uint32_t cs[4];
    const bool rows = tokens * z[2] != 0;
    if ((rows && (!x.ptr || !slots.ptr || (pages != 0 && (!cache.ptr || !scales.ptr)))) || !is_float(x.dtype) || cache.dtype < GPUOS_I8 || scales.dtype != GPUOS_F32 || slots.dtype != GPUOS_I32)
      return GPUOS_E_INVAL;
    if (!operand(x, 4, xz, !store, false, r.xs) || !operand(cache, 4, cz, store, true, cs) || !operand(scales, 4, sz, store, false, r.ss) ||
        !operand(slots, 2, pz, false, false, r.ps))
      return GPUOS_E_INVAL;
    if (!store) {
      if (z[1] > z[7] * page) return GPUOS_E_INVAL;          // the table names every row there may be
      if (lengths.ptr && (lengths.dtype != GPUOS_I32 || !operand(lengths, 1, pz, false, false, &r.ls))) return GPUOS_E_INVAL;
      r.lengths = (uint64_t)lengths.ptr;
    }
    for (int k = 0; k < 3; ++k) r.cs[k] = cs[k];
    r.h.dtype[0] = x.dtype; r.h.dtype[1] = cache.dtype;
    r.x = (uint64_t)x.ptr; r.cache = (uint64_t)cache.ptr; r.scales = (uint64_t)scales.ptr; r.slots = (uint64_t)slots.ptr;
    r.pages = (uint32_t)pages;
    r.page = (uint32_t)page;
    r.group = (uint32_t)group;
    r.heads = (uint32_t)z[2];
    r.seq = (uint32_t)z[1];
    r.h.d = (uint32_t)d;
    r.by_seq = store && join((uint32_t)z[0], r.seq, r.xs, r.ps) ? Div{0, 0} : make_div(r.seq);
    r.by_page = make_div(r.page);
    r.by_group = make_div(r.group);
    // Vectors: a lane takes eight elements of a row, 8 bytes of the cache.  (A row that is no whole number of eights is one group.)
    const uint32_t es = size_of(x.dtype);
    if (d >= 8 && (!cut.aligned || d % 8 == 0) && vectors(cut, r.x, es, r.xs, 3, r.xs[3] == 1) && vectors(cut, r.cache, 1, r.cs, 3, true)) r.h.vec = 1;
    if (!store && lines(r.x, es, r.xs, 3, (uint32_t)d)) r.h.flags |= MF_LINES;
    in_blocks(r, (uint64_t)tokens, r.h.vec ? (store ? cut.store_block : cut.load_block) : 1);
    cut_items(r.h, cut, (uint64_t)d * (es + 1) * r.h.block, rows_at_once(r.h.vec ? (uint32_t)(d + 7) / 8 : (uint32_t)d));
    return GPUOS_OK;
  }

  static int pack_penalty(const gpuos_model_task& t, PenaltyRecord& r, ModelCut cut) {
    if (!sizes(t, 3)) return GPUOS_E_INVAL;
    const int64_t b = t.size[0], v = t.size[1], n = t.size[2];
    const gpuos_model_operand &x = t.operand[0], &out = t.operand[1], &hist = t.operand[2], &prompt = t.operand[3], &params = t.operand[4],
                              &bias = t.operand[5], &allowed = t.operand[6];
    const int64_t xz[2] = {b, v}, hz[2] = {b, n}, pz[2] = {b, 3}, az[2] = {b, (v + 31) / 32};
    const bool rows = b * v != 0;
    if ((rows && (!x.ptr || !out.ptr)) || !is_float(x.dtype) || !is_float(out.dtype) || !operand(x, 2, xz, false, false, r.xs) || !operand(out, 2, xz, true, false, r.os))
      return GPUOS_E_INVAL;
    if (rows && ((hist.ptr == nullptr) != (params.ptr == nullptr) || (!hist.ptr && (n != 0 || prompt.ptr)))) return GPUOS_E_INVAL;
    if (hist.ptr && (hist.dtype != GPUOS_I32 || params.dtype != GPUOS_F32 || !operand(hist, 2, hz, false, false, r.hs) || !operand(params, 2, pz, false, false, r.ms)))
      return GPUOS_E_INVAL;
    if (prompt.ptr && (prompt.dtype != GPUOS_I32 || !operand(prompt, 1, xz, false, false, &r.ps))) return GPUOS_E_INVAL;
    if (bias.ptr && (!is_float(bias.dtype) || !operand(bias, 2, xz, false, false, r.bs))) return GPUOS_E_INVAL;
    if (allowed.ptr && (allowed.dtype != GPUOS_I32 || !operand(allowed, 2, az, false, false, r.as))) return GPUOS_E_INVAL;
    r.x = (uint64_t)x.ptr; r.out = (uint64_t)out.ptr; r.history = (uint64_t)hist.ptr; r.prompts = (uint64_t)prompt.ptr;
    r.params = (uint64_t)params.ptr; r.bias = (uint64_t)bias.ptr; r.allowed = (uint64_t)allowed.ptr;
    r.h.dtype[0] = x.dtype; r.h.dtype[1] = out.dtype; r.h.dtype[2] = bias.dtype;
    r.n = (uint32_t)n;
    r.h.d = (uint32_t)v;
    if (b == 0 || v == 0) return GPUOS_OK;
    r.seg = kSegment;
    const int64_t segs = (v + r.seg - 1) / r.seg;
    if (segs * b > kMost) return GPUOS_E_INVAL;
    r.segs = (uint32_t)segs;
    r.by_segs = make_div(r.segs);
    r.h.items = (uint32_t)(segs * b);
    const bool bias_ok = !bias.ptr || r.bs[1] == 1 || v == 1, allowed_ok = !allowed.ptr || r.as[1] == 1 || az[1] == 1;
    const uint32_t es = size_of(x.dtype);
    if (x.dtype == out.dtype && vectors(cut, r.x, es, r.xs, 1, v == 1 || r.xs[1] == 1) && vectors(cut, r.out, es, r.os, 1, v == 1 || r.os[1] == 1) &&
        bias_ok && allowed_ok)
      r.h.vec = 1;
    if (lines(r.out, es, r.os, 1, 64)) r.h.flags |= MF_LINES;
    cut_items(r.h, ModelCut{1, cut.most, cut.aligned, 0, 0}, 1, 1);
    return GPUOS_OK;
  }

 public:
  static constexpr uint32_t kNoRows = 0xffffffffu;   // NORM_ROPE_GRAD without rows, whose partial sums are written all the same
  static constexpr uint32_t kSegment = 4096;
};

}  // namespace gpuos
