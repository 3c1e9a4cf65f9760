// gpuos_model_device.h -- device code of the model operators (gpuos_model_task): norm and rotation of heads
// with its gradient, the 8-bit paged cache, penalties on logits.  One set of executors serves the worker
// (POL_COHERENT, called through exec_model) and the kernels of gpuos_launch_model (POL_PLAIN).
#pragma once
#include "gpuos_device.h"
#include "gpuos_model.h"

namespace gpuos {

// ---------------------------------------------------------------------------
// memory access by 64-bit address: rows of a chunk lie at any distance from each other, so there is no buffer resource to go by.
// POL_PLAIN: ordinary accesses, vectors at any address of an element.  POL_COHERENT: atomic ones of 8 bytes and less at the system's
// scope, which go past the caches that another die's writes do not reach; vectors begin on 8 bytes (ModelCut::aligned).
//
// A kernel's vector stores have the non-temporal hint, as those of row operations have it, where each writes whole pieces of 64 bytes
// (MF_LINES): what an operator writes is a matrix product away from its reader, and the inputs stay in the memory-side cache.  Without
// and with it, three sets of buffers in turn: norm and rotation of 84 MB 41.4 and 30.9 us, a sequence of 134 MB read back 41.9 and 25.9,
// penalties on 51 MB 35.6 and 30.1; with an addition that reads the result right behind it 69.4 and 66.2, 91.3 and 86.8, 50.5 and 51.7 (of 42, 34
// and 168 MB 5 and 8 % behind, and 3).  Pieces of such a block that two stores write each go to memory by themselves: 134 MB of fp32, whose eight
// elements are two stores, read back in 27.6 and 54, rows of 100 bf16 in 14.2 and 19.3.
// ---------------------------------------------------------------------------
typedef int v2i __attribute__((ext_vector_type(2)));
template <int POL> struct Glob {
  template <class T> using G = __attribute__((address_space(1))) T;
  typedef v4i __attribute__((aligned(2))) v4i_any;
  typedef v2i __attribute__((aligned(2))) v2i_any;
  typedef v2i __attribute__((aligned(1))) v2i_byte;
  template <class T> static DEV T at(uint64_t p) {
    if (POL == POL_COHERENT) return __hip_atomic_load((G<T>*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
    return *(const G<T>*)p;
  }
  template <class T> static DEV void put(uint64_t p, T v) {
    if (POL == POL_COHERENT) __hip_atomic_store((G<T>*)p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_SYSTEM);
    else *(G<T>*)p = v;
  }
  static DEV v2i ld8(uint64_t p) {
    if (POL == POL_COHERENT) return __builtin_bit_cast(v2i, at<uint64_t>(p));
    return *(const G<v2i_any>*)p;
  }
  // A coherent access of 16 bytes, by a buffer resource: whether the addresses of a wavefront's active lanes lie within a gigabyte of the
  // first one's; then r begins a gigabyte below that, so that no access reaches its end, and p is `off` from it.  (In two of 8 bytes, with gaps
  // of as many between the lanes', a store moves half lines: 744 MB read back from the cache 422 us, so 193.)
  static DEV bool near(uint64_t p, rsrc_t& r, uint32_t& off) {
    const uint64_t first = uni64(p), base = first > (1ull << 30) ? first - (1ull << 30) : 0;
    off = (uint32_t)(p - base);
    r = make_rsrc((const void*)(__UINTPTR_TYPE__)base, 0xffffffffu);
    return __builtin_amdgcn_ballot_w64((p - base) >> 31 != 0) == 0;
  }
  static DEV v4i ld16(uint64_t p) {
    if (POL == POL_COHERENT) {
      rsrc_t r;
      uint32_t off;
      if (near(p, r, off)) return __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, Mem<POL>::BASE);
      const v2i a = ld8(p), b = ld8(p + 8);
      return v4i{a[0], a[1], b[0], b[1]};
    }
    return *(const G<v4i_any>*)p;
  }
  static DEV void apart() { asm volatile(""); }      // (or the compiler makes one store without the hint of the two)
  static DEV void st8(uint64_t p, v2i q, bool nt = false) {
    if (POL == POL_COHERENT) put<uint64_t>(p, __builtin_bit_cast(uint64_t, q));
    else if (nt) { apart(); __builtin_nontemporal_store((v2i_any)q, (G<v2i_any>*)p); apart(); }
    else *(G<v2i_any>*)p = q;
  }
  static DEV void st16(uint64_t p, v4i q, bool nt = false) {
    if (POL == POL_COHERENT) {
      rsrc_t r;
      uint32_t off;
      if (near(p, r, off)) __builtin_amdgcn_raw_buffer_store_b128(q, r, (int)off, 0, Mem<POL>::BASE);
      else { st8(p, v2i{q[0], q[1]}); st8(p + 8, v2i{q[2], q[3]}); }
    } else if (nt) { apart(); __builtin_nontemporal_store((v4i_any)q, (G<v4i_any>*)p); apart(); }
    else *(G<v4i_any>*)p = q;
  }
  static DEV v2i ld8b(uint64_t p) { return POL == POL_COHERENT ? ld8(p) : (v2i)*(const G<v2i_byte>*)p; }      // bytes
  static DEV void st8b(uint64_t p, v2i q) { if (POL == POL_COHERENT) st8(p, q); else *(G<v2i_byte>*)p = q; }
  static DEV float ldf(uint64_t p) { return __builtin_bit_cast(float, at<uint32_t>(p)); }
  static DEV int32_t ldi(uint64_t p) { return (int32_t)at<uint32_t>(p); }
  static DEV void stf(uint64_t p, float f) { put<uint32_t>(p, __builtin_bit_cast(uint32_t, f)); }
  // an element of a float dtype known at run time (the aligned word that holds it: see load_rt)
  static DEV float ld_rt(uint64_t p, uint32_t dt) {
    const uint32_t w = at<uint32_t>(p & ~3ull), h = (p & 2u) ? (w >> 16) : (w & 0xffffu);
    return dt == GPUOS_F32 ? __builtin_bit_cast(float, w) : (dt == GPUOS_F16 ? h2f(h) : b2f(h));
  }
  static DEV void st_rt(uint64_t p, uint32_t dt, float f) {
    if (dt == GPUOS_F32) stf(p, f);
    else put<uint16_t>(p, (uint16_t)(dt == GPUOS_F16 ? f2h(f) : f2b(f)));
  }
  // four and eight elements that follow each other
  template <int DT> static DEV void ld4e(uint64_t p, float* f) {
    const v4i q = Elem<DT>::ES == 4 ? ld16(p) : ([&] { const v2i h = ld8(p); return v4i{h[0], h[1], 0, 0}; })();
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = Elem<DT>::get(q, k);
  }
  template <int DT> static DEV void ld8e(uint64_t p, float* f) {
    if (Elem<DT>::ES == 4) {
      ld4e<DT>(p, f);
      ld4e<DT>(p + 16, f + 4);
    } else {
      const v4i q = ld16(p);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] = Elem<DT>::get(q, k);
    }
  }
};
DEV uint32_t float_size(uint32_t dt) { return dt == GPUOS_F32 ? 4u : 2u; }
DEV uint32_t ceil_log2(uint32_t n) { return n <= 1 ? 0u : 32u - (uint32_t)__builtin_clz(n - 1); }
DEV Div uni_div(uint32_t mul, uint32_t shift) { return Div{uni(mul), uni(shift)}; }

// Eight elements as they lie in memory, in one piece or in two halves.
template <int POL, int DT> struct Eight {
  static constexpr int N = Elem<DT>::ES / 2;
  v4i q[N];
  DEV void clear() {
#pragma unroll
    for (int k = 0; k < N; ++k) q[k] = v4i{0, 0, 0, 0};
  }
  DEV float get(int i) const { return N == 2 ? Elem<DT>::get(q[N == 2 ? i / 4 : 0], i % 4) : Elem<DT>::get(q[0], i); }
  DEV void put(int i, float f) { if (N == 2) Elem<DT>::put(q[N == 2 ? i / 4 : 0], i % 4, f); else Elem<DT>::put(q[0], i, f); }
  DEV void load(uint64_t p) {
#pragma unroll
    for (int k = 0; k < N; ++k) q[k] = Glob<POL>::ld16(p + 16 * k);
  }
  DEV void load(uint64_t p, uint64_t p2) {
    if (N == 2) { q[0] = Glob<POL>::ld16(p); q[N - 1] = Glob<POL>::ld16(p2); }
    else { const v2i a = Glob<POL>::ld8(p), b = Glob<POL>::ld8(p2); q[0] = v4i{a[0], a[1], b[0], b[1]}; }
  }
  // lines: see MF_LINES
  DEV void store(uint64_t p, bool lines) const {
#pragma unroll
    for (int k = 0; k < N; ++k) Glob<POL>::st16(p + 16 * k, q[k], N == 1 && lines);
  }
  DEV void store(uint64_t p, uint64_t p2, bool lines) const {
    if (N == 2) { Glob<POL>::st16(p, q[0], lines); Glob<POL>::st16(p2, q[N - 1], lines); }
    else { Glob<POL>::st8(p, v2i{q[0][0], q[0][1]}, lines); Glob<POL>::st8(p2, v2i{q[0][2], q[0][3]}, lines); }
  }
};

// Rows of [B, S, H, D] come in items: a token and the heads [h, h + block) of it, by the item's number, blocks of heads running fastest.
// What belongs to the token (its position, slot, page, the divisions here) is then found once for a block.
struct Place { uint32_t b, s, h; };
template <class ARGS> DEV Place place(const ARGS& a, uint32_t item) {
  Place p;
  const uint32_t token = divided(item, a.by_blocks);
  p.h = (item - token * a.blocks) * a.block;
  p.b = divided(token, a.by_seq);
  p.s = token - p.b * a.seq;
  return p;
}
DEV uint64_t offset(const Place& p, const uint32_t (&st)[4]) { return (uint64_t)p.b * st[0] + (uint64_t)p.s * st[1] + (uint64_t)p.h * st[2]; }

// ---------------------------------------------------------------------------
// NORM_ROPE, NORM_ROPE_GRAD
//
// z = Rot(y), y = x r gamma, r = 1 / sqrt(mean(x^2) + eps);  backwards dy = Rot^T(dz), u = dy gamma,
//   dx = r (u - x r^2 mean(u x)),   dgamma = sum over rows of dy x r.
// Bound by memory: one read and one write of the rows (two reads backwards), some ten instructions an element.  A part of a wavefront
// holds a row in registers; what a lane holds are both halves of its pairs, so that a rotation needs no other lane, and of the sums
// only the row's go over lanes.  A lane has the same elements of every row, so gamma stays in its registers.
// As kernels, 128 bf16 a head, where a large copy moves 4.76 TB/s: 172 MB forwards 36.3 us (4.7 TB/s), 205 MB backwards 43.5 (4.7; the sums
// of gamma's shares another 4); 24 heads of one token 4.8.  As tasks of the ring 69, 96 and 14 us from submission to completion: there a
// workgroup waits for its loads before it makes the next pass, and three of them share a compute unit.
// ---------------------------------------------------------------------------
struct RopeArgs {
  uint64_t x, gamma, table, positions, out, dout, partial;
  uint32_t xs[4], os[4], zs[4], gs, ts, ps[2], cs, half, places, seq, heads, block, blocks, d, chunks, items, dtype[4];
  Div by_seq, by_blocks;
  bool pairs, lines;
  float eps;
};
template <class P> DEV RopeArgs rope_args(P p) {
  RopeArgs a;
  a.x = uni64(p->x); a.gamma = uni64(p->gamma); a.table = uni64(p->table); a.positions = uni64(p->positions); a.out = uni64(p->out); a.dout = uni64(p->dout);
  a.partial = uni64(p->partial);
#pragma unroll
  for (int k = 0; k < 4; ++k) { a.xs[k] = uni(p->xs[k]); a.os[k] = uni(p->os[k]); a.zs[k] = uni(p->zs[k]); a.dtype[k] = uni((uint32_t)p->h.dtype[k]); }
  a.gs = uni(p->gs); a.ts = uni(p->ts); a.ps[0] = uni(p->ps[0]); a.ps[1] = uni(p->ps[1]); a.cs = uni(p->cs);
  a.half = uni(p->half); a.places = uni(p->places); a.seq = uni(p->seq); a.heads = uni(p->heads);
  a.block = uni((uint32_t)p->h.block); a.blocks = uni(p->blocks);
  a.d = uni(p->h.d); a.chunks = uni(p->h.nchunks); a.items = uni(p->h.items);
  a.by_seq = uni_div(p->by_seq.mul, p->by_seq.shift); a.by_blocks = uni_div(p->by_blocks.mul, p->by_blocks.shift);
  a.pairs = (uni((uint32_t)p->h.flags) & MF_PAIRS) != 0;
  a.lines = (uni((uint32_t)p->h.flags) & MF_LINES) != 0;
  a.eps = __builtin_bit_cast(float, uni(__builtin_bit_cast(uint32_t, (float)p->h.alpha)));
  return a;
}
// the token's row of the table, or false: it has none
template <int POL> DEV bool table_row(const RopeArgs& a, const Place& p, uint64_t& row) {
  const uint32_t at = a.positions != 0 ? (uint32_t)Glob<POL>::ldi(a.positions + ((uint64_t)p.b * a.ps[0] + (uint64_t)p.s * a.ps[1]) * 4u) : p.s;
  const bool has = at < a.places;
  row = a.table + (uint64_t)(has ? at : 0u) * a.ts * 4u;
  return has;
}

// The columns of the partial sums: what the lanes have summed for their elements goes by way of LDS, in the order of the groups of lanes.
template <int POL> DEV void gamma_part(const RopeArgs& a, uint32_t chunk, uint32_t groups, const float* s, uint32_t tid) {
  __syncthreads();
  for (uint32_t j = tid; j < a.d; j += kThreads) {
    float sum = 0.0f;
    for (uint32_t g = 0; g < groups; ++g) sum += s[g * a.d + j];
    Glob<POL>::stf(a.partial + ((uint64_t)j * a.cs + chunk) * 4u, sum);
  }
}

template <int POL, int DT, bool PAIRS, bool GRAD>
DEV void rope_vectors(const RopeArgs& a, uint32_t chunk, float* s, uint32_t tid) {
  typedef Glob<POL> M;
  typedef Eight<POL, DT> E;
  constexpr uint32_t ES = Elem<DT>::ES;
  constexpr int U = GRAD ? kGradBlock : kRopeBlock;
  // A lane's eight elements are two windows of four, oa and ob on.  Halves: the same four of either half, or eight that follow
  // each other behind them; neighbours: eight that follow each other.  The last window of a part that is no whole number of them begins
  // early and ends with it: what it shares with the one before (below `from`) both compute and store, and only that one sums.
  const uint32_t units = rope_units(a.d, a.half, PAIRS), lg = ceil_log2(units), lanes = 1u << lg;
  const uint32_t u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const bool active = u < units;
  const uint32_t turned_units = PAIRS ? 0u : (a.half + 3u) / 4u, rest = PAIRS ? 8u * u : 2u * a.half + 8u * (u - turned_units);
  const bool turned = u < turned_units;
  uint32_t from_a = turned ? 4u * u : rest, from_b = turned ? a.half + 4u * u : rest + 4u, oa, ob;
  if (turned) { oa = from_a < a.half - 4u ? from_a : a.half - 4u; ob = oa + a.half; }
  else if (PAIRS) { oa = from_a < a.d - 8u ? from_a : a.d - 8u; ob = oa + 4u; from_b = from_a; }
  else { oa = from_a < a.d - 4u ? from_a : a.d - 4u; ob = from_b < a.d - 4u ? from_b : a.d - 4u; }
  bool va[4], vb[4], turns[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    turns[i] = PAIRS ? oa / 2u + i < a.half : turned;
    va[i] = (PAIRS ? oa + 2u * i : oa + i) >= from_a;
    vb[i] = (PAIRS ? oa + 2u * i + 1u : ob + i) >= from_b;
  }
  float ga[4], gb[4], da[4], db[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t ja = PAIRS ? oa + 2u * i : oa + i, jb = PAIRS ? oa + 2u * i + 1u : ob + i;
    ga[i] = gb[i] = 1.0f;
    da[i] = db[i] = 0.0f;
    if (a.gamma != 0 && active) {
      const uint32_t gdt = a.dtype[2];
      ga[i] = M::ld_rt(a.gamma + (uint64_t)ja * a.gs * float_size(gdt), gdt);
      gb[i] = M::ld_rt(a.gamma + (uint64_t)jb * a.gs * float_size(gdt), gdt);
    }
  }
  const float inv_d = 1.0f / (float)a.d;
  for (uint32_t base = chunk * step; base < a.items; base += a.chunks * step) {
    const uint32_t item = base + group;
    const Place p = place(a, item < a.items ? item : a.items - 1u);
    const uint32_t heads = item < a.items && active ? (a.heads - p.h < (uint32_t)U ? a.heads - p.h : (uint32_t)U) : 0u;
    const uint64_t xp = a.x + offset(p, a.xs) * ES, zp = a.dout + offset(p, a.zs) * ES, op = a.out + offset(p, a.os) * ES;
    E x[U], z[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      x[k].clear();
      if (GRAD) z[k].clear();
      if ((uint32_t)k < heads) {
        const uint64_t at = xp + (uint64_t)k * a.xs[2] * ES, zat = zp + (uint64_t)k * a.zs[2] * ES;
        if (PAIRS) x[k].load(at + oa * ES);
        else x[k].load(at + oa * ES, at + ob * ES);
        if (GRAD && PAIRS) z[k].load(zat + oa * ES);
        if (GRAD && !PAIRS) z[k].load(zat + oa * ES, zat + ob * ES);
      }
    }
    float c[4] = {1.0f, 1.0f, 1.0f, 1.0f}, sn[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    bool has = true;
    if (a.half != 0) {
      uint64_t row_p;
      has = table_row<POL>(a, p, row_p);
      const uint32_t pair = PAIRS ? oa / 2u : oa;                // of the window's first elements
      if (PAIRS ? pair + 4u <= a.half : turned) {
        M::template ld4e<GPUOS_F32>(row_p + pair * 4u, c);
        M::template ld4e<GPUOS_F32>(row_p + (a.half + pair) * 4u, sn);
      } else if (PAIRS && pair < a.half) {                       // (the rotated part ends inside)
#pragma unroll
        for (uint32_t i = 0; i < 3; ++i) {
          if (pair + i < a.half) { c[i] = M::ldf(row_p + (pair + i) * 4u); sn[i] = M::ldf(row_p + (a.half + pair + i) * 4u); }
        }
      }
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (__builtin_amdgcn_ballot_w64((uint32_t)k < heads) == 0) continue;       // (the same in every lane: the sums need them all)
      float xa[4], xb[4], ss = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        xa[i] = x[k].get(PAIRS ? 2 * i : i);
        xb[i] = x[k].get(PAIRS ? 2 * i + 1 : 4 + i);
        const float oxa = va[i] ? xa[i] : 0.0f, oxb = vb[i] ? xb[i] : 0.0f;
        ss = __builtin_fmaf(oxa, oxa, ss);
        ss = __builtin_fmaf(oxb, oxb, ss);
      }
      ss = wave_reduce<GPUOS_IMPL_SUM_LAST>(ss, lanes);
      float r = rsqrtf(__builtin_fmaf(ss, inv_d, a.eps));
      if (!has) r = __builtin_nanf("");
      E o;
      if (!GRAD) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float ya = xa[i] * r * ga[i], yb = xb[i] * r * gb[i];
          o.put(PAIRS ? 2 * i : i, turns[i] ? __builtin_fmaf(ya, c[i], -(yb * sn[i])) : ya);          // (not by an angle of 0: the other may be no number)
          o.put(PAIRS ? 2 * i + 1 : 4 + i, turns[i] ? __builtin_fmaf(yb, c[i], ya * sn[i]) : yb);
        }
      } else {
        float ua[4], ub[4], t = 0.0f;
        const float rk = (uint32_t)k < heads ? r : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float za = z[k].get(PAIRS ? 2 * i : i), zb = z[k].get(PAIRS ? 2 * i + 1 : 4 + i);
          const float ya = turns[i] ? __builtin_fmaf(za, c[i], zb * sn[i]) : za, yb = turns[i] ? __builtin_fmaf(zb, c[i], -(za * sn[i])) : zb;
          da[i] = __builtin_fmaf(ya, xa[i] * rk, da[i]);         // (rows that are not there: 0 * 0)
          db[i] = __builtin_fmaf(yb, xb[i] * rk, db[i]);
          ua[i] = ya * ga[i];
          ub[i] = yb * gb[i];
          t += va[i] ? ua[i] * xa[i] : 0.0f;
          t += vb[i] ? ub[i] * xb[i] : 0.0f;
        }
        t = wave_reduce<GPUOS_IMPL_SUM_LAST>(t, lanes);
        const float m = (t * inv_d) * r * r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          o.put(PAIRS ? 2 * i : i, r * __builtin_fmaf(-xa[i], m, ua[i]));
          o.put(PAIRS ? 2 * i + 1 : 4 + i, r * __builtin_fmaf(-xb[i], m, ub[i]));
        }
      }
      if ((uint32_t)k < heads) {
        const uint64_t to = op + (uint64_t)k * a.os[2] * ES;
        if (PAIRS) o.store(to + oa * ES, a.lines);
        else o.store(to + oa * ES, to + ob * ES, a.lines);
      }
    }
  }
  if (GRAD && a.partial != 0) {
    if (active) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t ja = PAIRS ? oa + 2u * i : oa + i, jb = PAIRS ? oa + 2u * i + 1u : ob + i;
        if (va[i]) s[group * a.d + ja] = da[i];
        if (vb[i]) s[group * a.d + jb] = db[i];
      }
    }
    gamma_part<POL>(a, chunk, step, s, tid);
  }
}

// Rows of any length, strides and dtypes, element by element: a lane takes pairs (two elements in place of one behind the rotated
// ones, i and i + half of the rest), next to each other's in neighbouring lanes.
template <int POL, bool GRAD>
DEV void rope_elements(const RopeArgs& a, uint32_t chunk, float* s, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr int K = 4;                                // 256 pairs of 512 elements over 64 lanes
  const uint32_t rest = a.d - 2u * a.half, rest_pairs = (rest + 1u) / 2u, pairs = a.half + rest_pairs;
  const uint32_t lg = pairs > 64u ? 6u : ceil_log2(pairs), lanes = 1u << lg;
  const uint32_t u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t end = a.items == ModelPack::kNoRows ? 0u : a.items;
  const uint32_t es = float_size(a.dtype[0]), eo = float_size(a.dtype[1]), ez = float_size(a.dtype[3]);
  uint32_t ja[K], jb[K];
  bool in_a[K], in_b[K], turned[K];
  float ga[K], gb[K], da[K], db[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const uint32_t i = u + k * lanes;
    turned[k] = i < a.half;
    ja[k] = turned[k] ? (a.pairs ? 2u * i : i) : a.half + i;                        // (2 half + (i - half))
    jb[k] = turned[k] ? (a.pairs ? 2u * i + 1u : i + a.half) : a.half + i + rest_pairs;
    in_a[k] = i < pairs;
    in_b[k] = in_a[k] && jb[k] < a.d;
    ga[k] = gb[k] = 1.0f;
    da[k] = db[k] = 0.0f;
    const uint32_t gdt = a.dtype[2];
    if (a.gamma != 0 && in_a[k]) ga[k] = M::ld_rt(a.gamma + (uint64_t)ja[k] * a.gs * float_size(gdt), gdt);
    if (a.gamma != 0 && in_b[k]) gb[k] = M::ld_rt(a.gamma + (uint64_t)jb[k] * a.gs * float_size(gdt), gdt);
  }
  const float inv_d = 1.0f / (float)a.d;
  for (uint32_t base = chunk * step; base < end; base += a.chunks * step) {
    const bool in = base + group < end;
    const Place p = place(a, in ? base + group : end - 1u);
    const uint64_t xp = a.x + offset(p, a.xs) * es, op = a.out + offset(p, a.os) * eo, zp = a.dout + offset(p, a.zs) * ez;
    uint64_t row_p = 0;
    bool has = true;
    if (a.half != 0) has = table_row<POL>(a, p, row_p);
    float xa[K], xb[K], za[K], zb[K], c[K], sn[K], ss = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      xa[k] = xb[k] = za[k] = zb[k] = 0.0f;
      c[k] = 1.0f;
      sn[k] = 0.0f;
      if (k * lanes >= pairs) continue;
      if (in_a[k]) xa[k] = M::ld_rt(xp + (uint64_t)ja[k] * a.xs[3] * es, a.dtype[0]);
      if (in_b[k]) xb[k] = M::ld_rt(xp + (uint64_t)jb[k] * a.xs[3] * es, a.dtype[0]);
      if (GRAD && in_a[k]) za[k] = M::ld_rt(zp + (uint64_t)ja[k] * a.zs[3] * ez, a.dtype[3]);
      if (GRAD && in_b[k]) zb[k] = M::ld_rt(zp + (uint64_t)jb[k] * a.zs[3] * ez, a.dtype[3]);
      if (turned[k]) {
        const uint32_t i = u + k * lanes;
        c[k] = M::ldf(row_p + i * 4u);
        sn[k] = M::ldf(row_p + (a.half + i) * 4u);
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) { ss = __builtin_fmaf(xa[k], xa[k], ss); ss = __builtin_fmaf(xb[k], xb[k], ss); }
    ss = wave_reduce<GPUOS_IMPL_SUM_LAST>(ss, lanes);
    float r = rsqrtf(__builtin_fmaf(ss, inv_d, a.eps));
    if (!has) r = __builtin_nanf("");
    float oa[K], ob[K];
    if (!GRAD) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const float ya = xa[k] * r * ga[k], yb = xb[k] * r * gb[k];
        oa[k] = turned[k] ? __builtin_fmaf(ya, c[k], -(yb * sn[k])) : ya;
        ob[k] = turned[k] ? __builtin_fmaf(yb, c[k], ya * sn[k]) : yb;
      }
    } else {
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const float ya = turned[k] ? __builtin_fmaf(za[k], c[k], zb[k] * sn[k]) : za[k], yb = turned[k] ? __builtin_fmaf(zb[k], c[k], -(za[k] * sn[k])) : zb[k];
        da[k] += in ? ya * (xa[k] * r) : 0.0f;
        db[k] += in ? yb * (xb[k] * r) : 0.0f;
        oa[k] = ya * ga[k];
        ob[k] = yb * gb[k];
        t = __builtin_fmaf(oa[k], xa[k], t);
        t = __builtin_fmaf(ob[k], xb[k], t);
      }
      t = wave_reduce<GPUOS_IMPL_SUM_LAST>(t, lanes);
      const float m = (t * inv_d) * r * r;
#pragma unroll
      for (int k = 0; k < K; ++k) { oa[k] = r * __builtin_fmaf(-xa[k], m, oa[k]); ob[k] = r * __builtin_fmaf(-xb[k], m, ob[k]); }
    }
    // (The gradient's offsets in the output are made again for every row: kept in registers over the loop, like those of its inputs, it
    // takes 133, and so 117, which is room for a block beside a worker's three and for a fourth on every unit: 262,144 heads of 128 bf16 and
    // a gradient of strides of 0 312 and 202 us.)
    uint32_t os = a.os[3];
    if (GRAD) asm volatile("" : "+s"(os));
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && in_a[k]) M::st_rt(op + (uint64_t)ja[k] * os * eo, a.dtype[1], oa[k]);
      if (in && in_b[k]) M::st_rt(op + (uint64_t)jb[k] * os * eo, a.dtype[1], ob[k]);
    }
  }
  if (GRAD && a.partial != 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in_a[k]) s[group * a.d + ja[k]] = da[k];
      if (in_b[k]) s[group * a.d + jb[k]] = db[k];
    }
    gamma_part<POL>(a, chunk, step, s, tid);
  }
}

// GAMMA_SUM: the workgroup a row of the partial sums (of any length; 4 KB at most as NORM_ROPE_GRAD makes them), always in the same order.
template <int POL> DEV void gamma_sum(const RopeArgs& a, uint32_t chunk, float* s, uint32_t tid) {
  typedef Glob<POL> M;
  for (uint32_t row = chunk; row < a.items; row += a.chunks) {
    const uint64_t p = a.partial + (uint64_t)row * a.cs * 4u;
    float sum = 0.0f;
    for (uint32_t i = tid; i < a.d; i += 4u * kThreads) {
      float f[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) f[k] = i + k * kThreads < a.d ? M::ldf(p + (uint64_t)(i + k * kThreads) * 4u) : 0.0f;
      sum += (f[0] + f[1]) + (f[2] + f[3]);
    }
    sum = wave_reduce<GPUOS_IMPL_SUM_LAST>(sum, 64u);
    if (row != chunk) __syncthreads();
    if ((tid & 63u) == 0) s[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) M::st_rt(a.out + (uint64_t)row * a.os[0] * float_size(a.dtype[1]), a.dtype[1], (s[0] + s[1]) + (s[2] + s[3]));
  }
}

// ---------------------------------------------------------------------------
// CACHE_STORE, CACHE_LOAD
//
// Bound by memory, three bytes of it an element of 16 bits.  A part of a wavefront takes a row: eight elements a lane, one load of 16
// bytes on the wide side and one of 8 on the cache's; a group's largest magnitude goes over the lanes that hold it, as an integer
// (magnitudes order like their bits, infinities and NaNs above all).
// As kernels, 128 bf16 a head: 16,384 tokens of 8 heads of keys and values (98 MB) stored in 19.6 us (5.0 TB/s, a part of it from the
// memory-side cache), 32 sequences of 4,096 such tokens at most read back (537 MB written, 208 read) in 123 (6.0 TB/s), 64 tokens stored in 3.5; as
// tasks of the ring 49, 169 and 13 us.
// ---------------------------------------------------------------------------
struct CacheArgs {
  uint64_t x, cache, scales, slots, lengths;
  uint32_t xs[4], cs[3], ss[4], ps[2], ls, pages, page, group, heads, seq, block, blocks, d, chunks, items, dtype, format;
  Div by_blocks, by_seq, by_page, by_group;
  bool lines;
};
template <class P> DEV CacheArgs cache_args(P p) {
  CacheArgs a;
  a.x = uni64(p->x); a.cache = uni64(p->cache); a.scales = uni64(p->scales); a.slots = uni64(p->slots); a.lengths = uni64(p->lengths);
#pragma unroll
  for (int k = 0; k < 4; ++k) { a.xs[k] = uni(p->xs[k]); a.ss[k] = uni(p->ss[k]); }
#pragma unroll
  for (int k = 0; k < 3; ++k) a.cs[k] = uni(p->cs[k]);
  a.ps[0] = uni(p->ps[0]); a.ps[1] = uni(p->ps[1]); a.ls = uni(p->ls);
  a.pages = uni(p->pages); a.page = uni(p->page); a.group = uni(p->group); a.heads = uni(p->heads); a.seq = uni(p->seq);
  a.block = uni((uint32_t)p->h.block); a.blocks = uni(p->blocks);
  a.d = uni(p->h.d); a.chunks = uni(p->h.nchunks); a.items = uni(p->h.items);
  a.dtype = uni((uint32_t)p->h.dtype[0]); a.format = uni((uint32_t)p->h.dtype[1]);
  a.lines = (uni((uint32_t)p->h.flags) & MF_LINES) != 0;
  a.by_blocks = uni_div(p->by_blocks.mul, p->by_blocks.shift); a.by_seq = uni_div(p->by_seq.mul, p->by_seq.shift); a.by_page = uni_div(p->by_page.mul, p->by_page.shift); a.by_group = uni_div(p->by_group.mul, p->by_group.shift);
  return a;
}
struct Quant { float inv, scale; bool bad; };
DEV Quant quant(uint32_t top_bits, uint32_t format) {
  const float qmax = format == GPUOS_I8 ? 127.0f : 448.0f;
  const float m = __builtin_fmaxf(__builtin_bit_cast(float, top_bits), 0x1p-100f);
  const bool bad = top_bits >= 0x7f800000u;
  return Quant{qmax / m, bad ? __builtin_nanf("") : m / qmax, bad};
}
DEV uint32_t magnitude(float f) { return __builtin_bit_cast(uint32_t, f) & 0x7fffffffu; }
// four values in 8 bits each (|y| <= qmax (1 + 2^-23): rounding to nearest stays in the format)
DEV uint32_t pack_q(const float* y, uint32_t format) {
  if (format == GPUOS_I8) {
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) w |= ((uint32_t)(int32_t)__builtin_rintf(y[k]) & 0xffu) << (8 * k);
    return w;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}
DEV void unpack_q(uint32_t w, uint32_t format, float* y) {
  if (format == GPUOS_I8) {
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = (float)((int32_t)(w << (24 - 8 * k)) >> 24);
  } else {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    y[0] = lo[0]; y[1] = lo[1]; y[2] = hi[0]; y[3] = hi[1];
  }
}
// where a slot's row of a head lies
DEV uint64_t cache_at(const CacheArgs& a, uint32_t page, uint32_t in, uint32_t h) {
  return a.cache + (uint64_t)page * a.cs[0] + (uint64_t)in * a.cs[1] + (uint64_t)h * a.cs[2];
}
DEV uint64_t scale_at(const CacheArgs& a, uint32_t page, uint32_t in, uint32_t h, uint32_t g) {
  return a.scales + ((uint64_t)page * a.ss[0] + (uint64_t)in * a.ss[1] + (uint64_t)h * a.ss[2] + (uint64_t)g * a.ss[3]) * 4u;
}

template <int POL, int DT> DEV void store_vectors(const CacheArgs& a, uint32_t chunk, uint32_t tid) {
  typedef Glob<POL> M;
  typedef Eight<POL, DT> E;
  constexpr int U = POL == POL_COHERENT ? kRingStoreBlock : kStoreBlock;
  const uint32_t units = (a.d + 7u) / 8u, lg = ceil_log2(units), lanes = 1u << lg;
  const uint32_t u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t at = 8u * u < a.d - 8u ? 8u * u : a.d - 8u;      // (the last window ends with the row: what two have both write alike)
  const uint32_t lg_width = a.group == a.d ? lg : ceil_log2(a.group) - 3u, width = 1u << lg_width;
  for (uint32_t base = chunk * step; base < a.items; base += a.chunks * step) {
    const uint32_t item = base + group;
    const Place p = place(a, item < a.items ? item : a.items - 1u);
    const uint32_t heads = item < a.items && u < units ? (a.heads - p.h < (uint32_t)U ? a.heads - p.h : (uint32_t)U) : 0u;
    const uint64_t xp = a.x + (offset(p, a.xs) + at) * Elem<DT>::ES;
    const uint32_t slot = (uint32_t)M::ldi(a.slots + ((uint64_t)p.b * a.ps[0] + (uint64_t)p.s * a.ps[1]) * 4u);
    E x[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      x[k].clear();
      if ((uint32_t)k < heads) x[k].load(xp + (uint64_t)k * a.xs[2] * Elem<DT>::ES);
    }
    const bool has = slot < a.pages * a.page;
    const uint32_t page = divided(has ? slot : 0u, a.by_page), in = slot - page * a.page;
    const uint64_t to = cache_at(a, page, in, p.h) + at, scale_to = scale_at(a, page, in, p.h, u >> lg_width);
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if (__builtin_amdgcn_ballot_w64((uint32_t)k < heads) == 0) continue;       // (the same in every lane: the maxima need them all)
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) { const uint32_t m = magnitude(x[k].get(i)); top = m > top ? m : top; }
      top = (uint32_t)wave_reduce<GPUOS_IMPL_MAX_LAST>((int32_t)top, width);
      const Quant q = quant(top, a.format);
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = q.bad ? 0.0f : x[k].get(i) * q.inv;
      const v2i w = {(int)pack_q(y, a.format), (int)pack_q(y + 4, a.format)};
      if (has && (uint32_t)k < heads) {
        M::st8b(to + (uint64_t)k * a.cs[2], w);
        if ((u & (width - 1u)) == 0) M::stf(scale_to + (uint64_t)k * a.ss[2] * 4u, q.scale);
      }
    }
  }
}
// rows of any length, strides and alignment: element by element, neighbouring lanes neighbouring elements
template <int POL> DEV void store_elements(const CacheArgs& a, uint32_t chunk, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr int K = 8;
  const uint32_t lg = a.d > 64u ? 6u : ceil_log2(a.d), lanes = 1u << lg, u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t es = float_size(a.dtype);
  // A group is the row, or a power of two: then `width` lanes of a register hold it, or `span` registers of all lanes.
  const bool whole = a.group == a.d;
  const uint32_t width = whole || a.group >= lanes ? lanes : a.group, span = whole ? (uint32_t)K : (a.group > lanes ? a.group >> lg : 1u);
  for (uint32_t base = chunk * step; base < a.items; base += a.chunks * step) {
    const bool in_row = base + group < a.items;
    const Place p = place(a, in_row ? base + group : a.items - 1u);
    int32_t slot = M::ldi(a.slots + ((uint64_t)p.b * a.ps[0] + (uint64_t)p.s * a.ps[1]) * 4u);
    if (!in_row || (uint32_t)slot >= a.pages * a.page) slot = -1;
    const uint64_t xp = a.x + offset(p, a.xs) * es;
    float x[K];
    int32_t top[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t j = u + k * lanes;
      x[k] = j < a.d ? M::ld_rt(xp + (uint64_t)j * a.xs[3] * es, a.dtype) : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < K; ++k) top[k] = (int32_t)magnitude(x[k]);
#pragma unroll
    for (int o = 1; o < K; o *= 2) {
      if ((uint32_t)o < span) {
        int32_t t[K];
#pragma unroll
        for (int k = 0; k < K; ++k) t[k] = top[k ^ o] > top[k] ? top[k ^ o] : top[k];
#pragma unroll
        for (int k = 0; k < K; ++k) top[k] = t[k];
      }
    }
    const uint32_t page = slot >= 0 ? divided((uint32_t)slot, a.by_page) : 0u, in = (uint32_t)slot - page * a.page;
    const uint64_t to = cache_at(a, page, in, p.h);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t j = u + k * lanes;
      const Quant q = quant((uint32_t)wave_reduce<GPUOS_IMPL_MAX_LAST>(top[k], width), a.format);
      const float y[4] = {q.bad ? 0.0f : x[k] * q.inv, 0.0f, 0.0f, 0.0f};
      const uint32_t w = pack_q(y, a.format);
      if (slot >= 0 && j < a.d) {
        M::template put<uint8_t>(to + j, (uint8_t)w);
        const uint32_t g = divided(j, a.by_group);
        if (j == g * a.group) M::stf(scale_at(a, page, in, p.h, g), q.scale);
      }
    }
  }
}

// where row l of sequence b lies: 0 in the cache, 1 behind the sequence, 2 in a page that there is not
template <int POL> DEV uint32_t sequence_row(const CacheArgs& a, const Place& p, uint32_t& page, uint32_t& in) {
  const int32_t length = a.lengths != 0 ? Glob<POL>::ldi(a.lengths + (uint64_t)p.b * a.ls * 4u) : (int32_t)a.seq;
  const uint32_t nth = divided(p.s, a.by_page);
  in = p.s - nth * a.page;
  page = 0;
  if ((int32_t)p.s >= length) return 1u;
  page = (uint32_t)Glob<POL>::ldi(a.slots + ((uint64_t)p.b * a.ps[0] + (uint64_t)nth * a.ps[1]) * 4u);
  return page < a.pages ? 0u : 2u;
}
template <int POL, int DT> DEV void load_vectors(const CacheArgs& a, uint32_t chunk, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr int U = POL == POL_COHERENT ? kRingLoadBlock : kLoadBlock;
  const uint32_t units = (a.d + 7u) / 8u, lg = ceil_log2(units), lanes = 1u << lg;
  const uint32_t u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t at = 8u * u < a.d - 8u ? 8u * u : a.d - 8u;
  const uint32_t lg_width = a.group == a.d ? lg : ceil_log2(a.group) - 3u;
  if (u >= units) return;
  for (uint32_t item = chunk * step + group; item < a.items; item += a.chunks * step) {
    const Place p = place(a, item);
    const uint32_t heads = a.heads - p.h < (uint32_t)U ? a.heads - p.h : (uint32_t)U;
    const uint64_t to = a.x + (offset(p, a.xs) + at) * Elem<DT>::ES;
    uint32_t page, in;
    const uint32_t what = sequence_row<POL>(a, p, page, in);
    const uint64_t from = cache_at(a, page, in, p.h) + at, scale_from = scale_at(a, page, in, p.h, u >> lg_width);
    v2i w[U];
    float scale[U];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      w[k] = v2i{0, 0};
      scale[k] = what == 1u ? 0.0f : __builtin_nanf("");
      if (what == 0u && (uint32_t)k < heads) {
        w[k] = M::ld8b(from + (uint64_t)k * a.cs[2]);
        scale[k] = M::ldf(scale_from + (uint64_t)k * a.ss[2] * 4u);
      }
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      if ((uint32_t)k < heads) {
        float y[8];
        unpack_q((uint32_t)w[k][0], a.format, y);
        unpack_q((uint32_t)w[k][1], a.format, y + 4);
        Eight<POL, DT> o;
        o.clear();
#pragma unroll
        for (int i = 0; i < 8; ++i) o.put(i, y[i] * scale[k]);
        o.store(to + (uint64_t)k * a.xs[2] * Elem<DT>::ES, a.lines);
      }
    }
  }
}
template <int POL> DEV void load_elements(const CacheArgs& a, uint32_t chunk, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr int K = 8;
  const uint32_t lg = a.d > 64u ? 6u : ceil_log2(a.d), lanes = 1u << lg, u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t es = float_size(a.dtype);
  for (uint32_t row = chunk * step + group; row < a.items; row += a.chunks * step) {
    const Place p = place(a, row);
    uint32_t page, in;
    const uint32_t what = sequence_row<POL>(a, p, page, in);
    const uint64_t from = cache_at(a, page, in, p.h), to = a.x + offset(p, a.xs) * es;
    uint32_t w[K];
    float scale[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t j = u + k * lanes;
      w[k] = 0;
      scale[k] = what == 1u ? 0.0f : __builtin_nanf("");
      if (what == 0u && j < a.d) {
        w[k] = M::template at<uint8_t>(from + j);
        scale[k] = M::ldf(scale_at(a, page, in, p.h, divided(j, a.by_group)));
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t j = u + k * lanes;
      float y[4];
      unpack_q(w[k], a.format, y);
      if (j < a.d) M::st_rt(to + (uint64_t)j * a.xs[3] * es, a.dtype, y[0] * scale[k]);
    }
  }
}

// ---------------------------------------------------------------------------
// LOGIT_PENALTY
//
// Bound by memory (one read and one write of the logits) while the history is short.  The workgroup takes a row in segments: the
// tokens of the row's history that fall into the segment are counted in LDS (additions of integers: their order does not matter), then
// the segment is changed and written.  Every segment reads the row's history, from the cache after the first: for long ones that is
// what bounds it.  64 rows of 100,352 bf16 with 2,048 tokens, bias and bits 10.2 us as a kernel (27 MB, 5.8 us at a copy's rate, and
// the 4 that the way from the record over the history to the counts takes), 8 of 65,537 with 32,768 tokens 8.4, one of 32,003 with 200 4.1; as tasks of the ring 46, 37 and 12.
// A count has 31 bits; the top bit says that the token is in the prompt.
// ---------------------------------------------------------------------------
struct PenaltyArgs {
  uint64_t x, out, history, prompts, params, bias, allowed;
  uint32_t xs[2], os[2], hs[2], ps, ms[2], bs[2], as[2], n, seg, segs, v, chunks, items, dtype[3];
  Div by_segs;
  bool lines;
};
template <class P> DEV PenaltyArgs penalty_args(P p) {
  PenaltyArgs a;
  a.x = uni64(p->x); a.out = uni64(p->out); a.history = uni64(p->history); a.prompts = uni64(p->prompts); a.params = uni64(p->params);
  a.bias = uni64(p->bias); a.allowed = uni64(p->allowed);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    a.xs[k] = uni(p->xs[k]); a.os[k] = uni(p->os[k]); a.hs[k] = uni(p->hs[k]); a.ms[k] = uni(p->ms[k]); a.bs[k] = uni(p->bs[k]); a.as[k] = uni(p->as[k]);
  }
  a.ps = uni(p->ps); a.n = uni(p->n); a.seg = uni(p->seg); a.segs = uni(p->segs); a.v = uni(p->h.d); a.chunks = uni(p->h.nchunks); a.items = uni(p->h.items);
#pragma unroll
  for (int k = 0; k < 3; ++k) a.dtype[k] = uni((uint32_t)p->h.dtype[k]);
  a.by_segs = uni_div(p->by_segs.mul, p->by_segs.shift);
  a.lines = (uni((uint32_t)p->h.flags) & MF_LINES) != 0;
  return a;
}
struct Penalty { float rep, freq, pres; };
DEV float penalize(float v, uint32_t seen, const Penalty& p) {
  if (seen != 0) {
    v = v > 0.0f ? v / p.rep : v * p.rep;
    const uint32_t count = seen & 0x7fffffffu;
    v = v - (float)count * p.freq - (count > 0 ? p.pres : 0.0f);
  }
  return v;
}
// The history goes by K loads of 16 bytes a lane, the next ones on their way while these are counted (and the first while the counts are
// cleared).
template <int POL, uint32_t T> DEV void count_tokens(const PenaltyArgs& a, uint32_t row, uint32_t v0, uint32_t nv, uint32_t* seen, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr uint32_t K = 2, kRound = K * T * 4u;
  const uint64_t h = a.history + (uint64_t)row * a.hs[0] * 4u;
  const int32_t prompt = a.prompts != 0 ? M::ldi(a.prompts + (uint64_t)row * a.ps * 4u) : 0;
  const uint32_t whole = POL == POL_PLAIN && a.hs[1] == 1u ? a.n & ~3u : 0u;      // what goes by fours
  auto ask = [&](v4i (&q)[K], uint32_t i) {
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
      q[k] = v4i{-1, -1, -1, -1};
      if (i + (k * T + tid) * 4u < whole) q[k] = M::ld16(h + ((uint64_t)i + (k * T + tid) * 4u) * 4u);
    }
  };
  auto take = [&](int32_t id, uint32_t i) {
    const uint32_t j = (uint32_t)id - v0;              // (an id below v0, negative ones too, is over nv so)
    if (j < nv) {
      if ((int32_t)i < prompt) __hip_atomic_fetch_or(&seen[j], 0x80000000u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      else __hip_atomic_fetch_add(&seen[j], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
  };
  v4i q[K], next[K];
  ask(q, 0);
  for (uint32_t j = tid; j < (nv + 3u) / 4u; j += T) ((v4i*)seen)[j] = v4i{0, 0, 0, 0};
  __syncthreads();
  for (uint32_t i = 0; i < whole; i += kRound) {
    ask(next, i + kRound);
#pragma unroll
    for (uint32_t k = 0; k < K; ++k) {
#pragma unroll
      for (uint32_t e = 0; e < 4; ++e) take(q[k][e], i + (k * T + tid) * 4u + e);
      q[k] = next[k];
    }
  }
  for (uint32_t i = whole + tid; i < a.n; i += 4u * T) {
    int32_t id[4];
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) id[k] = i + k * T < a.n ? M::ldi(h + (uint64_t)(i + k * T) * a.hs[1] * 4u) : -1;
#pragma unroll
    for (uint32_t k = 0; k < 4; ++k) take(id[k], i + k * T);
  }
  __syncthreads();
}
// one element of any operand, as it is to be written
template <int POL> DEV float penalized(const PenaltyArgs& a, uint32_t row, uint32_t v, uint32_t seen, const Penalty& pen) {
  typedef Glob<POL> M;
  float y = M::ld_rt(a.x + ((uint64_t)row * a.xs[0] + (uint64_t)v * a.xs[1]) * float_size(a.dtype[0]), a.dtype[0]);
  y = penalize(y, seen, pen);
  if (a.bias != 0) y += M::ld_rt(a.bias + ((uint64_t)row * a.bs[0] + (uint64_t)v * a.bs[1]) * float_size(a.dtype[2]), a.dtype[2]);
  if (a.allowed != 0 && ((M::template at<uint32_t>(a.allowed + ((uint64_t)row * a.as[0] + (uint64_t)(v >> 5) * a.as[1]) * 4u) >> (v & 31u)) & 1u) == 0)
    y = -__builtin_inff();
  return y;
}
template <int POL> DEV void put_logit(const PenaltyArgs& a, uint32_t row, uint32_t v, float y) {
  Glob<POL>::st_rt(a.out + ((uint64_t)row * a.os[0] + (uint64_t)v * a.os[1]) * float_size(a.dtype[1]), a.dtype[1], y);
}
// T threads; DT < 0: element by element
template <int POL, int DT, uint32_t T> DEV void penalty_segments(const PenaltyArgs& a, uint32_t chunk, float* s, uint32_t tid) {
  typedef Glob<POL> M;
  uint32_t* seen = (uint32_t*)s;
  for (uint32_t item = chunk; item < a.items; item += a.chunks) {
    const uint32_t row = divided(item, a.by_segs), v0 = (item - row * a.segs) * a.seg, nv = a.v - v0 < a.seg ? a.v - v0 : a.seg;
    if (a.history != 0 && item != chunk) __syncthreads();        // (the counts of the segment before have been read)
    Penalty pen = {1.0f, 0.0f, 0.0f};
    if (a.history != 0) {
      const uint64_t p = a.params + (uint64_t)row * a.ms[0] * 4u;
      pen = {M::ldf(p), M::ldf(p + (uint64_t)a.ms[1] * 4u), M::ldf(p + (uint64_t)a.ms[1] * 8u)};
    }
    if constexpr (DT < 0) {
      if (a.history != 0) count_tokens<POL, T>(a, row, v0, nv, seen, tid);
      for (uint32_t j = tid; j < nv; j += T) put_logit<POL>(a, row, v0 + j, penalized<POL>(a, row, v0 + j, a.history != 0 ? seen[j] : 0u, pen));
    } else {
      // The segment's elements and bits are asked for before its tokens are counted, eight to a lane.
      constexpr uint32_t ES = Elem<DT>::ES, U = ModelPack::kSegment / (8u * T);
      const uint64_t xp = a.x + ((uint64_t)row * a.xs[0] + v0) * ES, op = a.out + ((uint64_t)row * a.os[0] + v0) * ES;
      const uint64_t bp = a.bias + ((uint64_t)row * a.bs[0] + v0) * float_size(a.dtype[2]), ap = a.allowed + (uint64_t)row * a.as[0] * 4u;
      const uint32_t whole = nv & ~7u;
      Eight<POL, DT> x[U];
      uint32_t bits[U];
#pragma unroll
      for (uint32_t k = 0; k < U; ++k) {
        const uint32_t j = (k * T + tid) * 8u;
        x[k].clear();
        bits[k] = 0xffu;
        if (j < whole) {
          x[k].load(xp + j * ES);
          if (a.allowed != 0) bits[k] = M::template at<uint32_t>(ap + ((v0 + j) >> 5) * 4u) >> ((v0 + j) & 31u);
        }
      }
      if (a.history != 0) count_tokens<POL, T>(a, row, v0, nv, seen, tid);
#pragma unroll
      for (uint32_t k = 0; k < U; ++k) {
        const uint32_t j = (k * T + tid) * 8u;
        if (j >= whole) continue;
        float b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) b[i] = 0.0f;
        if (a.bias != 0) {
          if (POL == POL_COHERENT) {                   // (its vectors need an alignment that nothing gives the bias)
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = M::ld_rt(bp + (j + i) * float_size(a.dtype[2]), a.dtype[2]);
          } else if (a.dtype[2] == GPUOS_F32) M::template ld8e<GPUOS_F32>(bp + j * 4u, b);
          else if (a.dtype[2] == GPUOS_F16) M::template ld8e<GPUOS_F16>(bp + j * 2u, b);
          else M::template ld8e<GPUOS_BF16>(bp + j * 2u, b);
        }
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = x[k].get(i);
        if (a.history != 0) {
          // The penalty costs a division, and few tokens of a segment are in the history: each lane goes through its own, one a step.
          const v4i lo = *(const v4i*)(seen + j), hi = *(const v4i*)(seen + j + 4);
          uint32_t left = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) left |= (lo[i] != 0 ? 1u << i : 0u) | (hi[i] != 0 ? 16u << i : 0u);
          while (left != 0) {
            const uint32_t at = (uint32_t)__builtin_ctz(left);
            float v = y[0];
#pragma unroll
            for (uint32_t i = 1; i < 8; ++i) v = at == i ? y[i] : v;
            v = penalize(v, seen[j + at], pen);
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) y[i] = at == i ? v : y[i];
            left &= left - 1u;
          }
        }
        Eight<POL, DT> o;
        o.clear();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (a.bias != 0) y[i] += b[i];
          o.put(i, (bits[k] >> i) & 1u ? y[i] : -__builtin_inff());
        }
        o.store(op + j * ES, a.lines);
      }
      if (tid < nv - whole) put_logit<POL>(a, row, v0 + whole + tid, penalized<POL>(a, row, v0 + whole + tid, a.history != 0 ? seen[whole + tid] : 0u, pen));
    }
  }
}
constexpr uint32_t kPenaltyThreads = 512;              // of a kernel's workgroup
static_assert(ModelPack::kSegment <= kScratchFloats && ModelPack::kSegment % (8 * kPenaltyThreads) == 0, "a segment's counts fit the worker's scratch; its vectors are shared out evenly");

// ---------------------------------------------------------------------------
// the executor of a variant; and the worker's, functions of their own like its others
// ---------------------------------------------------------------------------
template <int POL, uint32_t V, uint32_t T, class P> DEV void run_model(P r, uint32_t chunk, float* s, uint32_t tid) {
  if constexpr (V < MV_SUM) {
    constexpr bool GRAD = V >= MV_GRAD;
    constexpr uint32_t K = V % MV_GRAD;
    const RopeArgs a = rope_args(&r->rope);
    if constexpr (K < 6) rope_vectors<POL, K % 3, K / 3 != 0, GRAD>(a, chunk, s, tid);
    else rope_elements<POL, GRAD>(a, chunk, s, tid);
  } else if constexpr (V == MV_SUM) {
    gamma_sum<POL>(rope_args(&r->rope), chunk, s, tid);
  } else if constexpr (V < MV_LOAD) {
    const CacheArgs a = cache_args(&r->cache);
    if constexpr (V < MV_STORE + 3) store_vectors<POL, V - MV_STORE>(a, chunk, tid);
    else store_elements<POL>(a, chunk, tid);
  } else if constexpr (V < MV_PENALTY) {
    const CacheArgs a = cache_args(&r->cache);
    if constexpr (V < MV_LOAD + 3) load_vectors<POL, V - MV_LOAD>(a, chunk, tid);
    else load_elements<POL>(a, chunk, tid);
  } else {
    penalty_segments<POL, V == MV_PENALTY + 3 ? -1 : (int)(V - MV_PENALTY), T>(penalty_args(&r->penalty), chunk, s, tid);
  }
}
template <uint32_t V> PATHFN void model_path(const ModelRecord* r_v, uint32_t chunk_v, float* s_v, uint32_t tid) {
  run_model<POL_COHERENT, V, kThreads>((const ModelRecord*)lds_arg(r_v), uni(chunk_v), lds_arg(s_v), tid);
}
struct ModelExec { template <int K> static DEV void run(const ModelRecord* r, uint32_t chunk, float* s, uint32_t tid) { model_path<K>(r, chunk, s, tid); } };
__attribute__((not_tail_called)) PATHFN void exec_model(const ModelRecord* r_v, uint32_t chunk_v, float* s_v, uint32_t tid) {
  const ModelRecord* r = lds_arg(r_v);
  const uint32_t v = model_variant(uni(r->h.impl), uni((uint32_t)r->h.vec), uni((uint32_t)r->h.dtype[0]), uni((uint32_t)r->h.flags));
  pick<0, MV_COUNT, ModelExec>(v, r, uni(chunk_v), lds_arg(s_v), tid);
}

}  // namespace gpuos
