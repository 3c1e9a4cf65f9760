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
  static DEV v4i ld16(uint64_t p) {
    if (POL == POL_COHERENT) {
      const v2i a = ld8(p), b = ld8(p + 8);
      return v4i{a[0], a[1], b[0], b[1]};
    }
    return *(const G<v4i_any>*)p;
  }
  static DEV void st8(uint64_t p, v2i q) {
    if (POL == POL_COHERENT) put<uint64_t>(p, __builtin_bit_cast(uint64_t, q));
    else *(G<v2i_any>*)p = q;
  }
  static DEV void st16(uint64_t p, v4i q) {
    if (POL == POL_COHERENT) { st8(p, v2i{q[0], q[1]}); st8(p + 8, v2i{q[2], q[3]}); }
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
  template <int DT> static DEV void st4e(uint64_t p, const float* f) {
    v4i q = {0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k) Elem<DT>::put(q, k, f[k]);
    if (Elem<DT>::ES == 4) st16(p, q);
    else st8(p, v2i{q[0], q[1]});
  }
  template <int DT> static DEV void st8e(uint64_t p, const float* f) {
    if (Elem<DT>::ES == 4) {
      st4e<DT>(p, f);
      st4e<DT>(p + 16, f + 4);
    } else {
      v4i q = {0, 0, 0, 0};
#pragma unroll
      for (int k = 0; k < 8; ++k) Elem<DT>::put(q, k, f[k]);
      st16(p, q);
    }
  }
};
DEV uint32_t float_size(uint32_t dt) { return dt == GPUOS_F32 ? 4u : 2u; }
DEV uint32_t ceil_log2(uint32_t n) { return n <= 1 ? 0u : 32u - (uint32_t)__builtin_clz(n - 1); }
DEV Div uni_div(uint32_t mul, uint32_t shift) { return Div{uni(mul), uni(shift)}; }

// A row of [B, S, H, D] by its number, the head running fastest.
struct Place { uint32_t b, s, h; };
DEV Place place(uint32_t row, uint32_t heads, Div by_heads, uint32_t seq, Div by_seq) {
  Place p;
  const uint32_t token = divided(row, by_heads);
  p.h = row - token * heads;
  p.b = divided(token, by_seq);
  p.s = token - p.b * seq;
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
// ---------------------------------------------------------------------------
struct RopeArgs {
  uint64_t x, gamma, table, positions, out, dout, partial;
  uint32_t xs[4], os[4], zs[4], gs, ts, ps[2], cs, half, places, seq, heads, d, chunk, rows, dtype[4];
  Div by_seq, by_heads;
  bool pairs;
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
  a.d = uni(p->h.d); a.chunk = uni(p->h.chunk); a.rows = uni(p->h.rows);
  a.by_seq = uni_div(p->by_seq.mul, p->by_seq.shift); a.by_heads = uni_div(p->by_heads.mul, p->by_heads.shift);
  a.pairs = (uni((uint32_t)p->h.flags) & MF_PAIRS) != 0;
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

template <int POL, int DT, bool PAIRS, bool GRAD, int U>
DEV void rope_pass(const RopeArgs& a, uint32_t first, uint32_t step, uint32_t end, uint32_t u, bool active, uint32_t lanes, const float (&ga)[4],
                   const float (&gb)[4], float (&da)[4], float (&db)[4]) {
  typedef Glob<POL> M;
  constexpr uint32_t ES = Elem<DT>::ES;
  const uint32_t turned_units = a.half / 4u;
  const bool turned = u < turned_units;
  const uint32_t oa = turned ? (PAIRS ? 8u : 4u) * u : 2u * a.half + 8u * (u - turned_units);
  const uint32_t ob = turned && !PAIRS ? a.half + 4u * u : oa + 4u;
  float xe[U][8], ze[U][8], c[U][4], s[U][4];
  uint64_t to[U];
  bool ok[U], has[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    uint32_t row = first + k * step;
    ok[k] = active && row < end;
    row = row < end ? row : end - 1u;
    const Place p = place(row, a.heads, a.by_heads, a.seq, a.by_seq);
    const uint64_t xp = a.x + offset(p, a.xs) * ES;
    to[k] = a.out + offset(p, a.os) * ES;
    if (active) {
      if (PAIRS) M::template ld8e<DT>(xp + oa * ES, xe[k]);
      else { M::template ld4e<DT>(xp + oa * ES, xe[k]); M::template ld4e<DT>(xp + ob * ES, xe[k] + 4); }
      if (GRAD) {
        const uint64_t zp = a.dout + offset(p, a.zs) * ES;
        if (PAIRS) M::template ld8e<DT>(zp + oa * ES, ze[k]);
        else { M::template ld4e<DT>(zp + oa * ES, ze[k]); M::template ld4e<DT>(zp + ob * ES, ze[k] + 4); }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) xe[k][i] = ze[k][i] = 0.0f;
    }
    has[k] = true;
#pragma unroll
    for (int i = 0; i < 4; ++i) { c[k][i] = 1.0f; s[k][i] = 0.0f; }
    if (a.half != 0) {
      uint64_t row_p;
      has[k] = table_row<POL>(a, p, row_p);
      if (turned) {
        M::template ld4e<GPUOS_F32>(row_p + u * 16u, c[k]);
        M::template ld4e<GPUOS_F32>(row_p + (a.half + u * 4u) * 4u, s[k]);
      }
    }
  }
  const float inv_d = 1.0f / (float)a.d;
#pragma unroll
  for (int k = 0; k < U; ++k) {
    float xa[4], xb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) { xa[i] = xe[k][PAIRS ? 2 * i : i]; xb[i] = xe[k][PAIRS ? 2 * i + 1 : 4 + i]; }
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) { ss = __builtin_fmaf(xa[i], xa[i], ss); ss = __builtin_fmaf(xb[i], xb[i], ss); }
    ss = wave_reduce<GPUOS_IMPL_SUM_LAST>(ss, lanes);
    float r = rsqrtf(__builtin_fmaf(ss, inv_d, a.eps));
    if (!has[k]) r = __builtin_nanf("");
    float o[8];
    if (!GRAD) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float ya = xa[i] * r * ga[i], yb = xb[i] * r * gb[i];
        o[PAIRS ? 2 * i : i] = __builtin_fmaf(ya, c[k][i], -(yb * s[k][i]));
        o[PAIRS ? 2 * i + 1 : 4 + i] = __builtin_fmaf(yb, c[k][i], ya * s[k][i]);
      }
    } else {
      float ua[4], ub[4], t = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float za = ze[k][PAIRS ? 2 * i : i], zb = ze[k][PAIRS ? 2 * i + 1 : 4 + i];
        const float ya = __builtin_fmaf(za, c[k][i], zb * s[k][i]), yb = __builtin_fmaf(zb, c[k][i], -(za * s[k][i]));
        da[i] += ok[k] ? ya * (xa[i] * r) : 0.0f;
        db[i] += ok[k] ? yb * (xb[i] * r) : 0.0f;
        ua[i] = ya * ga[i];
        ub[i] = yb * gb[i];
        t = __builtin_fmaf(ua[i], xa[i], t);
        t = __builtin_fmaf(ub[i], xb[i], t);
      }
      t = wave_reduce<GPUOS_IMPL_SUM_LAST>(t, lanes);
      const float m = (t * inv_d) * r * r;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[PAIRS ? 2 * i : i] = r * __builtin_fmaf(-xa[i], m, ua[i]);
        o[PAIRS ? 2 * i + 1 : 4 + i] = r * __builtin_fmaf(-xb[i], m, ub[i]);
      }
    }
    if (ok[k]) {
      if (PAIRS) M::template st8e<DT>(to[k] + oa * ES, o);
      else { M::template st4e<DT>(to[k] + oa * ES, o); M::template st4e<DT>(to[k] + ob * ES, o + 4); }
    }
  }
}

template <int POL, int DT, bool PAIRS, bool GRAD>
DEV void rope_vectors(const RopeArgs& a, uint32_t chunk, float* s, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr int U = GRAD ? (Elem<DT>::ES == 4 ? 1 : 2) : (Elem<DT>::ES == 4 ? 2 : 4);
  const uint32_t units = a.d / 8u, lg = ceil_log2(units), lanes = 1u << lg;
  const uint32_t u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const bool active = u < units;
  const uint32_t begin = chunk * a.chunk, end = a.rows - begin < a.chunk ? a.rows : begin + a.chunk;
  const uint32_t turned_units = a.half / 4u;
  const bool turned = u < turned_units;
  const uint32_t oa = turned ? (PAIRS ? 8u : 4u) * u : 2u * a.half + 8u * (u - turned_units);
  const uint32_t ob = turned && !PAIRS ? a.half + 4u * u : oa + 4u;
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
  uint32_t row = begin;
  if (begin < a.rows) {
    for (; row + (U - 1) * step < end; row += U * step) rope_pass<POL, DT, PAIRS, GRAD, U>(a, row + group, step, end, u, active, lanes, ga, gb, da, db);
    if (U > 1)
      for (; row < end; row += step) rope_pass<POL, DT, PAIRS, GRAD, 1>(a, row + group, step, end, u, active, lanes, ga, gb, da, db);
  }
  if (GRAD && a.partial != 0) {
    if (active) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t ja = PAIRS ? oa + 2u * i : oa + i, jb = PAIRS ? oa + 2u * i + 1u : ob + i;
        s[group * a.d + ja] = da[i];
        s[group * a.d + jb] = db[i];
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
  const bool empty = a.rows == ModelPack::kNoRows;
  const uint32_t rows = empty ? 0u : a.rows, begin = chunk * a.chunk, end = rows <= begin ? begin : (rows - begin < a.chunk ? rows : begin + a.chunk);
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
  for (uint32_t base = begin; base < end; base += step) {
    const bool in = base + group < end;
    const uint32_t row = in ? base + group : end - 1u;
    const Place p = place(row, a.heads, a.by_heads, a.seq, a.by_seq);
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
        oa[k] = __builtin_fmaf(ya, c[k], -(yb * sn[k]));
        ob[k] = __builtin_fmaf(yb, c[k], ya * sn[k]);
      }
    } else {
      float t = 0.0f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const float ya = __builtin_fmaf(za[k], c[k], zb[k] * sn[k]), yb = __builtin_fmaf(zb[k], c[k], -(za[k] * sn[k]));
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
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (in && in_a[k]) M::st_rt(op + (uint64_t)ja[k] * a.os[3] * eo, a.dtype[1], oa[k]);
      if (in && in_b[k]) M::st_rt(op + (uint64_t)jb[k] * a.os[3] * eo, a.dtype[1], ob[k]);
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

// GAMMA_SUM: a wavefront a row of the partial sums, always in the same order.
template <int POL> DEV void gamma_sum(const RopeArgs& a, uint32_t chunk, uint32_t tid) {
  typedef Glob<POL> M;
  const uint32_t begin = chunk * a.chunk, end = a.rows - begin < a.chunk ? a.rows : begin + a.chunk;
  const uint32_t lane = tid & 63u;
  for (uint32_t row = begin + (tid >> 6); row < end; row += kThreads / 64u) {
    const uint64_t p = a.partial + (uint64_t)row * a.cs * 4u;
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (uint32_t i = lane; i < a.d; i += 256u) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k * 64u < a.d) sum[k] += M::ldf(p + (uint64_t)(i + k * 64u) * 4u);
    }
    const float all = wave_reduce<GPUOS_IMPL_SUM_LAST>((sum[0] + sum[1]) + (sum[2] + sum[3]), 64u);
    if (lane == 0) M::st_rt(a.out + (uint64_t)row * a.os[0] * float_size(a.dtype[1]), a.dtype[1], all);
  }
}

// ---------------------------------------------------------------------------
// CACHE_STORE, CACHE_LOAD
//
// Bound by memory, three bytes of it an element of 16 bits.  A part of a wavefront takes a row: eight elements a lane, one load of 16
// bytes on the wide side and one of 8 on the cache's; a group's largest magnitude goes over the lanes that hold it, as an integer
// (magnitudes order like their bits, infinities and NaNs above all).
// ---------------------------------------------------------------------------
struct CacheArgs {
  uint64_t x, cache, scales, slots, lengths;
  uint32_t xs[4], cs[3], ss[4], ps[2], ls, pages, page, group, heads, seq, d, chunk, rows, dtype, format;
  Div by_heads, by_seq, by_page, by_group;
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
  a.d = uni(p->h.d); a.chunk = uni(p->h.chunk); a.rows = uni(p->h.rows);
  a.dtype = uni((uint32_t)p->h.dtype[0]); a.format = uni((uint32_t)p->h.dtype[1]);
  a.by_heads = uni_div(p->by_heads.mul, p->by_heads.shift); a.by_seq = uni_div(p->by_seq.mul, p->by_seq.shift); a.by_page = uni_div(p->by_page.mul, p->by_page.shift); a.by_group = uni_div(p->by_group.mul, p->by_group.shift);
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

template <int POL, int DT, int U>
DEV void store_pass(const CacheArgs& a, uint32_t first, uint32_t step, uint32_t end, uint32_t u, bool active, uint32_t width, uint32_t lg_width) {
  typedef Glob<POL> M;
  float x[U][8];
  int32_t slot[U];
  uint32_t h[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const uint32_t row = first + k * step;
    const bool in = row < end;
    const Place p = place(in ? row : end - 1u, a.heads, a.by_heads, a.seq, a.by_seq);
    h[k] = p.h;
    slot[k] = M::ldi(a.slots + ((uint64_t)p.b * a.ps[0] + (uint64_t)p.s * a.ps[1]) * 4u);
    if (!in || (uint32_t)slot[k] >= a.pages * a.page) slot[k] = -1;
    if (active) M::template ld8e<DT>(a.x + (offset(p, a.xs) + u * 8u) * Elem<DT>::ES, x[k]);
    else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[k][i] = 0.0f;
    }
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) { const uint32_t m = magnitude(x[k][i]); top = m > top ? m : top; }
    top = (uint32_t)wave_reduce<GPUOS_IMPL_MAX_LAST>((int32_t)top, width);
    const Quant q = quant(top, a.format);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = q.bad ? 0.0f : x[k][i] * q.inv;
    const v2i w = {(int)pack_q(y, a.format), (int)pack_q(y + 4, a.format)};
    if (slot[k] >= 0 && active) {
      const uint32_t page = divided((uint32_t)slot[k], a.by_page), in = (uint32_t)slot[k] - page * a.page;
      M::st8b(cache_at(a, page, in, h[k]) + u * 8u, w);
      if ((u & (width - 1u)) == 0) M::stf(scale_at(a, page, in, h[k], u >> lg_width), q.scale);
    }
  }
}
template <int POL, int DT> DEV void store_vectors(const CacheArgs& a, uint32_t chunk, uint32_t tid) {
  constexpr int U = Elem<DT>::ES == 4 ? 2 : 4;
  const uint32_t units = a.d / 8u, lg = ceil_log2(units), lanes = 1u << lg;
  const uint32_t u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t lg_width = a.group == a.d ? lg : ceil_log2(a.group) - 3u, width = 1u << lg_width;
  const uint32_t begin = chunk * a.chunk, end = a.rows - begin < a.chunk ? a.rows : begin + a.chunk;
  uint32_t row = begin;
  for (; row + (U - 1) * step < end; row += U * step) store_pass<POL, DT, U>(a, row + group, step, end, u, u < units, width, lg_width);
  for (; row < end; row += step) store_pass<POL, DT, 1>(a, row + group, step, end, u, u < units, width, lg_width);
}
// rows of any length, strides and alignment: element by element, neighbouring lanes neighbouring elements
template <int POL> DEV void store_elements(const CacheArgs& a, uint32_t chunk, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr int K = 8;
  const uint32_t lg = a.d > 64u ? 6u : ceil_log2(a.d), lanes = 1u << lg, u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t es = float_size(a.dtype);
  const uint32_t begin = chunk * a.chunk, end = a.rows - begin < a.chunk ? a.rows : begin + a.chunk;
  // A group is the row, or a power of two: then `width` lanes of a register hold it, or `span` registers of all lanes.
  const bool whole = a.group == a.d;
  const uint32_t width = whole || a.group >= lanes ? lanes : a.group, span = whole ? (uint32_t)K : (a.group > lanes ? a.group >> lg : 1u);
  for (uint32_t base = begin; base < end; base += step) {
    const bool in_row = base + group < end;
    const Place p = place(in_row ? base + group : end - 1u, a.heads, a.by_heads, a.seq, a.by_seq);
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
template <int POL, int DT, int U>
DEV void load_pass(const CacheArgs& a, uint32_t first, uint32_t step, uint32_t end, uint32_t u, bool active, uint32_t lg_width) {
  typedef Glob<POL> M;
  v2i w[U];
  float scale[U];
  uint32_t what[U];
  uint64_t to[U];
#pragma unroll
  for (int k = 0; k < U; ++k) {
    const uint32_t row = first + k * step;
    const bool in_row = row < end;
    const Place p = place(in_row ? row : end - 1u, a.heads, a.by_heads, a.seq, a.by_seq);
    to[k] = in_row && active ? a.x + (offset(p, a.xs) + u * 8u) * Elem<DT>::ES : 0;
    uint32_t page, in;
    what[k] = sequence_row<POL>(a, p, page, in);
    w[k] = v2i{0, 0};
    scale[k] = what[k] == 1u ? 0.0f : __builtin_nanf("");
    if (what[k] == 0u && active) {
      w[k] = M::ld8b(cache_at(a, page, in, p.h) + u * 8u);
      scale[k] = M::ldf(scale_at(a, page, in, p.h, u >> lg_width));
    }
  }
#pragma unroll
  for (int k = 0; k < U; ++k) {
    float y[8];
    unpack_q((uint32_t)w[k][0], a.format, y);
    unpack_q((uint32_t)w[k][1], a.format, y + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] *= scale[k];
    if (to[k] != 0) M::template st8e<DT>(to[k], y);
  }
}
template <int POL, int DT> DEV void load_vectors(const CacheArgs& a, uint32_t chunk, uint32_t tid) {
  constexpr int U = 4;
  const uint32_t units = a.d / 8u, lg = ceil_log2(units), lanes = 1u << lg;
  const uint32_t u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t lg_width = a.group == a.d ? lg : ceil_log2(a.group) - 3u;
  const uint32_t begin = chunk * a.chunk, end = a.rows - begin < a.chunk ? a.rows : begin + a.chunk;
  uint32_t row = begin;
  for (; row + (U - 1) * step < end; row += U * step) load_pass<POL, DT, U>(a, row + group, step, end, u, u < units, lg_width);
  for (; row < end; row += step) load_pass<POL, DT, 1>(a, row + group, step, end, u, u < units, lg_width);
}
template <int POL> DEV void load_elements(const CacheArgs& a, uint32_t chunk, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr int K = 8;
  const uint32_t lg = a.d > 64u ? 6u : ceil_log2(a.d), lanes = 1u << lg, u = tid & (lanes - 1u), group = tid >> lg, step = kThreads >> lg;
  const uint32_t es = float_size(a.dtype);
  const uint32_t begin = chunk * a.chunk, end = a.rows - begin < a.chunk ? a.rows : begin + a.chunk;
  for (uint32_t row = begin + group; row < end; row += step) {
    const Place p = place(row, a.heads, a.by_heads, a.seq, a.by_seq);
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
// the segment is read, changed and written once.  Every segment reads the row's history, from the cache after the first.
// A count has 31 bits; the top bit says that the token is in the prompt.
// ---------------------------------------------------------------------------
struct PenaltyArgs {
  uint64_t x, out, history, prompts, params, bias, allowed;
  uint32_t xs[2], os[2], hs[2], ps, ms[2], bs[2], as[2], n, seg, segs, v, chunk, rows, dtype[3];
  Div by_segs;
};
template <class P> DEV PenaltyArgs penalty_args(P p) {
  PenaltyArgs a;
  a.x = uni64(p->x); a.out = uni64(p->out); a.history = uni64(p->history); a.prompts = uni64(p->prompts); a.params = uni64(p->params);
  a.bias = uni64(p->bias); a.allowed = uni64(p->allowed);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    a.xs[k] = uni(p->xs[k]); a.os[k] = uni(p->os[k]); a.hs[k] = uni(p->hs[k]); a.ms[k] = uni(p->ms[k]); a.bs[k] = uni(p->bs[k]); a.as[k] = uni(p->as[k]);
  }
  a.ps = uni(p->ps); a.n = uni(p->n); a.seg = uni(p->seg); a.segs = uni(p->segs); a.v = uni(p->h.d); a.chunk = uni(p->h.chunk); a.rows = uni(p->h.rows);
#pragma unroll
  for (int k = 0; k < 3; ++k) a.dtype[k] = uni((uint32_t)p->h.dtype[k]);
  a.by_segs = uni_div(p->by_segs.mul, p->by_segs.shift);
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
template <int POL> DEV void count_tokens(const PenaltyArgs& a, uint32_t row, uint32_t v0, uint32_t nv, uint32_t* seen, uint32_t tid) {
  typedef Glob<POL> M;
  constexpr int K = 4;
  const uint64_t h = a.history + (uint64_t)row * a.hs[0] * 4u;
  const int32_t prompt = a.prompts != 0 ? M::ldi(a.prompts + (uint64_t)row * a.ps * 4u) : 0;
  for (uint32_t j = tid; j < (nv + 3u) / 4u; j += kThreads) ((v4i*)seen)[j] = v4i{0, 0, 0, 0};
  __syncthreads();
  auto take = [&](int32_t id, uint32_t i) {
    const uint32_t j = (uint32_t)id - v0;              // (an id below v0, negative ones too, is over nv so)
    if (j < nv) {
      if ((int32_t)i < prompt) __hip_atomic_fetch_or(&seen[j], 0x80000000u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
      else __hip_atomic_fetch_add(&seen[j], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    }
  };
  uint32_t i = 0;
  if (POL == POL_PLAIN && a.hs[1] == 1u) {
    for (; i + K * kThreads * 4u <= a.n; i += K * kThreads * 4u) {
      v4i q[K];
#pragma unroll
      for (int k = 0; k < K; ++k) q[k] = M::ld16(h + ((uint64_t)i + (k * kThreads + tid) * 4u) * 4u);
#pragma unroll
      for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) take(q[k][e], i + (k * kThreads + tid) * 4u + e);
      }
    }
  }
  for (i += tid; i < a.n; i += K * kThreads) {
    int32_t id[K];
#pragma unroll
    for (int k = 0; k < K; ++k) id[k] = i + k * kThreads < a.n ? M::ldi(h + (uint64_t)(i + k * kThreads) * a.hs[1] * 4u) : -1;
#pragma unroll
    for (int k = 0; k < K; ++k) take(id[k], i + k * kThreads);
  }
  __syncthreads();
}
// one element of any operand
template <int POL> DEV void penalize_one(const PenaltyArgs& a, uint32_t row, uint32_t v, uint32_t seen, const Penalty& pen) {
  typedef Glob<POL> M;
  float y = M::ld_rt(a.x + ((uint64_t)row * a.xs[0] + (uint64_t)v * a.xs[1]) * float_size(a.dtype[0]), a.dtype[0]);
  y = penalize(y, seen, pen);
  if (a.bias != 0) y += M::ld_rt(a.bias + ((uint64_t)row * a.bs[0] + (uint64_t)v * a.bs[1]) * float_size(a.dtype[2]), a.dtype[2]);
  if (a.allowed != 0 && ((M::template at<uint32_t>(a.allowed + ((uint64_t)row * a.as[0] + (uint64_t)(v >> 5) * a.as[1]) * 4u) >> (v & 31u)) & 1u) == 0)
    y = -__builtin_inff();
  M::st_rt(a.out + ((uint64_t)row * a.os[0] + (uint64_t)v * a.os[1]) * float_size(a.dtype[1]), a.dtype[1], y);
}
// DT < 0: element by element
template <int POL, int DT> DEV void penalty_segments(const PenaltyArgs& a, uint32_t chunk, float* s, uint32_t tid) {
  typedef Glob<POL> M;
  uint32_t* seen = (uint32_t*)s;
  const uint32_t begin = chunk * a.chunk, end = a.rows - begin < a.chunk ? a.rows : begin + a.chunk;
  for (uint32_t item = begin; item < end; ++item) {
    const uint32_t row = divided(item, a.by_segs), v0 = (item - row * a.segs) * a.seg, nv = a.v - v0 < a.seg ? a.v - v0 : a.seg;
    Penalty pen = {1.0f, 0.0f, 0.0f};
    if (a.history != 0) {
      if (item != begin) __syncthreads();              // (the counts of the segment before have been read)
      const uint64_t p = a.params + (uint64_t)row * a.ms[0] * 4u;
      pen = {M::ldf(p), M::ldf(p + (uint64_t)a.ms[1] * 4u), M::ldf(p + (uint64_t)a.ms[1] * 8u)};
      count_tokens<POL>(a, row, v0, nv, seen, tid);
    }
    uint32_t done = 0;
    if constexpr (DT >= 0) {
      constexpr uint32_t ES = Elem<DT>::ES;
      const uint64_t xp = a.x + ((uint64_t)row * a.xs[0] + v0) * ES, op = a.out + ((uint64_t)row * a.os[0] + v0) * ES;
      const uint64_t bp = a.bias + ((uint64_t)row * a.bs[0] + v0) * float_size(a.dtype[2]), ap = a.allowed + (uint64_t)row * a.as[0] * 4u;
      done = nv & ~7u;
      for (uint32_t j = tid * 8u; j < done; j += kThreads * 8u) {
        float y[8];
        M::template ld8e<DT>(xp + j * ES, y);
        uint32_t bits = 0xffu;
        if (a.allowed != 0) bits = M::template at<uint32_t>(ap + ((v0 + j) >> 5) * 4u) >> ((v0 + j) & 31u);
        if (a.history != 0) {
          const v4i lo = *(const v4i*)(seen + j), hi = *(const v4i*)(seen + j + 4);
          if ((lo[0] | lo[1] | lo[2] | lo[3] | hi[0] | hi[1] | hi[2] | hi[3]) != 0) {
#pragma unroll
            for (int k = 0; k < 4; ++k) { y[k] = penalize(y[k], (uint32_t)lo[k], pen); y[4 + k] = penalize(y[4 + k], (uint32_t)hi[k], pen); }
          }
        }
        if (a.bias != 0) {
          float b[8];
          if (POL == POL_COHERENT) {
#pragma unroll
            for (int k = 0; k < 8; ++k) b[k] = M::ld_rt(bp + (j + k) * float_size(a.dtype[2]), a.dtype[2]);
          } else if (a.dtype[2] == GPUOS_F32) M::template ld8e<GPUOS_F32>(bp + j * 4u, b);
          else if (a.dtype[2] == GPUOS_F16) M::template ld8e<GPUOS_F16>(bp + j * 2u, b);
          else M::template ld8e<GPUOS_BF16>(bp + j * 2u, b);
#pragma unroll
          for (int k = 0; k < 8; ++k) y[k] += b[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) y[k] = (bits >> k) & 1u ? y[k] : -__builtin_inff();
        M::template st8e<DT>(op + j * ES, y);
      }
    }
    for (uint32_t j = done + tid; j < nv; j += kThreads) penalize_one<POL>(a, row, v0 + j, a.history != 0 ? seen[j] : 0u, pen);
  }
}
static_assert(ModelPack::kSegment <= kScratchFloats && ModelPack::kSegment % 32 == 0, "a segment's counts fit the LDS scratch; its words of bits are whole");

// ---------------------------------------------------------------------------
// the executors of the worker: functions of their own, like its others
// ---------------------------------------------------------------------------
template <int VARIANT> PATHFN void rope_path(const RopeRecord* r_v, uint32_t chunk_v, float* s_v, uint32_t tid) {
  const RopeArgs a = rope_args(lds_arg(r_v));
  float* s = lds_arg(s_v);
  const uint32_t chunk = uni(chunk_v);
  if constexpr (VARIANT < 12) rope_vectors<POL_COHERENT, VARIANT % 3, (VARIANT / 3) % 2 != 0, VARIANT / 6 != 0>(a, chunk, s, tid);
  else if constexpr (VARIANT == 12) rope_elements<POL_COHERENT, false>(a, chunk, s, tid);
  else if constexpr (VARIANT == 13) rope_elements<POL_COHERENT, true>(a, chunk, s, tid);
  else gamma_sum<POL_COHERENT>(a, chunk, tid);
}
template <int VARIANT> PATHFN void cache_path(const CacheRecord* r_v, uint32_t chunk_v, uint32_t tid) {
  const CacheArgs a = cache_args(lds_arg(r_v));
  const uint32_t chunk = uni(chunk_v);
  if constexpr (VARIANT < 3) store_vectors<POL_COHERENT, VARIANT>(a, chunk, tid);
  else if constexpr (VARIANT == 3) store_elements<POL_COHERENT>(a, chunk, tid);
  else if constexpr (VARIANT < 7) load_vectors<POL_COHERENT, VARIANT - 4>(a, chunk, tid);
  else load_elements<POL_COHERENT>(a, chunk, tid);
}
template <int DT> PATHFN void penalty_path(const PenaltyRecord* r_v, uint32_t chunk_v, float* s_v, uint32_t tid) {
  const PenaltyArgs a = penalty_args(lds_arg(r_v));
  penalty_segments<POL_COHERENT, DT>(a, uni(chunk_v), lds_arg(s_v), tid);
}
struct RopeExec { template <int K> static DEV void run(const RopeRecord* r, uint32_t chunk, float* s, uint32_t tid) { rope_path<K>(r, chunk, s, tid); } };
struct CacheExec { template <int K> static DEV void run(const CacheRecord* r, uint32_t chunk, uint32_t tid) { cache_path<K>(r, chunk, tid); } };
struct PenaltyExec { template <int K> static DEV void run(const PenaltyRecord* r, uint32_t chunk, float* s, uint32_t tid) { penalty_path<K - 1>(r, chunk, s, tid); } };

// which executor a record asks for
DEV uint32_t rope_variant(uint32_t impl, uint32_t vec, uint32_t dt, bool pairs) {
  const uint32_t grad = impl == GPUOS_IMPL_NORM_ROPE_GRAD ? 1u : 0u;
  return impl == GPUOS_IMPL_GAMMA_SUM ? 14u : (vec != 0 ? dt + (pairs ? 3u : 0u) + 6u * grad : 12u + grad);
}
DEV uint32_t cache_variant(uint32_t impl, uint32_t vec, uint32_t dt) { return (vec != 0 ? dt : 3u) + (impl == GPUOS_IMPL_CACHE_LOAD ? 4u : 0u); }

__attribute__((not_tail_called)) PATHFN void exec_model(const ModelRecord* r_v, uint32_t chunk_v, float* s_v, uint32_t wave_v) {
  const ModelRecord* r = lds_arg(r_v);
  float* s = lds_arg(s_v);
  const uint32_t chunk = uni(chunk_v), tid = thread_index(uni(wave_v));
  const uint32_t impl = uni(r->h.impl), vec = uni((uint32_t)r->h.vec), dt = uni((uint32_t)r->h.dtype[0]);
  if (impl <= GPUOS_IMPL_GAMMA_SUM) pick<0, 15, RopeExec>(rope_variant(impl, vec, dt, (uni((uint32_t)r->h.flags) & MF_PAIRS) != 0), &r->rope, chunk, s, tid);
  else if (impl != GPUOS_IMPL_LOGIT_PENALTY) pick<0, 8, CacheExec>(cache_variant(impl, vec, dt), &r->cache, chunk, tid);
  else pick<0, 4, PenaltyExec>(vec != 0 ? dt + 1u : 0u, &r->penalty, chunk, s, tid);
}

}  // namespace gpuos
