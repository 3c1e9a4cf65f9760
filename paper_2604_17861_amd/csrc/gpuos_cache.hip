// gpuos_cache.hip -- the kernels of the cache operators: appending rotated keys and values, attention over a cache.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gpuos_cache.h"

namespace gpuos {

#define DEV __device__ __forceinline__
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
template <class T> using G = __attribute__((address_space(1))) T;
typedef u4 __attribute__((aligned(2))) u4_any;
typedef u2 __attribute__((aligned(1))) u2_any;
typedef u4 __attribute__((aligned(1))) u4_byte;
typedef uint32_t __attribute__((aligned(1))) u1_any;
template <class T> DEV T ld(uint64_t p) { return *(const G<T>*)p; }
template <class T> DEV void st(uint64_t p, T v) { *(G<T>*)p = v; }
DEV float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
DEV uint32_t as_u(float f) { return __builtin_bit_cast(uint32_t, f); }
constexpr uint32_t size_of(uint32_t dt) { return dt == GPUOS_F32 ? 4u : 2u; }
template <uint32_t DT> DEV float ld_elem(uint64_t p) {
  if (DT == GPUOS_F32) return ld<float>(p);
  const uint16_t h = ld<uint16_t>(p);
  return DT == GPUOS_F16 ? (float)__builtin_bit_cast(_Float16, h) : as_f((uint32_t)h << 16);
}
template <uint32_t DT> DEV uint32_t half_bits(float f) {
  asm("" : "+v"(f));                       // (or a product and its rounding to 16 bits become one instruction, with one rounding)
  return DT == GPUOS_F16 ? (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)f) : (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)f);
}
template <uint32_t DT> DEV void st_elem(uint64_t p, float f) {
  if (DT == GPUOS_F32) st<float>(p, f);
  else st<uint16_t>(p, (uint16_t)half_bits<DT>(f));
}
// eight elements that follow each other
template <uint32_t DT> DEV void ld8(uint64_t p, float* f) {
  const u4 a = ld<u4_any>(p);
  if (DT == GPUOS_F32) {
    const u4 b = ld<u4_any>(p + 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[i] = as_f(a[i]); f[4 + i] = as_f(b[i]); }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t h = i & 1 ? a[i / 2] >> 16 : a[i / 2] & 0xffffu;
      f[i] = DT == GPUOS_F16 ? (float)__builtin_bit_cast(_Float16, (uint16_t)h) : as_f(h << 16);
    }
  }
}
template <uint32_t DT> DEV void st8(uint64_t p, const float* f) {
  if (DT == GPUOS_F32) {
    st<u4_any>(p, u4{as_u(f[0]), as_u(f[1]), as_u(f[2]), as_u(f[3])});
    st<u4_any>(p + 16, u4{as_u(f[4]), as_u(f[5]), as_u(f[6]), as_u(f[7])});
  } else {
    u4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = half_bits<DT>(f[2 * i]) | (half_bits<DT>(f[2 * i + 1]) << 16);
    st<u4_any>(p, w);
  }
}

template <uint32_t DT> DEV void st4(uint64_t p, f4 f) {
  if (DT == GPUOS_F32) st<u4_any>(p, __builtin_bit_cast(u4, f));
  else st<u2_any>(p, u2{half_bits<DT>(f[0]) | (half_bits<DT>(f[1]) << 16), half_bits<DT>(f[2]) | (half_bits<DT>(f[3]) << 16)});
}

// ---------------------------------------------------------------------------
// GPUOS_CACHE_APPEND
//
// Bound by memory: rows are read once (a rotation reads its other half a second time, out of the line that a neighbouring lane has asked
// for), and written once, in 16 or 32 bits or as codes.  A power of two of lanes holds a row, eight elements each; what goes over
// lanes is a group's maximum.  Products and sums of the rotation are rounded by themselves (no fused multiply-add), so that the codes
// are those of the definition.
// Queries, keys and values are the grid's second index, so that what a workgroup does is the same in all its lanes: with heads of all three in one
// list, chosen by lanes, an item took 600 vector instructions, and those were what bounded it: 16,384 tokens of 32 + 8 + 8 heads of 128 bf16
// into 4 bits 103 us, so 82 (364 MB, 4.4 TB/s; a large copy makes 5.0); 8,192 of 16 + 16 + 16 of fp16 into e4m3 56 and 37.6 (170 MB, 4.5).  A token of
// 32 heads 4.2 us: three trips to memory.  Blocks of four heads instead of two cost a token 1.6 us and gain nothing, stores past
// the caches neither.  Element by element the 16,384 tokens take 546 us (a last dim of every second element; eight loads and addresses in place of one); heads
// of 100 318.
// ---------------------------------------------------------------------------
// eight codes of |y| <= qmax (1 + 2^-23): to the nearest, to the even one of two
DEV u2 encode(const float* y, uint32_t format) {
  u2 w = {0, 0};
  if (format == CF_E2M1) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], 1.0f, 3);
    w[0] = c;
  } else if (format == CF_I8) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i / 4] |= ((uint32_t)(int32_t)__builtin_rintf(y[i]) & 0xffu) << (8 * (i % 4));
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
      w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], c, true);
    }
  }
  return w;
}

// the largest over `width` lanes, a power of two of them
DEV uint32_t most_of(uint32_t v, uint32_t width) {
  auto with = [&](int other) { v = v > (uint32_t)other ? v : (uint32_t)other; };
  if (width > 1u) with(__builtin_amdgcn_update_dpp(0, (int)v, 0xb1, 0xf, 0xf, true));      // quad_perm 1 0 3 2
  if (width > 2u) with(__builtin_amdgcn_update_dpp(0, (int)v, 0x4e, 0xf, 0xf, true));      // quad_perm 2 3 0 1
  if (width > 4u) with(__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, true));     // half a row of 16 mirrored
  if (width > 8u) with(__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xf, 0xf, true));     // a row mirrored
  if (width > 16u) {
    auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = r[0] > r[1] ? r[0] : r[1];
  }
  if (width > 32u) {
    auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = r[0] > r[1] ? r[0] : r[1];
  }
  return v;
}

// The grid's second index is the side: queries, keys, values.  An item is a token and a block of its heads.
// VEC: rows in vectors of eight, each all first, all second or all not rotated elements (neighbours: all rotated or none), last dims dense;
// else element by element, a head at a time.
template <uint32_t DT, bool VEC> __global__ void __launch_bounds__(kThreads, 4) gpuos_cache_append_kernel(const AppendArgs args) {
  const AppendSide& a = args.side[blockIdx.y];
  if (blockIdx.x >= a.chunks) return;
  constexpr uint32_t ES = size_of(DT);
  constexpr int U = VEC ? kAppendBlock : 1;
  const uint32_t d = args.d, n = args.half, format = args.format;
  const bool stored = blockIdx.y != 0u, turns = blockIdx.y != 2u && n != 0u, pairs = args.pairs != 0u;
  const uint32_t units = (d + 7u) / 8u, lg = units <= 1u ? 0u : 32u - (uint32_t)__builtin_clz(units - 1u), lanes = 1u << lg;
  const uint32_t u = threadIdx.x & (lanes - 1u), row = threadIdx.x >> lg, step = kThreads >> lg;
  const uint32_t lg_width = args.group == d ? lg : 28u - (uint32_t)__builtin_clz(args.group), width = 1u << lg_width;      // lanes of a group
  const bool mine = u < units;                                               // (the others do as the last that has some, and store nothing)
  const uint32_t j0 = 8u * (mine ? u : units - 1u), left = VEC || d - j0 >= 8u ? 8u : d - j0;
  const bool first = j0 < n, turned = turns && j0 < 2u * n;                  // (of a vector's elements: all)
  for (uint32_t base = blockIdx.x * step; base < a.items; base += a.chunks * step) {
    const uint32_t item = base + row < a.items ? base + row : a.items - 1u;
    const bool there = base + row < a.items && mine;
    const uint32_t token = divided(item, a.by_blocks), h = (item - token * a.blocks) * U;
    const uint32_t b = divided(token, args.by_seq), s = token - b * args.seq;
    const uint64_t xp = a.x + ((uint64_t)b * a.xs[0] + (uint64_t)s * a.xs[1] + (uint64_t)h * a.xs[2]) * ES;
    const uint32_t last = a.heads - 1u - h < (uint32_t)U - 1u ? a.heads - 1u - h : (uint32_t)U - 1u;      // of the block's heads
    uint32_t place = 0, slot = 0;
    if (turns) place = args.positions != 0 ? ld<uint32_t>(args.positions + ((uint64_t)b * args.ps[0] + (uint64_t)s * args.ps[1]) * 4u) : s;
    if (stored) slot = ld<uint32_t>(args.slots + ((uint64_t)b * args.ls[0] + (uint64_t)s * args.ls[1]) * 4u);
    const bool has = place < args.places || !turns;
    const uint64_t cosines = args.table + (uint64_t)(has ? place : 0u) * args.ts * 4u, sines = cosines + (uint64_t)n * 4u;
    float z[U][8];
    if constexpr (VEC) {
      float p[U][8];                                                         // the other elements of their pairs
#pragma unroll
      for (uint32_t k = 0; k < (uint32_t)U; ++k) {
        const uint64_t at = xp + (uint64_t)(k < last ? k : last) * a.xs[2] * ES;
        ld8<DT>(at + j0 * ES, z[k]);
        if (turned && !pairs) ld8<DT>(at + (first ? j0 + n : j0 - n) * ES, p[k]);
      }
      if (turned) {
        float c[8], sn[8];
        if (pairs) {
          const u4 cc = ld<u4_any>(cosines + j0 * 2u), sc = ld<u4_any>(sines + j0 * 2u);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (uint32_t k = 0; k < (uint32_t)U; ++k) {
              const float y = z[k][2 * i], w = z[k][2 * i + 1];
              z[k][2 * i] = y * as_f(cc[i]) - w * as_f(sc[i]);
              z[k][2 * i + 1] = w * as_f(cc[i]) + y * as_f(sc[i]);
            }
          }
        } else {
          const uint32_t at = (first ? j0 : j0 - n) * 4u, sign = first ? 0x80000000u : 0u;
          ld8<GPUOS_F32>(cosines + at, c);
          ld8<GPUOS_F32>(sines + at, sn);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            sn[i] = as_f(as_u(sn[i]) ^ sign);
#pragma unroll
            for (uint32_t k = 0; k < (uint32_t)U; ++k) z[k][i] = z[k][i] * c[i] + p[k][i] * sn[i];
          }
        }
      }
    } else {
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i) {
        const uint32_t j = j0 + i;
        z[0][i] = 0.0f;
        if (i < left) {
          z[0][i] = ld_elem<DT>(xp + (uint64_t)j * a.xs[3] * ES);
          if (turns && j < 2u * n) {
            const uint32_t o = pairs ? j ^ 1u : (j < n ? j + n : j - n), at = pairs ? j / 2u : (j < n ? j : j - n);
            const float c = ld<float>(cosines + (uint64_t)at * 4u), sn = ld<float>(sines + (uint64_t)at * 4u), p = ld_elem<DT>(xp + (uint64_t)o * a.xs[3] * ES);
            z[0][i] = z[0][i] * c + p * ((pairs ? (j & 1u) == 0u : j < n) ? -sn : sn);
          }
        }
      }
    }
    if (__builtin_amdgcn_ballot_w64(!has) != 0) {                            // a position outside the table
#pragma unroll
      for (uint32_t k = 0; k < (uint32_t)U; ++k) {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) z[k][i] = has || i >= left ? z[k][i] : __builtin_nanf("");
      }
    }
    if (!stored) {
      const uint64_t to = a.to + ((uint64_t)b * a.ts[0] + (uint64_t)s * a.ts[1] + (uint64_t)h * a.ts[2]) * ES;
#pragma unroll
      for (uint32_t k = 0; k < (uint32_t)U; ++k) {
        if (!there || k > last) continue;
        const uint64_t at = to + (uint64_t)k * a.ts[2] * ES;
        if constexpr (VEC) st8<DT>(at + j0 * ES, z[k]);
        else {
#pragma unroll
          for (uint32_t i = 0; i < 8; ++i) {
            if (i < left) st_elem<DT>(at + (uint64_t)(j0 + i) * a.ts[3] * ES, z[k][i]);
          }
        }
      }
      continue;
    }
    const bool kept = there && slot < args.pages * args.page;
    const uint32_t page = divided(kept ? slot : 0u, args.by_page), in = kept ? slot - page * args.page : 0u;
    const uint64_t to = a.to + (uint64_t)page * a.ts[0] + (uint64_t)in * a.ts[1] + (uint64_t)h * a.ts[2];
    const uint64_t scale_to = a.scales + ((uint64_t)page * a.ss[0] + (uint64_t)in * a.ss[1] + (uint64_t)h * a.ss[2] + (uint64_t)(u >> lg_width) * a.ss[3]) * 4u;
    const float qmax = format == CF_E2M1 ? 6.0f : (format == CF_I8 ? 127.0f : 448.0f);
#pragma unroll
    for (uint32_t k = 0; k < (uint32_t)U; ++k) {
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t m = as_u(z[k][i]) & 0x7fffffffu;
        top = m > top ? m : top;
      }
      top = most_of(top, width);                                             // (lanes without elements have the last one's)
      const float m = __builtin_fmaxf(as_f(top), 0x1p-100f), inv = qmax / m;
      const bool bad = top >= 0x7f800000u;
      if (__builtin_amdgcn_ballot_w64(bad) != 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[k][i] = bad ? 0.0f : z[k][i];
      }
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = z[k][i] * inv;
      const u2 w = encode(y, format);
      if (!kept || k > last) continue;
      const uint64_t at = to + (uint64_t)k * a.ts[2];
      if (format == CF_E2M1) {
        if (VEC || left == 8u) st<u1_any>(at + j0 / 2u, w[0]);
        else for (uint32_t i = 0; i < left / 2u; ++i) st<uint8_t>(at + j0 / 2u + i, (uint8_t)(w[0] >> (8u * i)));
      } else {
        if (VEC || left == 8u) st<u2_any>(at + j0, w);
        else for (uint32_t i = 0; i < left; ++i) st<uint8_t>(at + j0 + i, (uint8_t)((i < 4u ? w[0] : w[1]) >> (8u * (i & 3u))));
      }
      if ((u & (width - 1u)) == 0u) st<float>(scale_to + (uint64_t)k * a.ss[2] * 4u, bad ? __builtin_nanf("") : m / qmax);
    }
  }
}

int launch_append(const AppendArgs& a, void* stream) {
  const uint32_t chunks = a.side[0].chunks > a.side[1].chunks ? a.side[0].chunks : a.side[1].chunks;
  const void* const kernels[] = {(const void*)gpuos_cache_append_kernel<GPUOS_F32, true>,   (const void*)gpuos_cache_append_kernel<GPUOS_F16, true>,
                                 (const void*)gpuos_cache_append_kernel<GPUOS_BF16, true>,  (const void*)gpuos_cache_append_kernel<GPUOS_F32, false>,
                                 (const void*)gpuos_cache_append_kernel<GPUOS_F16, false>, (const void*)gpuos_cache_append_kernel<GPUOS_BF16, false>};
  void* args[] = {(void*)&a};
  return (int)hipLaunchKernel(kernels[a.dtype + (a.vec ? 0u : 3u)], dim3(chunks, 3), dim3(kThreads), args, 0, (hipStream_t)stream);
}

// ---------------------------------------------------------------------------
// GPUOS_CACHE_ATTENTION
//
// o_r = sum_t p_rt v_t / sum_t p_rt,  p_rt = 2^(x_rt - m_r),  x_rt = scale log2(e) q_r . k_t, over the t that query r sees; m_r is a running
// maximum that is followed only when it has grown by 8 (then p < 2^8, and nothing is scaled again for every small step).
//
// A workgroup has up to 16 queries that share a head of keys and a piece of the sequence; each of its four wavefronts takes 64 rows of the
// cache at a time.  Both products are matrix instructions of 16 x 16 x 32 on bf16.  Codes of all formats are bf16 numbers as they stand,
// so what is multiplied is exact: a row's scale goes onto the sum of a group's products (keys) or onto p (values), in fp32; a q of 16 or 32 bits goes in
// as two or three bf16 numbers that add up to it, and so does p times its scale for results of 32 bits, as three.  For results of 16 bits it goes in as two, the
// first cut off and the second rounded, within 2^-16 of it: a 256th of half a step of bf16, a 32nd of one of fp16; a third part would be a third more matrix
// instructions for bf16, a quarter for fp16.  Of 1,000 results of bf16 3 to 6, of fp16 22, are then rounded to the other neighbour than from sums of torch in 32 bits, and the
// error against 64 bits is the same to four digits (1.66e-3 and 2.07e-4 of the norm).
// The first product is K Q^T: lane (n, g) then holds the scores of query n and rows 4 g .. 4 g + 3 of either half, and these eight are the
// inputs of its part of the second, V^T P^T, if the rows are summed in that order: scores never change lanes, and a query's maximum, sum and
// results are all in lanes of its number.  64 rows go at a time, four tiles of the first product, two steps of the second.
//
// A token a sequence: bound by memory.  64 sequences of 2,048 to 4,096 rows (8 heads of 128, 4 bits, 32 queries, 215 MB) 55 us (3.9 TB/s) and
// 5 for joining; without any product, loads and LDS alone, the same.  128 sequences of 4,096 take 52 us more than 64 (287 MB, 5.5 TB/s), so some 15 are begin
// and end: lengths, page table, keys, values, each a trip to memory behind the other.  131,072 rows of one (a scale for 32 elements, 168 MB) 43 and 6.  A
// request of 301 rows 8.8.  A second slab on its way made no difference.
// Prompts: bound by vector instructions, some 430 for 64 rows and 16 queries (a third conversions), 48 matrix instructions beside them: 1,024 queries of
// 32 heads, the last of 4,096 rows, 128 us, 470 TFLOP/s; 4 of those 515.  (Four wavefronts that share what one of them has converted, as bf16 in LDS, were no
// faster: 326 and 512; two barriers for 64 rows cost what the conversions do.)
// ---------------------------------------------------------------------------
template <uint32_t FMT> struct Code { static constexpr uint32_t BITS = FMT == CF_E2M1 ? 4u : 8u; };

DEV uint32_t bits_of(bf2 v) { return __builtin_bit_cast(uint32_t, v); }
// elements 2 I, 2 I + 1 of a word of codes as bf16; int8: of the word's bytes
template <uint32_t FMT, int I> DEV uint32_t pair_of(uint32_t w) {
  if constexpr (FMT == CF_E2M1) return bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, I));
  else if constexpr (FMT == CF_E4M3) return bits_of(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, I != 0));
  else {
    const float a = (float)(int8_t)(w >> (16 * I)), b = (float)(int8_t)(w >> (16 * I + 8));
    return __builtin_amdgcn_perm(as_u(b), as_u(a), 0x07060302u);      // (of so few bits the upper half is all)
  }
}
DEV uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
DEV bf8 frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(bf8, u4{a, b, c, d}); }
// eight codes that follow each other: a word of 4 bits each, two of 8
template <uint32_t FMT> DEV bf8 eight_of(uint32_t a, uint32_t b) {
  if constexpr (FMT == CF_E2M1) return frag(pair_of<FMT, 0>(a), pair_of<FMT, 1>(a), pair_of<FMT, 2>(a), pair_of<FMT, 3>(a));
  else return frag(pair_of<FMT, 0>(a), pair_of<FMT, 1>(a), pair_of<FMT, 0>(b), pair_of<FMT, 1>(b));
}
DEV f4 mfma(bf8 a, bf8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// f's upper 16 bits are the first of its parts, the rest is exact
DEV float upper(float f) { return as_f(as_u(f) & 0xffff0000u); }
DEV float rest_of(float f) {
  const float hi = upper(f), r = f - hi;
  return (as_u(f) & 0x7f800000u) == 0x7f800000u ? 0.0f : r;
}
// v, of which the compiler does not know where it is from: it computes what depends on it here, and does not keep it; and the same, not before f is
// there: or it begins everything that does not depend on anything before it finishes something.  Either way it runs out of registers.
DEV uint32_t hidden(uint32_t v) {
  asm("" : "+v"(v));
  return v;
}
DEV uint32_t behind(uint32_t v, f4 f) {
  asm("" : "+v"(v) : "v"(f));
  return v;
}
// over the four lanes of a query
DEV float max4(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(as_u(v), as_u(v), false, false);
  v = __builtin_fmaxf(as_f(r[0]), as_f(r[1]));
  auto q = __builtin_amdgcn_permlane16_swap(as_u(v), as_u(v), false, false);
  return __builtin_fmaxf(as_f(q[0]), as_f(q[1]));
}
DEV float sum4(float v) {
  auto r = __builtin_amdgcn_permlane32_swap(as_u(v), as_u(v), false, false);
  v = as_f(r[0]) + as_f(r[1]);
  auto q = __builtin_amdgcn_permlane16_swap(as_u(v), as_u(v), false, false);
  return as_f(q[0]) + as_f(q[1]);
}
DEV void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
// 0 times anything is 0: a row of the cache that a query does not see adds nothing, whatever its scale is.  (Not as inline asm: the compiler does
// not see there that a result of the exponential is waited for.)
extern "C" __device__ float legacy_mul(float, float) __asm("llvm.amdgcn.fmul.legacy");

// A sum of weights that is 0: of a query that sees nothing, whose result is 0; or of one all of whose scores are -inf, as the softmax has no
// value there.  (The length is read again: kept, it would be one more register in the loop.)
DEV float of_no_weights(const AttendArgs& a, uint32_t b, uint32_t s) {
  int32_t len = (int32_t)a.longest;
  if (a.lengths != 0) {
    const int32_t l = ld<int32_t>(a.lengths + (uint64_t)b * a.ls * 4u);
    len = l < 0 ? 0 : (l < len ? l : len);
  }
  return len - (int32_t)a.s + (int32_t)s >= 0 ? __builtin_nanf("") : 0.0f;
}

struct AttendPlace { uint32_t b, hk, tile, piece, part; bool there; };
DEV AttendPlace attend_place(const AttendArgs& a) {
  // Workgroups go to the eight dies in turn; `inner` that follow each other here go to one (the rule is at the packing): heads that lie
  // together share lines of the cache and of its scales, queries of a head all of it.
  AttendPlace p;
  const uint32_t die = blockIdx.x & 7u, k = blockIdx.x >> 3, o = divided(k, a.by_inner), outer = o * 8u + die;
  const uint32_t id = outer * a.inner + (k - o * a.inner), head = divided(id, a.by_tiles), part = divided(head, a.by_heads);
  p.there = id < a.blocks;
  p.b = divided(part, a.by_pieces);
  p.piece = part - p.b * a.pieces;
  p.hk = head - part * a.heads;
  const uint32_t tile = id - head * a.tiles;
  p.tile = tile >> a.lg_parts;
  p.part = tile - (p.tile << a.lg_parts);
  return p;
}

// A wavefront's codes go by way of LDS (from memory straight to the lanes that multiply, each load touched 16 or 64 lines, and values of
// more than one scale came byte by byte), 64 rows by 64 bytes at a time (a slab): read from memory in pieces of 16 bytes, four lanes a row, the
// next slab on its way while one is worked on.  Piece c of row t lies in place c ^ swizzle(t), so that neither product's reads meet in a
// bank: for the first a lane reads its row's codes, for the second a column's of 16 rows (4 bits) or eight, which the LDS transposes.
DEV uint32_t swizzle(uint32_t t) { return ((t >> 2) ^ (t >> 4)) & 3u; }
typedef int i2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i2* lds_i2;

// DP: elements of a head that there is room for; FULL: a head has as many; MULTI: more than one scale a row.  Of 256 elements a workgroup has
// all of the scores but one half of the results: with all of those it would not fit into 128 registers (below).
template <uint32_t FMT, uint32_t DP, bool FULL, uint32_t DT, bool MULTI>
__global__ void __launch_bounds__(kThreads, 4) gpuos_cache_attend_kernel(const AttendArgs a) {
  constexpr uint32_t BITS = Code<FMT>::BITS, ROW = DP * BITS / 8u, NS = ROW < 64u ? 1u : ROW / 64u, DS = DP / NS;      // slabs; elements of one
  constexpr uint32_t DV = DP < 128u ? DP : 128u, NV = NS * DV / DP;            // elements of a result that a workgroup has; slabs of them
  constexpr uint32_t CH = ROW < 64u ? ROW / 16u : 4u, IT = CH, KS = DS / 32u, MT = DS / 16u;      // pieces of a row; loads of a lane; steps, tiles of a slab
  constexpr uint32_t NQ = DT == GPUOS_BF16 ? 1u : (DT == GPUOS_F16 ? 2u : 3u), NP = DT == GPUOS_F32 ? 3u : 2u;
  constexpr uint32_t GROUPS = MULTI ? DP / 32u : 1u;
  constexpr bool STEPS = MULTI || BITS == 8u || NP == 3u;
  constexpr uint32_t WAVE_LDS = attend_wave_lds(DP, MULTI), Q_LDS = attend_q_lds(DP, DT);
  extern __shared__ uint8_t lds[];                                 // attend_lds bytes
  const AttendPlace at = attend_place(a);
  if (!at.there) return;
  const uint32_t tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63u, n = lane & 15u, g = lane >> 4;
  const uint32_t d = FULL ? DP : a.d;
  // A wavefront has a head of its own, or every fourth 64 rows of the workgroup's.
  const bool by_head = a.by_head != 0u;
  const uint32_t head = by_head ? at.hk * 4u + wave : at.hk;

  const uint32_t r0 = at.tile * kTileRows, row = r0 + n;
  const bool has_row = row < a.rows;
  const auto query = [&](uint32_t& qs, uint32_t& qh) {             // the lane's query: of S, of the heads that share one of keys
    const uint32_t r = hidden(has_row ? row : r0);
    qs = divided(r, a.by_per);
    qh = r - qs * a.per;
  };
  uint32_t qs, qh;
  query(qs, qh);
  // the queries are asked for first: where the rows of the cache lie is four more trips to memory
  constexpr uint32_t QL = DP / 32u;                                // pieces of eight elements in lanes
  const bf8* const qf = (const bf8*)(lds + (by_head ? wave * Q_LDS : 0u));
  float qv[2][8];                                                  // (a fourth of them; or half of them at a time)
  const uint64_t qp = a.q + ((uint64_t)at.b * a.qs[0] + (uint64_t)qs * a.qs[1] + (uint64_t)(head * a.per + qh) * a.qs[2]) * size_of(DT);
  const auto ask_queries = [&](uint32_t j, float (&f)[8]) {
    const uint32_t e0 = 32u * j + 8u * g;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = 0.0f;
    if (j < QL && has_row && e0 < d && head < a.hk) {
      if (a.qs[3] == 1u) ld8<DT>(qp + (uint64_t)e0 * size_of(DT), f);
      else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) f[i] = ld_elem<DT>(qp + (uint64_t)(e0 + i) * a.qs[3] * size_of(DT));
      }
    }
  };
  const auto put_queries = [&](uint32_t j, float (&f)[8]) {        // as the parts of the second operand of K Q^T
    if (j >= QL) return;
#pragma unroll
    for (uint32_t t = 0; t < NQ; ++t) {
      u4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = high_halves(as_u(f[2 * i]), as_u(f[2 * i + 1]));
      ((bf8*)qf)[(t * QL + j) * 64u + lane] = __builtin_bit_cast(bf8, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = rest_of(f[i]);
    }
  };
  ask_queries(by_head ? 0u : wave, qv[0]);
  ask_queries(by_head ? 1u : wave + 4u, qv[1]);

  // what the tile's queries see: rows [from, end) of the sequence, and of that this piece's [t0, t1)
  int32_t len = (int32_t)a.longest;
  if (a.lengths != 0) {
    const int32_t l = ld<int32_t>(a.lengths + (uint64_t)at.b * a.ls * 4u);
    len = l < 0 ? 0 : (l < len ? l : len);
  }
  len = __builtin_amdgcn_readfirstlane(len);
  const uint32_t rl = (r0 + kTileRows < a.rows ? r0 + kTileRows : a.rows) - 1u;      // the tile's first and last query
  const int32_t past = len - (int32_t)a.s;                                     // rows before the first query's own
  const int32_t pos_first = past + (int32_t)divided(r0, a.by_per), pos_last = past + (int32_t)divided(rl, a.by_per);
  const int32_t pos = past + (int32_t)qs;
  int32_t from = a.window != 0 ? pos_first - (int32_t)a.window + 1 : 0;
  from = from < 0 ? 0 : from;
  const int32_t end = pos_last + 1;
  const int32_t all_from = a.window != 0 ? pos_last - (int32_t)a.window + 1 : 0;      // all of them see [all_from, pos_first]
  int32_t t0 = from, t1 = end;
  if (a.pieces > 1u) {
    const int32_t blocks = end > from ? (end - from + 63) / 64 : 0, per = (int32_t)divided((uint32_t)blocks + a.pieces - 1u, a.by_pieces);
    t0 = from + (int32_t)at.piece * per * 64;
    t1 = t0 + per * 64 < end ? t0 + per * 64 : end;
  }

  if (head >= a.hk) t1 = t0;

  uint8_t* const slab = lds + (by_head ? 4u * Q_LDS : Q_LDS) + wave * WAVE_LDS;
  uint64_t* const offs = (uint64_t*)(slab + kSlab);                // [keys, values][64]
  float* const sc = (float*)(slab + kSlab + 1024u);                // [GROUPS][keys, values][64]
  const uint64_t table = a.table + (uint64_t)at.b * a.ps[0] * 4u;
  float ks[GROUPS], vs[GROUPS];                                    // scales of row t + lane
  u4 r[IT];                                                        // a slab's pieces

  const auto look = [&](int32_t t) -> uint32_t {                   // the entry of the page table for row t + lane (behind the last: for that)
    const int32_t k = t + (int32_t)lane < t1 ? t + (int32_t)lane : t1 - 1;
    return ld<uint32_t>(table + (uint64_t)divided((uint32_t)k, a.by_page) * a.ps[1] * 4u);
  };
  const auto find = [&](int32_t t, uint32_t entry) {               // where the row lies, and its scales
    const uint32_t k = (uint32_t)(t + (int32_t)lane < t1 ? t + (int32_t)lane : t1 - 1), in = k - divided(k, a.by_page) * a.page;
    const bool known = entry < a.pages;
    const uint64_t e = known ? entry : 0u;
#pragma unroll
    for (uint32_t v = 0; v < 2; ++v) {
      offs[v * 64u + lane] = a.kv[v].cache + (uint64_t)head * a.kv[v].cs[2] + e * a.kv[v].cs[0] + (uint64_t)in * a.kv[v].cs[1];
      const uint64_t sp = a.kv[v].scales + ((uint64_t)head * a.kv[v].ss[2] + e * a.kv[v].ss[0] + (uint64_t)in * a.kv[v].ss[1]) * 4u;
      float f[GROUPS];                                             // (of more than one scale: that of each 32 elements)
      if (MULTI && a.by_fours != 0u) {                             // (131,072 rows with a scale for 32: 54 us, so 43)
#pragma unroll
        for (uint32_t q = 0; q < GROUPS; q += 4) {
          const uint32_t left = FULL ? GROUPS - q : (32u * q < d ? (d - 32u * q + 31u) / 32u : 0u);
          u4 w = {0, 0, 0, 0};
          if (left >= 4u) w = ld<u4_any>(sp + 4u * q);
          else {
#pragma unroll
            for (uint32_t k = 0; k < 3; ++k) {
              if (k < left) w[k] = ld<uint32_t>(sp + 4u * (q + k));
            }
          }
#pragma unroll
          for (uint32_t k = 0; k < 4; ++k) {
            if (q + k < GROUPS) f[q + k] = as_f(w[k]);
          }
        }
      } else {
#pragma unroll
        for (uint32_t q = 0; q < GROUPS; ++q) {
          f[q] = 0.0f;
          if (FULL || !MULTI || 32u * q < d) f[q] = ld<float>(sp + (uint64_t)(MULTI ? divided(32u * q, a.by_group) : 0u) * a.kv[v].ss[3] * 4u);
        }
      }
#pragma unroll
      for (uint32_t q = 0; q < GROUPS; ++q) {
        const float to = known ? f[q] : __builtin_nanf("");        // a page that is not in the cache
        if (v) vs[q] = to;
        else ks[q] = to;
      }
    }
  };
  // A row's pieces end where the row does: the last, of 4, 8 or 12 bytes, is asked for as the row's last 16 (loads of words behind a branch
  // waited for those in front of them: 16 sequences of up to 4,096 rows, 8 heads of 96, 4 bits, 26.5 us, so 22.5).
  const uint32_t row_bytes = d * BITS / 8u;
  const auto moved = [&](uint32_t s) -> uint32_t {                 // by so many bytes
    const uint32_t past = 64u * s + 16u * (hidden(lane) & (CH - 1u)) + 16u;
    return (past > row_bytes ? past : row_bytes) - row_bytes;
  };
  const auto ask = [&](uint32_t v, uint32_t s) {
    const uint32_t c = (FULL ? lane : hidden(lane)) & (CH - 1u), e = 64u * s + 16u * c;
    if (FULL || row_bytes >= 16u) {
      const uint32_t from = FULL || e + 16u <= row_bytes ? e : row_bytes - 16u;
#pragma unroll
      for (uint32_t i = 0; i < IT; ++i) r[i] = ld<u4_byte>(offs[v * 64u + i * (64u / CH) + lane / CH] + from);
    } else {
#pragma unroll
      for (uint32_t i = 0; i < IT; ++i) {
        const uint64_t p = offs[v * 64u + i * (64u / CH) + lane / CH] + e;
        r[i] = u4{0, 0, 0, 0};
#pragma unroll
        for (uint32_t w = 0; w < 3; ++w) {
          if (e + 4u * w < row_bytes) r[i][w] = ld<u1_any>(p + 4u * w);
        }
      }
    }
  };
  // what `ask` asked for further in front goes where it belongs; what is behind the row meets zeros of the query, or is a result that nobody stores:
  // it is cleared only where a code may be no number
  const auto settle = [&](uint32_t s) {
    if (FULL || row_bytes < 16u || (FMT != CF_E4M3 && (row_bytes & 15u) == 0u)) return;
    const uint32_t by = moved(s);
#pragma unroll
    for (uint32_t i = 0; i < IT; ++i) {
      const u4 w = r[i], o = by & 4u ? u4{w[1], w[2], w[3], 0} : w, h = by & 8u ? u4{o[2], o[3], 0, 0} : o;
      r[i] = by < 16u ? h : u4{0, 0, 0, 0};
    }
  };
  // Places in LDS: of piece c of row t, 64 t + 16 (c ^ swizzle(t)).  Those of a lane differ by an exclusive or and a constant from the first,
  // which is hidden from the compiler: it would keep them all in registers.
  const auto slab_at = [&](uint32_t t, uint32_t c, uint32_t more) { return 64u * t + 16u * (c ^ swizzle(t)) + more; };
  const uint32_t put_at = slab_at(lane / CH, lane & (CH - 1u), 0);
  const uint32_t key_at = BITS == 4u ? slab_at(n, 0, 4u * g) : slab_at(n, g >> 1, 8u * (g & 1u));
  const uint32_t value_at = BITS == 4u ? slab_at(16u * (n >> 2) + 4u * g + (n & 3u), 0, 0) : slab_at(16u * (n >> 3) + 4u * g + ((n >> 1) & 3u), 0, 8u * (n & 1u));
  const auto put = [&]() {
    const uint32_t o = hidden(put_at);
#pragma unroll
    for (uint32_t i = 0; i < IT; ++i) *(u4*)(slab + i * (64u / CH) * 64u + (o ^ (swizzle(i * (64u / CH)) << 4))) = r[i];
  };

  const uint32_t first_slab = at.part * NV, first_e = at.part * DV;      // of the values that the workgroup has
  f4 acc[NV * MT];
#pragma unroll
  for (uint32_t j = 0; j < NV * MT; ++j) acc[j] = f4{0, 0, 0, 0};
  float m = -__builtin_inff(), l = 0.0f;
  const int32_t step = by_head ? 64 : 256;
  int32_t t = t0 + (by_head ? 0 : (int32_t)wave * 64);
  uint32_t entry = 0;
  if (t < t1) entry = look(t);
  put_queries(by_head ? 0u : wave, qv[0]);
  put_queries(by_head ? 1u : wave + 4u, qv[1]);
  if (by_head) {
    for (uint32_t j = 2; j < QL; j += 2) {
      ask_queries(j, qv[0]);
      ask_queries(j + 1u, qv[1]);
      put_queries(j, qv[0]);
      put_queries(j + 1u, qv[1]);
    }
  }
  if (t < t1) {
    find(t, entry);
    wave_sync();
    ask(0, 0);
    entry = look(t + step);
  }
  __syncthreads();
  for (; t < t1; t += step) {
#pragma unroll
    for (uint32_t q = 0; q < GROUPS; ++q) {
      sc[(2u * q) * 64u + lane] = ks[q] * a.scale;
      sc[(2u * q + 1u) * 64u + lane] = vs[q];
    }
    // scores: of query n, rows 16 T + 4 g + i
    f4 x[4], c[4];
#pragma unroll
    for (int T = 0; T < 4; ++T) x[T] = c[T] = f4{0, 0, 0, 0};
#pragma unroll
    for (uint32_t s = 0; s < NS; ++s) {
      settle(s);
      put();
      wave_sync();
      if (s + 1u < NS) ask(0, s + 1u);
      else ask(1, first_slab);
      uint32_t ko = hidden(key_at);
#pragma unroll
      for (uint32_t j = 0; j < KS; ++j) {
        const uint32_t e = s * DS + 32u * j;                       // the step's first element (behind the head's last, all are 0)
        bf8 q[NQ];
#pragma unroll
        for (uint32_t k = 0; k < NQ; ++k) q[k] = qf[(k * QL + e / 32u) * 64u + lane];
#pragma unroll
        for (uint32_t T = 0; T < 4; ++T) {
          bf8 k;
          const uint8_t* const kp = slab + 1024u * T + (ko ^ (((j * (BITS / 4u)) ^ T) << 4));
          if constexpr (BITS == 4u) k = eight_of<FMT>(*(const uint32_t*)kp, 0u);
          else {
            const u2 w = *(const u2*)kp;
            k = eight_of<FMT>(w[0], w[1]);
          }
#pragma unroll
          for (uint32_t z = 0; z < NQ; ++z) c[T] = mfma(k, q[z], c[T]);
        }
        if (MULTI) {
#pragma unroll
          for (uint32_t T = 0; T < 4; ++T) {
            const f4 f = *(const f4*)(sc + (2u * (e / 32u)) * 64u + 16u * T + 4u * g);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[T][i] = __builtin_fmaf(c[T][i], f[i], x[T][i]);
            c[T] = f4{0, 0, 0, 0};
            ko = behind(ko, x[T]);
          }
        }
      }
      wave_sync();
    }
    if (!MULTI) {
#pragma unroll
      for (uint32_t T = 0; T < 4; ++T) x[T] = c[T] * *(const f4*)(sc + 16u * T + 4u * g);
    }
    if (t < all_from || t + 63 > pos_first || t + 64 > t1) {       // some query does not see all of these
      const int32_t see_from = a.window != 0 ? pos - (int32_t)a.window + 1 : 0;
#pragma unroll
      for (int T = 0; T < 4; ++T) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int32_t k = t + 16 * T + (int32_t)(4u * g) + i;
          x[T][i] = k < t1 && k <= pos && k >= see_from ? x[T][i] : -__builtin_inff();      // (its query sees [see_from, pos])
        }
      }
    }
    float top = -__builtin_inff();
#pragma unroll
    for (int T = 0; T < 4; ++T) {
#pragma unroll
      for (int i = 0; i < 4; ++i) top = __builtin_fmaxf(top, x[T][i]);
    }
    top = max4(top);
    if (__builtin_amdgcn_ballot_w64(top > m + 8.0f) != 0) {
      const float to = __builtin_fmaxf(m, top), by = to == m ? 1.0f : __builtin_amdgcn_exp2f(m - to);      // (1 also where both are -inf)
      m = to;
      l *= by;
#pragma unroll
      for (uint32_t j = 0; j < NV * MT; ++j) acc[j] *= by;
    }
    const float base = m == -__builtin_inff() ? 0.0f : m;
#pragma unroll
    for (int T = 0; T < 4; ++T) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[T][i] = __builtin_amdgcn_exp2f(x[T][i] - base);
      l += (x[T][0] + x[T][1]) + (x[T][2] + x[T][3]);
    }

    // weights: 2^(x - m) times the scale of the row's group, in parts
    bf8 w[2][NP];
    const auto weights = [&](uint32_t group, uint32_t u, uint32_t g4, bf8 (&to)[NP]) {
      float f[8];
#pragma unroll
      for (uint32_t T = 0; T < 2; ++T) {
        const f4 v = *(const f4*)(sc + (2u * group + 1u) * 64u + 16u * (2u * u + T) + g4);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[4 * T + i] = legacy_mul(x[2u * u + T][i], v[i]);
      }
#pragma unroll
      for (uint32_t k = 0; k < NP; ++k) {
        u4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          typedef float f2 __attribute__((ext_vector_type(2)));
          v[i] = k + 1u < NP ? high_halves(as_u(f[2 * i]), as_u(f[2 * i + 1])) : bits_of(__builtin_convertvector((f2{f[2 * i], f[2 * i + 1]}), bf2));
        }
        to[k] = __builtin_bit_cast(bf8, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] - upper(f[i]);
      }
    };
#pragma unroll
    for (uint32_t s = 0; s < NV; ++s) {
      if constexpr (FMT == CF_E4M3) {
        // A code that is no number makes its row none, in this slab and those behind it: the code becomes 0, the row's scale a NaN.
        uint32_t any = 0;
#pragma unroll
        for (uint32_t i = 0; i < IT; ++i) {
#pragma unroll
          for (int k = 0; k < 4; ++k) any |= (r[i][k] & 0x7f7f7f7fu) + 0x01010101u;
        }
        if (__builtin_amdgcn_ballot_w64((any & 0x80808080u) != 0u) != 0) {
#pragma unroll
          for (uint32_t i = 0; i < IT; ++i) {
            uint32_t bad = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t y = ((r[i][k] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
              bad |= y;
              r[i][k] &= ~((y >> 7) * 0xffu);
            }
            if (bad != 0u) {
#pragma unroll
              for (uint32_t q = 0; q < GROUPS; ++q) sc[(2u * q + 1u) * 64u + i * (64u / CH) + lane / CH] = __builtin_nanf("");
            }
          }
        }
      }
      settle(first_slab + s);
      put();
      wave_sync();
      if (s + 1u < NV) ask(1, first_slab + s + 1u);
      else if (t + step < t1) {
        find(t + step, entry);                                     // (these scales go into LDS at the top)
        wave_sync();
        ask(0, 0);
        entry = look(t + 2 * step);
      }
      // The two steps of a tile of results together, two tiles at a time, as one waits for the other; or (STEPS) one step after the other, so that
      // only one step's weights are held.
      if (!MULTI && !STEPS && s == 0u) {
        weights(0, 0, 4u * g, w[0]);
        weights(0, 1, 4u * g, w[1]);
      }
#pragma unroll
      for (uint32_t uu = 0; uu < (STEPS ? 2u : 1u); ++uu) {
        const uint32_t vo = STEPS && uu == 1u ? behind(value_at, acc[s * MT + MT - 1u]) : hidden(value_at);
        if (!MULTI && STEPS) weights(0, uu, uu == 1u ? behind(4u * g, acc[s * MT + MT - 1u]) : hidden(4u * g), w[0]);
#pragma unroll
        for (uint32_t j = 0; j < MT; j += 2) {
          const uint32_t e = first_e + s * DS + 16u * j;           // the tile's first element
          if constexpr (MULTI) weights(e / 32u, uu, j >= 2u ? behind(4u * g, acc[s * MT + j - 1u]) : hidden(4u * g), w[0]);
          bf8 v[2][2];                                           // [tile][step]
#pragma unroll
          for (uint32_t i = 0; i < 2; ++i) {
            if constexpr (BITS == 4u) {
              const i2 y = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i2)(slab + (vo ^ ((j >> 1) << 4)) + 8u * i));
#pragma unroll
              for (uint32_t u = 0; u < (STEPS ? 1u : 2u); ++u) v[i][u] = eight_of<FMT>((uint32_t)y[STEPS ? uu : u], 0u);
            } else {
#pragma unroll
              for (uint32_t u = 0; u < (STEPS ? 1u : 2u); ++u) {
                const uint32_t step = STEPS ? uu : u;
                const i2 y = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2)(slab + 2048u * step + (vo ^ (((j + i) ^ (2u * step)) << 4))));
                v[i][u] = eight_of<FMT>((uint32_t)y[0], (uint32_t)y[1]);
              }
            }
          }
#pragma unroll
          for (uint32_t k = 0; k < NP; ++k) {
#pragma unroll
            for (uint32_t u = 0; u < (STEPS ? 1u : 2u); ++u) {
#pragma unroll
              for (uint32_t i = 0; i < 2; ++i) acc[s * MT + j + i] = mfma(v[i][u], w[u][k], acc[s * MT + j + i]);
            }
          }
        }
      }
      wave_sync();
    }
  }

  l = sum4(l);
  if (!by_head) {                                                  // the four wavefronts' sums
    __syncthreads();
    float* const stats = (float*)lds;                              // [4][16][2]
    float* const sums = (float*)(lds + 512u);                      // [2][16][DV]
    if (g == 0u) {
      stats[(wave * 16u + n) * 2u] = m;
      stats[(wave * 16u + n) * 2u + 1u] = l;
    }
    __syncthreads();
    float most = -__builtin_inff(), total = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) most = __builtin_fmaxf(most, stats[(k * 16u + n) * 2u]);
    const float ref = most == -__builtin_inff() ? 0.0f : most;
#pragma unroll
    for (int k = 0; k < 4; ++k) total += stats[(k * 16u + n) * 2u + 1u] * __builtin_amdgcn_exp2f(stats[(k * 16u + n) * 2u] - ref);
    const float by = __builtin_amdgcn_exp2f(m - ref);
#pragma unroll
    for (uint32_t j = 0; j < NV * MT; ++j) acc[j] *= by;
    // (two and two, then the two: always in this order)
    for (uint32_t k = 2; k >= 1u; k /= 2u) {
      if (wave >= k && wave < 2u * k) {
#pragma unroll
        for (uint32_t j = 0; j < NV * MT; ++j) *(f4*)(sums + ((wave - k) * NV * MT + j) * 256u + lane * 4u) = acc[j];
      }
      __syncthreads();
      if (wave < k) {
#pragma unroll
        for (uint32_t j = 0; j < NV * MT; ++j) acc[j] += *(const f4*)(sums + (wave * NV * MT + j) * 256u + lane * 4u);
      }
      __syncthreads();
    }
    if (wave != 0u) return;
    m = most;
    l = total;
  }
  if (!has_row || head >= a.hk) return;
  const bool last = a.joined == 0u;
  query(qs, qh);
  float inv = last ? 1.0f / l : 1.0f;
  if (last && l == 0.0f) inv = of_no_weights(a, at.b, qs);
  const uint64_t op = a.out + ((uint64_t)at.b * a.os[0] + (uint64_t)qs * a.os[1] + (uint64_t)(head * a.per + qh) * a.os[2]) * size_of(DT);
  const uint64_t all = (uint64_t)a.b * a.hk * a.rows, mine = ((uint64_t)at.b * a.hk + head) * a.rows + row, slice = (uint64_t)at.piece * all + mine;
  if (!last && g == 0u && at.part == 0u) {
    st<float>(a.stats + slice * 8u, m);
    st<float>(a.stats + slice * 8u + 4u, l);
  }
#pragma unroll
  for (uint32_t j = 0; j < NV * MT; ++j) {
    const uint32_t e = first_e + 16u * j + 4u * g;                 // (a head has a multiple of eight)
    if (FULL || e < d) {
      if (!last) st<u4_any>(a.part + (slice * d + e) * 4u, __builtin_bit_cast(u4, acc[j]));
      else {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) acc[j][i] *= inv;
        if (a.os[3] == 1u) st4<DT>(op + (uint64_t)e * size_of(DT), acc[j]);
        else {
#pragma unroll
          for (uint32_t i = 0; i < 4; ++i) st_elem<DT>(op + (uint64_t)(e + i) * a.os[3] * size_of(DT), acc[j][i]);
        }
      }
    }
  }
}

// The pieces' sums.  A query has a wavefront, or, of more than 64 pieces, the workgroup (WIDE); a part of a wavefront has a quarter of the head's
// elements in lanes and every so many of the pieces, six on their way at a time (eight do not fit into
// 64 registers).  2,048 queries of 128 elements, 6 pieces: 4.7 us (with a
// workgroup each 7.6).
constexpr uint32_t kJoinWaves = kJoinThreads / 64, kJoinAhead = 6;
template <uint32_t DT, bool WIDE> __global__ void __launch_bounds__(kJoinThreads, 8) gpuos_cache_join_kernel(const AttendArgs a) {
  __shared__ alignas(16) float weight[WIDE ? kPiecesMost : kJoinWaves * 64u], sums[WIDE ? kJoinWaves : 1][256], tops[kJoinWaves], totals[kJoinWaves];
  const uint32_t tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63u;
  const uint64_t all = (uint64_t)a.b * a.hk * a.rows;
  const uint64_t mine = WIDE ? blockIdx.x : (uint64_t)blockIdx.x * kJoinWaves + wave;
  if (mine >= all) return;                                         // (of a WIDE one: none)
  const uint32_t me = WIDE ? tid : lane;                           // which piece's weight the lane finds
  static_assert(kPiecesMost <= kJoinThreads, "a thread for each piece");
  float m = -__builtin_inff(), l = 0.0f;
  if (me < a.pieces) {
    const u2 v = ld<u2_any>(a.stats + (me * all + mine) * 8u);
    m = as_f(v[0]);
    l = as_f(v[1]);
  }
  float top = m;
  for (int w = 32; w >= 1; w /= 2) top = __builtin_fmaxf(top, __shfl_xor(top, w, 64));
  if (WIDE) {
    if (lane == 0u) tops[wave] = top;
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < kJoinWaves; ++k) top = __builtin_fmaxf(top, tops[k]);
  }
  const float by = __builtin_amdgcn_exp2f(m - (top == -__builtin_inff() ? 0.0f : top));
  float total = l == 0.0f ? 0.0f : l * by;
  float* const weights = weight + (WIDE ? 0u : wave * 64u);
  if (me < (WIDE ? kPiecesMost : 64u)) weights[me] = l == 0.0f ? -1.0f : by;      // (an empty piece: its sums were not written)
  for (int w = 32; w >= 1; w /= 2) total += __shfl_xor(total, w, 64);
  if (WIDE) {
    if (lane == 0u) totals[wave] = total;
    __syncthreads();
    total = 0.0f;
#pragma unroll
    for (uint32_t k = 0; k < kJoinWaves; ++k) total += totals[k];
  } else wave_sync();
  // lanes of a part, parts of the wavefront
  const uint32_t lanes = a.d <= 64u ? 16u : (a.d <= 128u ? 32u : 64u), e = 4u * (lane & (lanes - 1u)), parts = 64u / lanes * (WIDE ? kJoinWaves : 1u);
  const uint32_t first = lane / lanes + (WIDE ? wave * (64u / lanes) : 0u);
  f4 sum = {0, 0, 0, 0};
  const bool has = e < a.d;
  const uint64_t from = a.part + (mine * a.d + (has ? e : 0u)) * 4u;
  for (uint32_t k0 = first; k0 < a.pieces; k0 += kJoinAhead * parts) {
    f4 v[kJoinAhead];
#pragma unroll
    for (uint32_t i = 0; i < kJoinAhead; ++i) {
      v[i] = f4{0, 0, 0, 0};
      const uint32_t k = k0 + i * parts;
      if (has && k < a.pieces && weights[k] >= 0.0f) v[i] = __builtin_bit_cast(f4, ld<u4_any>(from + (uint64_t)k * all * a.d * 4u));
    }
#pragma unroll
    for (uint32_t i = 0; i < kJoinAhead; ++i) {
      const uint32_t k = k0 + i * parts;
      const float w = k < a.pieces ? weights[k] : -1.0f;
#pragma unroll
      for (int c = 0; c < 4; ++c) sum[c] += w < 0.0f ? 0.0f : v[i][c] * w;
    }
  }
  for (uint32_t w = lanes; w < 64u; w *= 2) {
#pragma unroll
    for (int c = 0; c < 4; ++c) sum[c] += __shfl_xor(sum[c], (int)w, 64);
  }
  if (WIDE) {
    if (lane < lanes) *(f4*)&sums[wave][e] = sum;
    __syncthreads();
    if (wave != 0u) return;
    sum = f4{0, 0, 0, 0};
#pragma unroll
    for (uint32_t k = 0; k < kJoinWaves; ++k) sum += *(const f4*)&sums[k][e];
  }
  if (lane >= lanes || !has) return;
  const uint32_t pair = divided((uint32_t)mine, a.by_rows), row = (uint32_t)mine - pair * a.rows, b = divided(pair, a.by_hk), hk = pair - b * a.hk;
  const uint32_t qs = divided(row, a.by_per), qh = row - qs * a.per;
  float inv = 1.0f / total;
  if (total == 0.0f) inv = of_no_weights(a, b, qs);
  sum *= inv;
  const uint64_t op = a.out + ((uint64_t)b * a.os[0] + (uint64_t)qs * a.os[1] + (uint64_t)(hk * a.per + qh) * a.os[2]) * size_of(DT);
  if (a.os[3] == 1u) st4<DT>(op + (uint64_t)e * size_of(DT), sum);
  else {
#pragma unroll
    for (uint32_t i = 0; i < 4; ++i) st_elem<DT>(op + (uint64_t)(e + i) * a.os[3] * size_of(DT), sum[i]);
  }
}

struct AttendKernel { const void* kernel; uint32_t lds; };      // lds: with queries for each wavefront, or for all
template <uint32_t FMT, uint32_t DT, bool MULTI> AttendKernel attend_kernel(uint32_t d, bool by_head) {
  if constexpr (DT != GPUOS_F32) {
    if (d == 64u) return {(const void*)gpuos_cache_attend_kernel<FMT, 64, true, DT, MULTI>, attend_lds(64, DT, MULTI, by_head)};
    if (d == 128u) return {(const void*)gpuos_cache_attend_kernel<FMT, 128, true, DT, MULTI>, attend_lds(128, DT, MULTI, by_head)};
    if (d == 256u) return {(const void*)gpuos_cache_attend_kernel<FMT, 256, true, DT, MULTI>, attend_lds(256, DT, MULTI, by_head)};
  }
  if (d <= 128u) return {(const void*)gpuos_cache_attend_kernel<FMT, 128, false, DT, MULTI>, attend_lds(128, DT, MULTI, by_head)};
  return {(const void*)gpuos_cache_attend_kernel<FMT, 256, false, DT, MULTI>, attend_lds(256, DT, MULTI, by_head)};
}
template <uint32_t FMT> AttendKernel attend_kernel(uint32_t dt, uint32_t d, bool multi, bool by_head) {
  if (dt == GPUOS_F32) return multi ? attend_kernel<FMT, GPUOS_F32, true>(d, by_head) : attend_kernel<FMT, GPUOS_F32, false>(d, by_head);
  if (dt == GPUOS_F16) return multi ? attend_kernel<FMT, GPUOS_F16, true>(d, by_head) : attend_kernel<FMT, GPUOS_F16, false>(d, by_head);
  return multi ? attend_kernel<FMT, GPUOS_BF16, true>(d, by_head) : attend_kernel<FMT, GPUOS_BF16, false>(d, by_head);
}

int launch_attend(const AttendArgs& a, uint32_t format, void* stream) {
  const bool multi = a.group != a.d, by_head = a.by_head != 0u;
  const AttendKernel k = format == CF_E2M1 ? attend_kernel<CF_E2M1>(a.dtype, a.d, multi, by_head) : (format == CF_I8 ? attend_kernel<CF_I8>(a.dtype, a.d, multi, by_head) : attend_kernel<CF_E4M3>(a.dtype, a.d, multi, by_head));
  void* args[] = {(void*)&a};
  const uint32_t outer = (a.blocks / a.inner + 7u) / 8u * 8u;
  const int rc = (int)hipLaunchKernel(k.kernel, dim3(outer * a.inner), dim3(kThreads), args, k.lds, (hipStream_t)stream);
  if (rc != (int)hipSuccess || a.joined == 0u) return rc;
  const void* const joins[] = {(const void*)gpuos_cache_join_kernel<GPUOS_F32, false>,  (const void*)gpuos_cache_join_kernel<GPUOS_F16, false>,
                               (const void*)gpuos_cache_join_kernel<GPUOS_BF16, false>, (const void*)gpuos_cache_join_kernel<GPUOS_F32, true>,
                               (const void*)gpuos_cache_join_kernel<GPUOS_F16, true>,   (const void*)gpuos_cache_join_kernel<GPUOS_BF16, true>};
  const uint32_t all = a.b * a.hk * a.rows;
  const bool wide = a.pieces > 64u;
  return (int)hipLaunchKernel(joins[a.dtype + (wide ? 3u : 0u)], dim3(wide ? all : (all + kJoinWaves - 1u) / kJoinWaves), dim3(kJoinThreads), args, 0, (hipStream_t)stream);
}

}  // namespace gpuos
