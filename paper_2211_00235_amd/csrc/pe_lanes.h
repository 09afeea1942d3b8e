// Sums and maxima over groups of consecutive lanes on the vector unit (DPP and lane swaps; __shfl_xor goes through LDS), and
// vectors of V elements in fp32.
#pragma once
#include "pe_common.h"

template <int CTRL> PE_DEV uint32_t dpp_u(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
template <int CTRL> PE_DEV float dpp_f(float v) { return __uint_as_float(dpp_u<CTRL>(__float_as_uint(v))); }
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140;

// Sum over the L consecutive lanes that a lane belongs to (L a power of two, at most 64); every lane gets the same bits.
// Quads are level after two steps, so the mirrored lane of 8, then of 16, holds the other half's sum.
template <int L> PE_DEV float lanes_sum(float v) {
  if constexpr (L >= 2) v += dpp_f<DPP_XOR1>(v);
  if constexpr (L >= 4) v += dpp_f<DPP_XOR2>(v);
  if constexpr (L >= 8) v += dpp_f<DPP_HALF_MIRROR>(v);
  if constexpr (L >= 16) v += dpp_f<DPP_MIRROR>(v);
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}
// Sum over the lanes that are a multiple of L apart (the lanes of a wave that hold the same columns)
template <int L> PE_DEV float strided_sum(float v) {
  static_assert(L >= 4, "quads stay apart");
  if constexpr (L <= 4) v += __shfl_xor(v, 4, 64);
  if constexpr (L <= 8) v += __shfl_xor(v, 8, 64);
  if constexpr (L <= 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (L <= 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return v;
}
template <int L> PE_DEV uint32_t lanes_umax(uint32_t v) {
  static_assert(L <= 32, "groups of at most 32 lanes");
  if constexpr (L >= 2) v = max(v, dpp_u<DPP_XOR1>(v));
  if constexpr (L >= 4) v = max(v, dpp_u<DPP_XOR2>(v));
  if constexpr (L >= 8) v = max(v, dpp_u<DPP_HALF_MIRROR>(v));
  if constexpr (L >= 16) v = max(v, dpp_u<DPP_MIRROR>(v));
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max((uint32_t)r[0], (uint32_t)r[1]);
  }
  return v;
}

// V consecutive elements as they lie in memory.  raw_load / raw_store: 16-byte aligned addresses for V = 8.  The _any forms need the
// element's alignment only (global accesses of 16 bytes may start at any byte).
template <typename T, int V> struct Raw;
template <> struct Raw<bf16, 8> { bf16x8 v; PE_DEV float get(int i) const { return (float)v[i]; } PE_DEV void set(int i, float f) { v[i] = (bf16)f; } };
template <> struct Raw<bf16, 1> { bf16 v; PE_DEV float get(int) const { return (float)v; } PE_DEV void set(int, float f) { v = (bf16)f; } };
template <> struct Raw<float, 8> {
  f32x4 v[2];
  PE_DEV float get(int i) const { return v[i >> 2][i & 3]; }
  PE_DEV void set(int i, float f) { v[i >> 2][i & 3] = f; }
};
template <> struct Raw<float, 1> { float v; PE_DEV float get(int) const { return v; } PE_DEV void set(int, float f) { v = f; } };
// NT: a non-temporal load, for tensors that are read once and much larger than what the caches keep: lines that such a stream allocates push
// out what the kernels before have written, whose way to memory then stands in the stream's.
template <bool NT, typename U> PE_DEV U load_as(const U* p) {
  if constexpr (NT) return __builtin_nontemporal_load(p); else return *p;
}
template <typename T, int V, bool NT = false> PE_DEV Raw<T, V> raw_load(const T* p) {
  Raw<T, V> r;
  if constexpr (sizeof(Raw<T, V>) == 32) {
    r.v[0] = load_as<NT>(reinterpret_cast<const f32x4*>(p));
    r.v[1] = load_as<NT>(reinterpret_cast<const f32x4*>(p) + 1);
  } else {
    r.v = load_as<NT>(reinterpret_cast<const decltype(r.v)*>(p));
  }
  return r;
}
template <typename T, int V> PE_DEV void raw_store(T* p, const Raw<T, V>& r) { *reinterpret_cast<Raw<T, V>*>(p) = r; }
template <typename T, int V> PE_DEV Raw<T, V> raw_zero() {
  Raw<T, V> r;
#pragma unroll
  for (int i = 0; i < V; i++) r.set(i, 0.0f);
  return r;
}
typedef bf16 bf16x8_any __attribute__((ext_vector_type(8), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));
template <bool NT> PE_DEV Raw<bf16, 8> raw_load_any(const bf16* p) { Raw<bf16, 8> r; r.v = load_as<NT>(reinterpret_cast<const bf16x8_any*>(p)); return r; }
template <bool NT> PE_DEV Raw<float, 8> raw_load_any(const float* p) {
  Raw<float, 8> r;
  r.v[0] = load_as<NT>(reinterpret_cast<const f32x4_any*>(p));
  r.v[1] = load_as<NT>(reinterpret_cast<const f32x4_any*>(p + 4));
  return r;
}
PE_DEV void raw_store_any(bf16* p, const Raw<bf16, 8>& r) { *reinterpret_cast<bf16x8_any*>(p) = r.v; }
PE_DEV void raw_store_any(float* p, const Raw<float, 8>& r) {
  *reinterpret_cast<f32x4_any*>(p) = r.v[0];
  *reinterpret_cast<f32x4_any*>(p + 4) = r.v[1];
}

// How a lane's V of a row's c elements lie.  WHOLE: c a multiple of V, rows aligned to V elements.  Ragged (V = 8, c >= 8): any c and any
// alignment; the last vector of a row starts at c - 8, and its first `skip` elements are the vector's before it: they are
// loaded, count as zero, and are not stored.
template <int V, bool WHOLE> struct Slot {
  int at, skip;
  bool in;
  PE_DEV Slot(int vec, int c) {
    if constexpr (WHOLE) { in = vec < c / V; at = vec * V; skip = 0; }
    else { in = vec * V < c; at = min(vec * V, c - V); skip = vec * V - at; }
  }
  PE_DEV bool has(int i) const { return WHOLE || i >= skip; }
  template <bool NT = false, typename T> PE_DEV Raw<T, V> load(const T* row) const {
    if constexpr (WHOLE) return raw_load<T, V, NT>(row + at); else return raw_load_any<NT>(row + at);
  }
  template <typename T> PE_DEV void store(T* row, const Raw<T, V>& r) const {
    if constexpr (WHOLE) raw_store<T, V>(row + at, r);
    else if (skip == 0) raw_store_any(row + at, r);
    else
#pragma unroll
      for (int i = 1; i < V; i++)
        if (i >= skip) row[at + i] = (T)r.get(i);
  }
};

// V consecutive fp32 numbers at an address of which only 4-byte alignment is known, in as few accesses as there are 16-byte pieces
template <int V> PE_DEV void load_f32(const float* p, float (&v)[V]) {
  if constexpr (V == 8) {
    const f32x4_any a = *reinterpret_cast<const f32x4_any*>(p), b = *reinterpret_cast<const f32x4_any*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; i++) { v[i] = a[i]; v[4 + i] = b[i]; }
  } else {
    v[0] = *p;
  }
}
