// Activation checkpoints in 8 bits.
//
// Groups of 32 consecutive channels of a row share a scale 2^e: the smallest e >= -126 with max|x| <= 127 2^e, and 121 at most, since
// 64 2^122 is no number of either type any more (magnitudes above 127 2^121 become that).  A code is
// rint(x 2^-e) within -127..127, the value it stands for code 2^e.  A power of two makes every step but that one rounding exact (scaling,
// restoring, and the restored value in bf16: 7 bits of magnitude), so packing what was restored gives the same codes,
// and the result does not depend on how a division rounds.  The error is at most 2^(e-1), between 1/254 and 1/127 of the group's
// largest magnitude.  A group that holds an infinity or NaN is restored as NaN throughout: the loss stays visible.
//
// Layout of a checkpoint of [rows][c]: int8 codes [rows][c], then, at the next multiple of 256 bytes, one byte e + 127 per
// group, [rows][ceil(c / 32)]; 255 marks a group that was not finite.
#pragma once
#include "pe_lanes.h"

constexpr int CK_GROUP = 32;

// largest magnitude's bits (sign cleared) -> the group's scale byte
PE_DEV uint32_t ck_scale_byte(uint32_t m) {
  const int sb = (int)(m >> 23) - 6 + ((m & 0x7fffffu) > 0x7e0000u ? 1 : 0);     // 64 <= max|x| 2^-e <= 127; above 127/64 of a power of two: the next e
  return m >= 0x7f800000u ? 255u : (uint32_t)min(max(sb, 1), 248);
}
PE_DEV float ck_inverse(uint32_t sb) { return __uint_as_float((254u - sb) << 23); }    // 2^-e, sb 1..248
PE_DEV float ck_scale(uint32_t sb) { return sb == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(sb << 23); }
PE_DEV int ck_code(float x, float inv) { return (int)rintf(__builtin_amdgcn_fmed3f(x * inv, -127.0f, 127.0f)); }

template <int V> struct Codes;       // V consecutive codes
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(1)));
template <> struct Codes<8> {
  uint2 v;
  PE_DEV int get(int i) const { return (int)(int8_t)((i < 4 ? v.x : v.y) >> (8 * (i & 3))); }
  PE_DEV void clear() { v.x = v.y = 0; }
  PE_DEV void put(int i, int c) { (i < 4 ? v.x : v.y) |= ((uint32_t)c & 255u) << (8 * (i & 3)); }
};
template <> struct Codes<1> {
  int8_t v;
  PE_DEV int get(int) const { return (int)v; }
  PE_DEV void clear() { v = 0; }
  PE_DEV void put(int, int c) { v = (int8_t)c; }
};

// a lane's codes of a row (the row of codes has no gaps, so its alignment goes with c)
template <int V, bool WHOLE> PE_DEV Codes<V> codes_load(const int8_t* row, const Slot<V, WHOLE>& s) {
  Codes<V> c;
  if constexpr (WHOLE || V == 1) c = *reinterpret_cast<const Codes<V>*>(row + s.at);
  else { const u32x2_any w = *reinterpret_cast<const u32x2_any*>(row + s.at); c.v.x = w[0]; c.v.y = w[1]; }
  return c;
}
template <int V, bool WHOLE> PE_DEV void codes_store(int8_t* row, const Slot<V, WHOLE>& s, const Codes<V>& c) {
  if constexpr (WHOLE || V == 1) *reinterpret_cast<Codes<V>*>(row + s.at) = c;
  else if (s.skip == 0) *reinterpret_cast<u32x2_any*>(row + s.at) = u32x2_any{c.v.x, c.v.y};
  else
#pragma unroll
    for (int i = 1; i < V; i++)
      if (i >= s.skip) row[s.at + i] = (int8_t)c.get(i);
}

// V elements of each of the LG lanes that share a group -> the scale byte of the group (in all of its lanes) and this lane's codes.
// Elements that are not the lane's have to be zero.
template <int V, int LG> PE_DEV uint32_t ck_encode(const float (&x)[V], Codes<V>& codes) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < V; i++) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);    // as integers NaN is above infinity above every number
  const uint32_t sb = ck_scale_byte(lanes_umax<LG>(m));
  const float inv = ck_inverse(sb == 255u ? 127u : sb);
  codes.clear();
#pragma unroll
  for (int i = 0; i < V; i++) codes.put(i, sb == 255u ? 0 : ck_code(x[i], inv));
  return sb;
}

// One item = V channels of a row; a row has `per_row` items, a multiple of the LG that share a group (V = 8: 4; V = 1, rows of
// fewer than 8 channels: 8, one group per row), so item / LG numbers the groups.  A wave takes 64 U consecutive items, all of its
// loads in flight at once; their scales are 64 U / LG consecutive bytes, stored by as many lanes together.  `flat`: no gaps and
// whole groups; whole vectors then need no rows, it is one long row.  HBM-bound.  Workgroups behind the first CK_GRID_X are in further rows of the grid.
constexpr int CK_GRID_X = 1 << 22;
template <typename T, int V, bool WHOLE, int U, bool PACK, bool NT>
__global__ __launch_bounds__(256) void ckpt_kernel(const T* x, long long ld, int8_t* codes, uint8_t* scales, T* y, long long rows,
                                                   int c, int per_row, int flat) {
  constexpr int LG = V == 8 ? 4 : 8;
  const int lane = threadIdx.x & 63;
  const long long items = rows * per_row, first = (((long long)blockIdx.y * CK_GRID_X + blockIdx.x) * 4 + (threadIdx.x >> 6)) * (64 * U);
  const bool line = WHOLE && flat;
  const long long row0 = line ? 0 : first / per_row;
  const uint32_t rem = line ? 0 : (uint32_t)(first - row0 * per_row);
  long long at[U], code_at[U];       // element offsets of the row in x or y, and in the codes (flat: of the item)
  int vec[U];
  bool in[U];
  Raw<T, V> v[U];
  Codes<V> cd[U];
  uint32_t sb[U];
#pragma unroll
  for (int u = 0; u < U; u++) {
    const long long item = first + 64 * u + lane;
    if (line) {
      in[u] = item < items;
      vec[u] = 0;
      at[u] = code_at[u] = item * V;
    } else {
      const uint32_t off = rem + 64u * u + lane, dr = off / (uint32_t)per_row;
      const long long row = row0 + dr;
      vec[u] = (int)(off - dr * (uint32_t)per_row);
      in[u] = item < items && vec[u] * V < c;
      at[u] = row * ld;
      code_at[u] = row * c;
    }
    const Slot<V, WHOLE> s(vec[u], c);
    if constexpr (PACK) {
      v[u] = in[u] ? s.template load<NT>(x + at[u]) : raw_zero<T, V>();
    } else if (in[u]) {
      cd[u] = codes_load(codes + code_at[u], s);
      sb[u] = scales[item / LG];
    }
  }
#pragma unroll
  for (int u = 0; u < U; u++) {
    const Slot<V, WHOLE> s(vec[u], c);
    if constexpr (PACK) {
      float f[V];
#pragma unroll
      for (int i = 0; i < V; i++) f[i] = s.has(i) ? v[u].get(i) : 0.0f;
      sb[u] = ck_encode<V, LG>(f, cd[u]);
      if (in[u]) codes_store(codes + code_at[u], s, cd[u]);
    } else if (in[u]) {
      const float scale = ck_scale(sb[u]);
#pragma unroll
      for (int i = 0; i < V; i++) v[u].set(i, (float)cd[u].get(i) * scale);
      s.store(y + at[u], v[u]);
    }
  }
  if constexpr (PACK) {
    constexpr int PER = 64 / LG, N = U * PER;      // groups per 64 items, per wave
    static_assert(N <= 64, "a lane stores one scale");
    uint32_t mine = 0;
#pragma unroll
    for (int u = 0; u < U; u++) {
      const uint32_t t = (uint32_t)__shfl((int)sb[u], (lane % PER) * LG, 64);
      if (lane / PER == u) mine = t;
    }
    const long long group = first / LG + lane;
    if (lane < N && group < items / LG) scales[group] = (uint8_t)mine;
  }
}
