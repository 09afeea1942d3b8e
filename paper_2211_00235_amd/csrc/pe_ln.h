// Layer norm as an operator of its own: forward and backward over [rows][c] with row strides.
//
//   y  = [add +] (x - mean) rstd gain + offset                                    mean, rstd: of the row, variance in two passes
//   dx = [add +] rstd (u - mean(u) - z mean(u z)),  u = gain dy,  z = (x - mean) rstd
//   d_gain = sum over rows of dy z,  d_offset = sum over rows of dy
//
// HBM-bound: 8 vector operations per element forward, 15 backward, against 4 to 8 bytes.  A row lies in the registers of L
// lanes (NV vectors of V elements each), so that it is read once: L = 4..64 lanes, several rows per wave, up to 1024 channels,
// whole workgroups above.  Other channel counts and alignments than whole, aligned 16-byte pieces take the same kernels with WHOLE = false; rows of fewer
// than 8 channels have a lane per channel.  Statistics and sums are fp32; a result is rounded once, to the storage type.  A lane keeps its columns'
// d_gain and d_offset in registers over all of its rows; workgroups write one fp32 partial each, and columns_sum_kernel adds
// them in a fixed order.
#pragma once
#include "pe_ckpt.h"

struct LnArgs {
  const void* x; long long ld_x;          // x, or null where codes / scales hold it in 8 bits
  const int8_t* codes; const uint8_t* scales;
  const void* add; long long ld_add;
  const void* dy; long long ld_dy;
  void* out; long long ld_out;            // y, or dx (null: not wanted)
  int8_t* k_codes; uint8_t* k_scales;     // forward: x in 8 bits (null: not wanted)
  const float* gain; const float* offset; // null: 1, 0
  float* stats;
  const float* stats_in;
  float* part;                            // backward: [workgroups][2][c] (null: not wanted)
  long long rows;
  int c;
  float eps;
};

// Sum over the L lanes of a row; above 64 lanes the waves of the workgroup exchange theirs through `red`.  A row uses two
// slots of `red` and the next row the other two, so one barrier per sum is enough.
template <int L> PE_DEV float row_sum(float v, float* red) {
  v = lanes_sum<(L < 64 ? L : 64)>(v);
  if constexpr (L > 64) {
    constexpr int W = L / 64;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < W; w++) v += red[w];
  }
  return v;
}

// two sums at once, with one barrier
template <int L> PE_DEV void row_sums(float& p, float& q, float* red, float* red2) {
  p = lanes_sum<(L < 64 ? L : 64)>(p);
  q = lanes_sum<(L < 64 ? L : 64)>(q);
  if constexpr (L > 64) {
    constexpr int W = L / 64;
    if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6] = p; red2[threadIdx.x >> 6] = q; }
    __syncthreads();
    p = q = 0.0f;
#pragma unroll
    for (int w = 0; w < W; w++) { p += red[w]; q += red2[w]; }
  }
}

// Workgroup shape of a row of L lanes: rows side by side
template <int L> struct LnShape {
  static constexpr int THREADS = L > 256 ? L : 256;
  static constexpr int ROWS = THREADS / L;
};

template <typename T, int V, bool WHOLE, int L, int NV>
__global__ __launch_bounds__(LnShape<L>::THREADS) void ln_op_fwd_kernel(const LnArgs a) {
  constexpr int ROWS = LnShape<L>::ROWS, LG = V == 8 ? 4 : 8;
  __shared__ float red[4][16];
  const int li = threadIdx.x % L;                        // this lane's place in its row
  const int c = a.c, groups = (c + CK_GROUP - 1) / CK_GROUP;
  const float inv_c = 1.0f / (float)c;
  auto slot_of = [&](int n) { return Slot<V, WHOLE>(n * L + li, c); };
  float gain[NV][V], offs[NV][V];
#pragma unroll
  for (int n = 0; n < NV; n++) {
#pragma unroll
    for (int i = 0; i < V; i++) { gain[n][i] = 1.0f; offs[n][i] = 0.0f; }
    const auto sl = slot_of(n);
    if (sl.in && a.gain) load_f32<V>(a.gain + sl.at, gain[n]);
    if (sl.in && a.offset) load_f32<V>(a.offset + sl.at, offs[n]);
  }
  const T* x = (const T*)a.x;
  const T* add = (const T*)a.add;
  T* y = (T*)a.out;
  long long row = (long long)blockIdx.x * ROWS + threadIdx.x / L;
  const long long step = (long long)gridDim.x * ROWS;
  Raw<T, V> next[NV];
  auto fetch = [&](long long r) {
#pragma unroll
    for (int n = 0; n < NV; n++) {
      const auto sl = slot_of(n);
      next[n] = sl.in && r < a.rows ? sl.load(x + r * a.ld_x) : raw_zero<T, V>();
    }
  };
  fetch(row);
  int slot = 0;
  for (; row < a.rows; row += step, slot ^= 2) {
    Raw<T, V> v[NV], ad[NV];
#pragma unroll
    for (int n = 0; n < NV; n++) v[n] = next[n];
    if (add) {
#pragma unroll
      for (int n = 0; n < NV; n++) {
        const auto sl = slot_of(n);
        if (sl.in) ad[n] = sl.load(add + row * a.ld_add);
      }
    }
    fetch(row + step);
    float s = 0.0f;
#pragma unroll
    for (int n = 0; n < NV; n++)
#pragma unroll
      for (int i = 0; i < V; i++) s += slot_of(n).has(i) ? v[n].get(i) : 0.0f;
    const float mean = row_sum<L>(s, red[slot]) * inv_c;
    float q = 0.0f;
#pragma unroll
    for (int n = 0; n < NV; n++)
#pragma unroll
      for (int i = 0; i < V; i++) {
        const auto sl = slot_of(n);
        const float t = sl.in && sl.has(i) ? v[n].get(i) - mean : 0.0f;
        q += t * t;
      }
    const float rstd = rsqrtf(row_sum<L>(q, red[slot + 1]) * inv_c + a.eps);
    if (a.stats && li == 0) *reinterpret_cast<f32x2*>(a.stats + 2 * row) = f32x2{mean, rstd};
#pragma unroll
    for (int n = 0; n < NV; n++) {
      Raw<T, V> o;
#pragma unroll
      for (int i = 0; i < V; i++) {
        float f = (v[n].get(i) - mean) * rstd * gain[n][i] + offs[n][i];
        if (add) f += ad[n].get(i);
        o.set(i, f);
      }
      const auto sl = slot_of(n);
      if (sl.in) sl.store(y + row * a.ld_out, o);
      if (a.k_codes) {
        float f[V];
#pragma unroll
        for (int i = 0; i < V; i++) f[i] = sl.has(i) ? v[n].get(i) : 0.0f;
        Codes<V> cd;
        const uint32_t sb = ck_encode<V, LG>(f, cd);
        if (sl.in) {
          const int vec = n * L + li;
          codes_store(a.k_codes + row * c, sl, cd);
          if (vec % LG == 0) a.k_scales[row * groups + vec / LG] = (uint8_t)sb;
        }
      }
    }
  }
}

template <typename T, int V, bool WHOLE, int L, int NV, bool KEPT>
__global__ __launch_bounds__(LnShape<L>::THREADS) void ln_op_bwd_kernel(const LnArgs a) {
  constexpr int ROWS = LnShape<L>::ROWS, LG = V == 8 ? 4 : 8, W = LnShape<L>::THREADS / 64;
  __shared__ float red[4][16];
  const int li = threadIdx.x % L;
  const int c = a.c, groups = (c + CK_GROUP - 1) / CK_GROUP;
  const float inv_c = 1.0f / (float)c;
  auto slot_of = [&](int n) { return Slot<V, WHOLE>(n * L + li, c); };
  float gain[NV][V], dg[NV][V], db[NV][V];
#pragma unroll
  for (int n = 0; n < NV; n++) {
#pragma unroll
    for (int i = 0; i < V; i++) { gain[n][i] = 1.0f; dg[n][i] = db[n][i] = 0.0f; }
    const auto sl = slot_of(n);
    if (sl.in && a.gain) load_f32<V>(a.gain + sl.at, gain[n]);
  }
  const T* x = (const T*)a.x;
  const T* dy = (const T*)a.dy;
  const T* add = (const T*)a.add;
  T* dx = (T*)a.out;
  long long row = (long long)blockIdx.x * ROWS + threadIdx.x / L;
  const long long step = (long long)gridDim.x * ROWS;
  Raw<T, V> nx[NV], ny[NV];
  Codes<V> nc[NV];
  uint32_t nsb[NV];
  f32x2 nst;
  auto fetch = [&](long long r) {
    const bool live = r < a.rows;
    nst = live ? *reinterpret_cast<const f32x2*>(a.stats_in + 2 * r) : f32x2{0.0f, 0.0f};
#pragma unroll
    for (int n = 0; n < NV; n++) {
      const auto sl = slot_of(n);
      const bool on = sl.in && live;
      ny[n] = on ? sl.load(dy + r * a.ld_dy) : raw_zero<T, V>();
      if constexpr (KEPT) {
        nc[n].clear();
        nsb[n] = 0;
        if (on) {
          nc[n] = codes_load(a.codes + r * c, sl);
          nsb[n] = a.scales[r * groups + (n * L + li) / LG];
        }
      } else {
        nx[n] = on ? sl.load(x + r * a.ld_x) : raw_zero<T, V>();
      }
    }
  };
  constexpr bool AHEAD = L <= 512;      // the next row is requested ahead; 1024 lanes have 128 registers each, too few for it
  if constexpr (AHEAD) fetch(row);
  int slot = 0;
  for (; row < a.rows; row += step, slot ^= 2) {
    Raw<T, V> y[NV], ad[NV], xv[NV];
    Codes<V> cd[NV];
    float sc[NV];
    if constexpr (!AHEAD) fetch(row);
    const float mean = nst[0], rstd = nst[1];
#pragma unroll
    for (int n = 0; n < NV; n++) {
      y[n] = ny[n];
      if constexpr (KEPT) { cd[n] = nc[n]; sc[n] = ck_scale(nsb[n]); } else xv[n] = nx[n];
    }
    if (add && dx) {
#pragma unroll
      for (int n = 0; n < NV; n++) {
        const auto sl = slot_of(n);
        if (sl.in) ad[n] = sl.load(add + row * a.ld_add);
      }
    }
    if constexpr (AHEAD) fetch(row + step);
    auto z_of = [&](int n, int i) {
      float f;
      if constexpr (KEPT) f = (float)cd[n].get(i) * sc[n]; else f = xv[n].get(i);
      return (f - mean) * rstd;
    };
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int n = 0; n < NV; n++)
#pragma unroll
      for (int i = 0; i < V; i++) {
        const auto sl = slot_of(n);
        const float d = sl.has(i) ? y[n].get(i) : 0.0f, z = sl.in && sl.has(i) ? z_of(n, i) : 0.0f, u = d * gain[n][i];
        dg[n][i] += d * z;
        db[n][i] += d;
        s1 += u;
        s2 += u * z;
      }
    if (dx) {
      row_sums<L>(s1, s2, red[slot], red[slot + 1]);
      const float m1 = s1 * inv_c, m2 = s2 * inv_c;
#pragma unroll
      for (int n = 0; n < NV; n++) {
        Raw<T, V> o;
#pragma unroll
        for (int i = 0; i < V; i++) {
          float f = rstd * (y[n].get(i) * gain[n][i] - m1 - z_of(n, i) * m2);
          if (add) f += ad[n].get(i);
          o.set(i, f);
        }
        const auto sl = slot_of(n);
        if (sl.in) sl.store(dx + row * a.ld_out, o);
      }
    }
  }
  if (!a.part) return;
  float* part = a.part + (long long)blockIdx.x * 2 * c;
  if constexpr (L <= 64) {     // the lanes of a wave that hold the same columns, then the waves
    __shared__ float cols[2][W][L][V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int n = 0; n < NV; n++) {
#pragma unroll
      for (int i = 0; i < V; i++) {
        if constexpr (L < 64) { dg[n][i] = strided_sum<L>(dg[n][i]); db[n][i] = strided_sum<L>(db[n][i]); }
        if (lane < L) { cols[0][wave][lane][i] = dg[n][i]; cols[1][wave][lane][i] = db[n][i]; }
      }
      __syncthreads();
      for (int k = threadIdx.x; k < 2 * L * V; k += LnShape<L>::THREADS) {
        const int t = k / (L * V), e = k % (L * V);
        const Slot<V, WHOLE> sl(n * L + e / V, c);
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < W; w++) s += (&cols[t][w][0][0])[e];
        if (sl.in && sl.has(e % V)) part[t * c + sl.at + e % V] = s;
      }
      __syncthreads();
    }
  } else {                     // every column is one lane's
#pragma unroll
    for (int n = 0; n < NV; n++) {
      const auto sl = slot_of(n);
      if (sl.in)
#pragma unroll
        for (int i = 0; i < V; i++)
          if (sl.has(i)) {
            part[sl.at + i] = dg[n][i];
            part[c + sl.at + i] = db[n][i];
          }
    }
  }
}

// out[col] (+)= sum over p of part[p][col], in a fixed order: a workgroup has 16 columns (64 bytes of a partial) and 64 lanes per
// column, which add every 64th partial each; then a tree.  Columns from `split` on go to out1.  The loads of a thread do not
// wait for one another: with a thread per column 1024 partials took longer than the pass that wrote them.
__global__ __launch_bounds__(1024) void columns_sum_kernel(const float* part, int n_part, int cols, float* out0, float* out1, int split,
                                                           int accumulate) {
  __shared__ float sums[64][17];
  const int cl = threadIdx.x & 15, p0 = threadIdx.x >> 4, col = blockIdx.x * 16 + cl;
  float s = 0.0f;
  if (col < cols) {
    int p = p0;
    for (; p + 192 < n_part; p += 256) {
      const float* q = part + (long long)p * cols + col;
      const long long st = 64LL * cols;
      const float v0 = q[0], v1 = q[st], v2 = q[2 * st], v3 = q[3 * st];
      s += (v0 + v1) + (v2 + v3);
    }
    for (; p < n_part; p += 64) s += part[(long long)p * cols + col];
  }
  sums[p0][cl] = s;
  __syncthreads();
  if (threadIdx.x < 256) {
    const int c2 = threadIdx.x >> 4, l = threadIdx.x & 15, oc = blockIdx.x * 16 + c2;     // 16 lanes per column
    float t = (sums[l][c2] + sums[l + 16][c2]) + (sums[l + 32][c2] + sums[l + 48][c2]);
    t = lanes_sum<16>(t);
    if (l == 0 && oc < cols) {
      float* to = oc < split ? out0 : out1;      // null: not wanted
      if (to) {
        float* o = to + (oc < split ? oc : oc - split);
        *o = accumulate ? *o + t : t;
      }
    }
  }
}
