// Relative position embedding by buckets, and the gradient of its table.
//
// d = pos_q - pos_k falls into bucket #{k : edge_k <= d}; the edges are ascending integers, so a bucket is exact whatever rule
// made them.  A pair of different segments has a bucket of its own behind the others.
//   layout PAIR :  out[q][k][ch] = [add +] table[bucket][ch]         (the pair representation)
//   layout HEADS:  out[ch][q][k] = [add +] table[bucket][ch]         (the bias of an attention, ch = head)
//   d_table[b][ch] = sum over the pairs (q, k) in bucket b of d_out
// HBM-bound: the output (and `add`) once, or d_out once.
#pragma once
#include "pe_lanes.h"

constexpr int RP_MAX_EDGES = 254;
struct RpArgs {
  const int* pos_q; const int* pos_k; const int* seg_q; const int* seg_k;     // seg_*: null without segments
  const float* table;
  const void* add;
  void* out;
  const void* d_out;
  float* part;
  long long ld;            // elements between rows q
  int n_q, n_k, c, nb;     // nb: buckets, the one of different segments among them
  int n_edges, dense;      // dense: the edges are consecutive integers
  int edges[RP_MAX_EDGES];
};

// Difference of two positions, clamped to 32 bits: no edge is the least 32-bit number, so the clamped value is in the same bucket
PE_DEV int rp_diff(int a, int b) {
  const long long d = (long long)a - b;
  return (int)(d < -2147483647LL - 1 ? -2147483647LL - 1 : d > 2147483647LL ? 2147483647LL : d);
}
// Edges in LDS.  Consecutive edges (clipped distances) need no search.
struct RpBuckets {
  const int* lds;
  int n, dense, first, other;
  // every thread of the workgroup; the caller passes a barrier before the first use
  static PE_DEV void fill(int* lds, const RpArgs& a) {
    for (int i = threadIdx.x; i < a.n_edges; i += blockDim.x) lds[i] = a.edges[i];
  }
  PE_DEV RpBuckets(const int* l, const RpArgs& a) : lds(l), n(a.n_edges), dense(a.dense), first(a.dense ? a.edges[0] : 0), other(a.nb - 1) {}
  PE_DEV int of(int pq, int pk) const {
    const int d = rp_diff(pq, pk);
    if (dense) {
      if (d < first) return 0;
      const uint32_t u = (uint32_t)d - (uint32_t)first;      // at least 0: no overflow
      return u >= (uint32_t)n ? n : (int)u + 1;
    }
    int lo = 0, len = n;                                     // edges before lo are <= d
    while (len > 0) {
      const int half = (len + 1) >> 1;
      if (lds[lo + half - 1] <= d) lo += half, len -= half; else len = half - 1;
    }
    return lo;
  }
  PE_DEV int of(int pq, int pk, int sq, int sk) const { return sq != sk ? other : of(pq, pk); }
};

// ---------------------------------------------------------------------------------------------------------------------
// PAIR, forward: a workgroup has one q and RP_PK positions k: first the buckets of those, while `add` is on its way, then
// V channels per lane and step.
// ---------------------------------------------------------------------------------------------------------------------
template <typename T, int V, int U>
__global__ __launch_bounds__(256) void relpos_pair_fwd_kernel(const RpArgs a, int tile_k) {
  __shared__ int edges[RP_MAX_EDGES + 2];
  __shared__ int bucket[1024];
  const int q = blockIdx.y + blockIdx.z * 65535, k0 = blockIdx.x * tile_k;
  if (q >= a.n_q) return;
  const int nk = min(tile_k, a.n_k - k0), vecs = a.c / V, total = nk * vecs;     // at most 1024 positions
  const long long base = (long long)q * a.ld + (long long)k0 * a.c;
  const T* add = (const T*)a.add;
  T* out = (T*)a.out;
  Raw<T, V> ad[U];
  if (add) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int e = threadIdx.x + 256 * u;
      if (e < total) ad[u] = raw_load<T, V>(add + base + (long long)e * V);
    }
  }
  RpBuckets::fill(edges, a);
  __syncthreads();
  const RpBuckets rb(edges, a);
  const int pq = a.pos_q[q], sq = a.seg_q ? a.seg_q[q] : 0;
  for (int i = threadIdx.x; i < nk; i += 256) bucket[i] = rb.of(pq, a.pos_k[k0 + i], sq, a.seg_q ? a.seg_k[k0 + i] : 0);
  __syncthreads();
#pragma unroll
  for (int u = 0; u < U; u++) {
    const int e = threadIdx.x + 256 * u;
    if (e < total) {
      const int k = e / vecs;
      const float* t = a.table + (long long)bucket[k] * a.c + (e - k * vecs) * V;
      Raw<T, V> o;
#pragma unroll
      for (int i = 0; i < V; i++) o.set(i, add ? ad[u].get(i) + t[i] : t[i]);
      raw_store<T, V>(out + base + (long long)e * V, o);
    }
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// HEADS, forward: a workgroup has one q, 256 V positions k and `heads` heads, whose table columns lie in LDS as [head][bucket]
// (neighbouring distances are neighbouring banks).  A lane finds its V buckets once for all heads.
// ---------------------------------------------------------------------------------------------------------------------
template <typename T, int V>
__global__ __launch_bounds__(256) void relpos_heads_fwd_kernel(const RpArgs a, int heads, int rows) {
  extern __shared__ float tab[];       // [heads][nb]
  __shared__ int edges[RP_MAX_EDGES + 2];
  const int h0 = blockIdx.z * heads, nh = min(heads, a.c - h0);
  const int k = (blockIdx.x * 256 + threadIdx.x) * V;
  RpBuckets::fill(edges, a);
  for (int i = threadIdx.x; i < nh * a.nb; i += 256) {
    const int b = i / nh, h = i - b * nh;
    tab[h * a.nb + b] = a.table[(long long)b * a.c + h0 + h];
  }
  __syncthreads();
  if (k >= a.n_k) return;
  const RpBuckets rb(edges, a);
  int pk[V], sk[V];
#pragma unroll
  for (int i = 0; i < V; i++) { pk[i] = a.pos_k[k + i]; sk[i] = a.seg_q ? a.seg_k[k + i] : 0; }
  const T* add = (const T*)a.add;
  T* out = (T*)a.out;
  for (int q = blockIdx.y * rows; q < min(a.n_q, (int)(blockIdx.y + 1) * rows); q++) {
    const int pq = a.pos_q[q], sq = a.seg_q ? a.seg_q[q] : 0;
    int b[V];
#pragma unroll
    for (int i = 0; i < V; i++) b[i] = rb.of(pq, pk[i], sq, sk[i]);
    for (int h = 0; h < nh; h++) {
      const long long at = ((long long)(h0 + h) * a.n_q + q) * a.ld + k;
      Raw<T, V> o, ad;
      if (add) ad = raw_load<T, V>(add + at);
#pragma unroll
      for (int i = 0; i < V; i++) o.set(i, add ? ad.get(i) + tab[h * a.nb + b[i]] : tab[h * a.nb + b[i]]);
      raw_store<T, V>(out + at, o);
    }
  }
}

// v is added to an LDS word that belongs to this lane alone (LDS operations of a wave execute in order, so the sum's order is
// the program's): one instruction without a result to wait for
PE_DEV void lds_add(float* p, float v) { __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

// ---------------------------------------------------------------------------------------------------------------------
// PAIR, backward.  Lane = channel; a wave walks over positions and adds each to the LDS word [bucket][lane] of its own
// accumulators.  S positions share a wave where c <= 32.  blockIdx.y: slab of 64 channels (S = 1).
// ---------------------------------------------------------------------------------------------------------------------
template <typename T, int S, int U>
__global__ __launch_bounds__(512) void relpos_pair_bwd_kernel(const RpArgs a, long long per_group) {
  extern __shared__ float acc[];       // [waves][nb][64], then the edges
  constexpr int CL = 64 / S;           // lanes per position
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int sub = lane / CL, ch = blockIdx.y * 64 + lane % CL;
  int* edges = reinterpret_cast<int*>(acc + waves * a.nb * 64);
  float* mine = acc + wave * a.nb * 64 + lane;
  RpBuckets::fill(edges, a);
  for (int i = threadIdx.x; i < waves * a.nb * 64; i += blockDim.x) acc[i] = 0.0f;
  __syncthreads();
  const RpBuckets rb(edges, a);
  const T* g = (const T*)a.d_out;
  const long long n = (long long)a.n_q * a.n_k;
  const long long p0 = (long long)blockIdx.x * per_group, p1 = min(n, p0 + per_group);
  const bool on = ch < a.c;
  // a wave takes runs of 64 positions: lane l finds the bucket of the l-th
  for (long long p = p0 + wave * 64; p < p1; p += 64LL * waves) {
    const int cnt = (int)min((long long)64, p1 - p);
    const int q0 = (int)(p / a.n_k), kk = (int)(p - (long long)q0 * a.n_k);    // of the first position
    int b = 0;
    long long row = 0;                                                        // this lane's position's offset in d_out
    if (lane < cnt) {
      const int over = kk + lane, dq = over / a.n_k, q = q0 + dq, k = over - dq * a.n_k;
      b = rb.of(a.pos_q[q], a.pos_k[k], a.seg_q ? a.seg_q[q] : 0, a.seg_q ? a.seg_k[k] : 0);
      row = (long long)q * a.ld + (long long)k * a.c;
    }
    const int rlo = (int)(uint32_t)(uint64_t)row, rhi = (int)(uint32_t)((uint64_t)row >> 32);
#pragma unroll 1
    for (int j = 0; j < 64; j += S * U) {
      if (j >= cnt) break;
      float v[U];
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int l = j + u * S + sub;
        long long r;
        if constexpr (S == 1) {
          const uint32_t lo = __builtin_amdgcn_readlane(rlo, l), hi = __builtin_amdgcn_readlane(rhi, l);
          r = (long long)(((uint64_t)hi << 32) | lo);
        } else {
          r = (long long)(((uint64_t)(uint32_t)__shfl(rhi, l, 64) << 32) | (uint32_t)__shfl(rlo, l, 64));
        }
        v[u] = on && l < cnt ? (float)g[r + ch] : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int l = j + u * S + sub;
        int bb;
        if constexpr (S == 1) bb = __builtin_amdgcn_readlane(b, l); else bb = __shfl(b, l, 64);
        lds_add(mine + bb * 64, v[u]);
      }
    }
  }
  __syncthreads();
  // the waves' accumulators and the positions side by side, in a fixed order
  float* part = a.part + (long long)blockIdx.x * a.nb * a.c;
  for (int i = threadIdx.x; i < a.nb * CL; i += blockDim.x) {
    const int b = i / CL, l = i % CL, cc = blockIdx.y * 64 + l;
    float s = 0.0f;
    for (int w = 0; w < waves; w++)
#pragma unroll
      for (int t = 0; t < S; t++) s += acc[(w * a.nb + b) * 64 + t * CL + l];
    if (cc < a.c) part[(long long)b * a.c + cc] = s;
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// HEADS, backward.  Lane = V positions k; a wave walks over rows q of one head and adds each element to the LDS word [bucket][lane]
// of its own accumulators (bank = lane whatever the buckets are).
// ---------------------------------------------------------------------------------------------------------------------
template <typename T, int V>
__global__ __launch_bounds__(512) void relpos_heads_bwd_kernel(const RpArgs a, int rows) {
  extern __shared__ float acc[];       // [waves][nb][64], then the edges
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int* edges = reinterpret_cast<int*>(acc + waves * a.nb * 64);
  float* mine = acc + wave * a.nb * 64 + lane;
  RpBuckets::fill(edges, a);
  for (int i = threadIdx.x; i < waves * a.nb * 64; i += blockDim.x) acc[i] = 0.0f;
  __syncthreads();
  const RpBuckets rb(edges, a);
  const int h = blockIdx.z, k = (blockIdx.x * 64 + lane) * V;
  const int q1 = min(a.n_q, (int)(blockIdx.y + 1) * rows);
  if (k < a.n_k) {
    int pk[V], sk[V];
#pragma unroll
    for (int i = 0; i < V; i++) { pk[i] = a.pos_k[k + i]; sk[i] = a.seg_q ? a.seg_k[k + i] : 0; }
    const T* g = (const T*)a.d_out + (long long)h * a.n_q * a.ld + k;
    for (int q = blockIdx.y * rows + wave; q < q1; q += waves) {
      const Raw<T, V> v = raw_load<T, V>(g + (long long)q * a.ld);
      const int pq = a.pos_q[q], sq = a.seg_q ? a.seg_q[q] : 0;
#pragma unroll
      for (int i = 0; i < V; i++) lds_add(mine + rb.of(pq, pk[i], sq, sk[i]) * 64, v.get(i));
    }
  }
  __syncthreads();
  float* part = a.part + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * a.nb * a.c;
  for (int b = wave; b < a.nb; b += waves) {
    float s = 0.0f;
    for (int w = 0; w < waves; w++) s += acc[(w * a.nb + b) * 64 + lane];
    s = lanes_sum<64>(s);
    if (lane == 0) part[(long long)b * a.c + h] = s;
  }
}
