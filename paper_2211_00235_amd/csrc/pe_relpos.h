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
constexpr int RP_LUT = 4096;     // widest range of distances with a table of its own
struct RpArgs {
  const int* pos_q; const int* pos_k; const int* seg_q; const int* seg_k;     // seg_*: null without segments
  const float* table;
  const void* add;
  void* out;
  const void* d_out;
  float* part;
  long long ld;            // elements between rows q
  int n_q, n_k, c, nb;     // nb: buckets, the one of different segments among them
  int n_edges;
  int mode;                // RpMode, by which the host side picks the kernel
  int lo, hi;              // DENSE, LUT: first edge - 1, last edge (0, 0 without edges)
  int edges[RP_MAX_EDGES];
};

// How a bucket is found.  DENSE: the edges are consecutive integers (clipped distances), the clamped distance is the bucket.
// LUTS: the edges span at most RP_LUT distances; a byte per distance in LDS.  SEARCH: edges in LDS, by bisection, up to eight reads that
// wait for one another: backward of 16 heads over 2048 x 2048 positions 67 us, with the bytes 35.  The bytes take a workgroup about
// 1 us, which pays from some ten lookups per lane on: kernels with fewer (PAIR, one row of HEADS: 4.6 us, 3.7 by bisection) search.
enum RpMode { RP_DENSE = 0, RP_LUTS = 1, RP_SEARCH = 2 };
constexpr int rp_lds_words(int mode) { return mode == RP_DENSE ? 1 : mode == RP_LUTS ? RP_LUT / 4 + 1 : RP_MAX_EDGES + 2; }

// Difference of two positions, clamped to 32 bits: no edge is the least 32-bit number, so the clamped value is in the same bucket
PE_DEV int rp_diff(int a, int b) {
  const long long d = (long long)a - b;
  return (int)(d < -2147483647LL - 1 ? -2147483647LL - 1 : d > 2147483647LL ? 2147483647LL : d);
}
template <typename E> PE_DEV int rp_search(E&& edge, int n, int d) {
  int lo = 0, len = n;                                     // edges before lo are <= d, the answer is at most lo + len
  while (len > 0) {
    const int half = (len + 1) >> 1;
    if (edge(lo + half - 1) <= d) lo += half, len -= half; else len = half - 1;
  }
  return lo;
}
template <int MODE> struct RpBuckets {
  const int* lds;
  int n, lo, hi, other;
  // every thread of the workgroup; the caller passes a barrier before the first use
  static PE_DEV void fill(int* lds, const RpArgs& a) {
    if constexpr (MODE == RP_LUTS) {      // a wave fills a bucket's bytes (a search per byte is a chain of loads: 3 us at the start of every workgroup)
      const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
      for (int b = wave; b <= a.n_edges; b += waves) {
        const int from = b == 0 ? 0 : a.edges[b - 1] - a.lo, to = b == a.n_edges ? a.hi - a.lo + 1 : a.edges[b] - a.lo;
        for (int i = from + lane; i < to; i += 64) reinterpret_cast<uint8_t*>(lds)[i] = (uint8_t)b;
      }
    }
    if constexpr (MODE == RP_SEARCH)
      for (int i = threadIdx.x; i < a.n_edges; i += blockDim.x) lds[i] = a.edges[i];
  }
  PE_DEV RpBuckets(const int* l, const RpArgs& a) : lds(l), n(a.n_edges), lo(a.lo), hi(a.hi), other(a.nb - 1) {}
  PE_DEV int of(int pq, int pk) const {
    const int d = rp_diff(pq, pk);
    if constexpr (MODE == RP_SEARCH) return rp_search([&](int k) { return lds[k]; }, n, d);
    const int i = min(max(d, lo), hi) - lo;                // 0: below the first edge
    if constexpr (MODE == RP_LUTS) return reinterpret_cast<const uint8_t*>(lds)[i];
    return i;
  }
  PE_DEV int of(int pq, int pk, int sq, int sk) const {
    const int b = of(pq, pk);
    return sq != sk ? other : b;
  }
};

// V neighbouring positions k of a lane.  far(): the bucket of all of them against q where it can be told without a look at each (all
// beyond the outermost edges, or all of one other segment), otherwise -1.
// (a ragged slot's elements that are its neighbour's among them)
template <int V> struct RpLane {
  int pos[V], seg[V], least, most;
  bool one_seg;
  PE_DEV RpLane(const RpArgs& a, int k) {
#pragma unroll
    for (int i = 0; i < V; i++) { pos[i] = a.pos_k[k + i]; seg[i] = a.seg_q ? a.seg_k[k + i] : 0; }
    least = most = pos[0];
    one_seg = true;
#pragma unroll
    for (int i = 1; i < V; i++) { least = min(least, pos[i]); most = max(most, pos[i]); one_seg = one_seg && seg[i] == seg[0]; }
  }
  template <int MODE> PE_DEV int far(const RpBuckets<MODE>& rb, int pq, int sq) const {
    if constexpr (V == 1) return rb.of(pq, pos[0], sq, seg[0]);
    if (!one_seg) return -1;
    if (sq != seg[0]) return rb.other;
    if (rp_diff(pq, least) <= rb.lo) return 0;            // the largest distance is below the first edge
    if (rp_diff(pq, most) >= rb.hi) return rb.n;
    return -1;
  }
};

// ---------------------------------------------------------------------------------------------------------------------
// PAIR, forward: a workgroup has one q and tile_k positions k.  A lane has V channels of U positions; the positions' numbers and
// `add` are requested together, then the U table rows, so two round trips to memory lie one behind the other.  Lanes find their
// buckets each for itself: with buckets passed through LDS two barriers joined the chain (16.8 MB written and read: 21 us).
// vecs: vectors per position; vec_magic: ceil(2^32 / vecs), 0 for 1
// ---------------------------------------------------------------------------------------------------------------------
template <typename T, int V, bool WHOLE, int U, int MODE>
__global__ __launch_bounds__(256) void relpos_pair_fwd_kernel(const RpArgs a, int tile_k, int vecs, uint32_t vec_magic) {
  __shared__ int edges[rp_lds_words(MODE)];
  const int q = blockIdx.y + blockIdx.z * 65535, k0 = blockIdx.x * tile_k;
  if (q >= a.n_q) return;
  const int nk = min(tile_k, a.n_k - k0), total = nk * vecs;
  const long long base = (long long)q * a.ld + (long long)k0 * a.c;
  const T* add = (const T*)a.add;
  T* out = (T*)a.out;
  Raw<T, V> ad[U];
  int e[U], k[U], pk[U], sk[U];
#pragma unroll
  for (int u = 0; u < U; u++) {
    e[u] = min((int)threadIdx.x + 256 * u, total - 1);     // lanes behind the end repeat the last vector
    k[u] = vec_magic ? (int)__umulhi((uint32_t)e[u], vec_magic) : e[u];
    pk[u] = a.pos_k[k0 + k[u]];
    sk[u] = a.seg_q ? a.seg_k[k0 + k[u]] : 0;
  }
  auto slot = [&](int u) { return Slot<V, WHOLE>(e[u] - k[u] * vecs, a.c); };
  if (add)
#pragma unroll
    for (int u = 0; u < U; u++) ad[u] = slot(u).load(add + base + k[u] * a.c);
  const int pq = a.pos_q[q], sq = a.seg_q ? a.seg_q[q] : 0;
  if constexpr (MODE != RP_DENSE) {
    RpBuckets<MODE>::fill(edges, a);
    __syncthreads();
  }
  const RpBuckets<MODE> rb(edges, a);
  float t[U][V];
#pragma unroll
  for (int u = 0; u < U; u++) load_f32<V>(a.table + (long long)rb.of(pq, pk[u], sq, sk[u]) * a.c + slot(u).at, t[u]);
#pragma unroll
  for (int u = 0; u < U; u++) {
    Raw<T, V> o;
#pragma unroll
    for (int i = 0; i < V; i++) o.set(i, add ? ad[u].get(i) + t[u][i] : t[u][i]);
    if ((int)threadIdx.x + 256 * u < total) slot(u).store(out + base + k[u] * a.c, o);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// HEADS, forward: a workgroup has one q, 256 V positions k and `heads` heads, whose table columns lie in LDS as [head][bucket]
// (neighbouring distances are neighbouring banks).  A lane finds its V buckets once for all heads.
// ---------------------------------------------------------------------------------------------------------------------
template <typename T, int V, bool WHOLE, int MODE>
__global__ __launch_bounds__(256) void relpos_heads_fwd_kernel(const RpArgs a, int heads, int rows) {
  extern __shared__ float tab[];       // [heads][nb]
  __shared__ int edges[rp_lds_words(MODE)];
  const int h0 = blockIdx.z * heads, nh = min(heads, a.c - h0);
  const Slot<V, WHOLE> sl(blockIdx.x * 256 + threadIdx.x, a.n_k);
  RpBuckets<MODE>::fill(edges, a);
  for (int i = threadIdx.x; i < nh * a.nb; i += 256) {
    const int b = i / nh, h = i - b * nh;
    tab[h * a.nb + b] = a.table[(long long)b * a.c + h0 + h];
  }
  __syncthreads();
  if (!sl.in) return;
  const RpBuckets<MODE> rb(edges, a);
  const RpLane<V> at(a, sl.at);
  const T* add = (const T*)a.add;
  T* out = (T*)a.out;
  for (int q = blockIdx.y * rows; q < min(a.n_q, (int)(blockIdx.y + 1) * rows); q++) {
    const int pq = a.pos_q[q], sq = a.seg_q ? a.seg_q[q] : 0, far = at.far(rb, pq, sq);
    int b[V];
    if (far >= 0) {
#pragma unroll
      for (int i = 0; i < V; i++) b[i] = far;
    } else {
#pragma unroll
      for (int i = 0; i < V; i++) b[i] = rb.of(pq, at.pos[i], sq, at.seg[i]);
    }
    const bool all_far = V > 1 && __all(far >= 0);       // of the wave: one table entry per lane and head
    for (int h = 0; h < nh; h++) {
      const long long o_at = ((long long)(h0 + h) * a.n_q + q) * a.ld;
      Raw<T, V> o, ad;
      if (add) ad = sl.load(add + o_at);
      float t[V];
      if (all_far) {
        const float one = tab[h * a.nb + far];
#pragma unroll
        for (int i = 0; i < V; i++) t[i] = one;
      } else {
#pragma unroll
        for (int i = 0; i < V; i++) t[i] = tab[h * a.nb + b[i]];
      }
#pragma unroll
      for (int i = 0; i < V; i++) o.set(i, add ? ad.get(i) + t[i] : t[i]);
      sl.store(out + o_at, o);
    }
  }
}

// v is added to an LDS word that belongs to this lane alone, by a read and a write: the LDS operations of a wave execute in order, so
// the sum's order is the program's.  An LDS atomic took 200 cycles of a CU per 64 lanes (heads 2048 x 2048 x 16: 341 us).
PE_DEV void lds_add(float* p, float v) { *p += v; }

// ---------------------------------------------------------------------------------------------------------------------
// PAIR, backward.  Lane = channel; a wave walks over positions and adds each to the LDS word [bucket][lane] of its own
// accumulators.  Neighbouring positions of the same bucket (all that are farther than the outermost edges) are added in a register
// first, which the whole wave decides together where it has one position at a time.  S positions share a wave where c <= 32.
// blockIdx.y: slab of 64 channels (S = 1).  NEAR: offsets of d_out in bytes fit 32 bits, which
// halves the instructions of a load.  A batch of loads is in flight per wave; lanes behind the last channel or position load a valid one,
// since a load under a condition is waited for by itself.  For what the kernel below does not take: rows with gaps (384 x 384 x 128 bf16 with the
// sums 21.3 us, the kernel below 19.2 without gaps) and up to 16 channels (384 x 384 x 16: 11.7).
// ---------------------------------------------------------------------------------------------------------------------
template <typename T, int S, int U, int MODE, bool NEAR>
__global__ __launch_bounds__(512) void relpos_pair_bwd_kernel(const RpArgs a) {
  extern __shared__ float acc[];       // [waves][nb][64], then the edges
  constexpr int CL = 64 / S, BATCH = U * S;    // lanes per position; positions of a batch
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const int sub = lane / CL, ch = blockIdx.y * 64 + lane % CL;
  int* edges = reinterpret_cast<int*>(acc + waves * a.nb * 64);
  float* mine = acc + wave * a.nb * 64 + lane;
  const T* g = (const T*)a.d_out + min(ch, a.c - 1);
  const uint32_t ch_bytes = min(ch, a.c - 1) * (uint32_t)sizeof(T);
  const long long n = (long long)a.n_q * a.n_k;
  const long long p1 = n, step = 64LL * waves * gridDim.x;        // the workgroups take 64 positions per wave in turn
  // A wave takes 64 positions, each as many behind the last as there are waves, so that every wave has its share of those whose bucket
  // changes from one to the next.  Lane l finds the place and the distance of the l-th (lanes behind the last repeat it).
  struct Places { int cnt, pq, pk, sq, sk, lo, hi; };
  auto locate = [&](long long p) {
    Places r;
    p = min(p, p1 - 1);                                      // behind the end: any place
    r.cnt = (int)min((long long)64, (p1 - p + waves - 1) / waves);      // p: the first of the wave's
    const int q0 = (int)(p / a.n_k), kk = (int)(p - (long long)q0 * a.n_k);    // of the first position
    const int over = kk + min(lane, r.cnt - 1) * waves, dq = over / a.n_k, q = q0 + dq, k = over - dq * a.n_k;
    r.pq = a.pos_q[q];
    r.pk = a.pos_k[k];
    r.sq = a.seg_q ? a.seg_q[q] : 0;
    r.sk = a.seg_q ? a.seg_k[k] : 0;
    const long long row = ((long long)q * a.ld + (long long)k * a.c) * (NEAR ? (int)sizeof(T) : 1);   // the position's offset in d_out
    r.lo = (int)(uint32_t)(uint64_t)row;
    r.hi = (int)(uint32_t)((uint64_t)row >> 32);
    return r;
  };
  T next[U];
  auto load = [&](int lo, int hi, int j) {
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int l = j + u * S + sub;
      const uint32_t x = S == 1 ? (uint32_t)__builtin_amdgcn_readlane(lo, l) : (uint32_t)__shfl(lo, l, 64);
      if constexpr (NEAR) {
        next[u] = *reinterpret_cast<const T*>((const char*)a.d_out + (x + ch_bytes));
      } else {
        const uint32_t y = S == 1 ? (uint32_t)__builtin_amdgcn_readlane(hi, l) : (uint32_t)__shfl(hi, l, 64);
        next[u] = g[(long long)(((uint64_t)y << 32) | x)];
      }
    }
  };
  long long p = 64LL * waves * blockIdx.x + wave;
  Places now;
  if (p < p1) { now = locate(p); load(now.lo, now.hi, 0); }      // on their way while the accumulators are cleared
  RpBuckets<MODE>::fill(edges, a);
  for (int i = threadIdx.x * 4; i < waves * a.nb * 64; i += blockDim.x * 4) *reinterpret_cast<f32x4*>(acc + i) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  __syncthreads();
  const RpBuckets<MODE> rb(edges, a);
  while (p < p1) {
    const int b = rb.of(now.pq, now.pk, now.sq, now.sk), cnt = now.cnt;
    const uint64_t change = S == 1 ? __ballot(b != __shfl_up(b, 1, 64)) : 0;   // lane 0 compares with itself
    int run = __builtin_amdgcn_readlane(b, 0);                                 // S = 1: bucket of the run that is being added up
    float sum = 0.0f;
    p += step;
    Places then = now;
    if (p < p1) then = locate(p);
    // batches: while one is added up the next is on its way, the first of the next 64 behind the last.  The loop stays a loop: its
    // 64 positions written out one after the other are 10 KB of instructions that every workgroup fetches anew.
#pragma unroll 1
    for (int j = 0; j < cnt; j += BATCH) {
      T v[U];
#pragma unroll
      for (int u = 0; u < U; u++) v[u] = next[u];
      const bool more = j + BATCH < cnt;
      if (more || p < p1) load(more ? now.lo : then.lo, more ? now.hi : then.hi, more ? j + BATCH : 0);
      if constexpr (S == 1) {
#pragma unroll
        for (int u0 = 0; u0 < U; u0 += 8) {
          if (j + u0 + 8 <= cnt && ((change >> (j + u0)) & 255) == 0) {        // most: all far from the outermost edges
            sum += (((float)v[u0] + (float)v[u0 + 1]) + ((float)v[u0 + 2] + (float)v[u0 + 3])) +
                   (((float)v[u0 + 4] + (float)v[u0 + 5]) + ((float)v[u0 + 6] + (float)v[u0 + 7]));
          } else {
#pragma unroll
            for (int u = u0; u < u0 + 8; u++) {
              if (j + u < cnt) {
                const int bb = __builtin_amdgcn_readlane(b, j + u);
                if (bb != run) { lds_add(mine + run * 64, sum); run = bb; sum = 0.0f; }
                sum += (float)v[u];
              }
            }
          }
        }
      } else {
#pragma unroll
        for (int u = 0; u < U; u++) {
          const int l = j + u * S + sub, bb = __shfl(b, l, 64);
          if (l < cnt) lds_add(mine + bb * 64, (float)v[u]);
        }
      }
    }
    if constexpr (S == 1) lds_add(mine + run * 64, sum);
    now = then;
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
// PAIR, backward, on the matrix unit: d_table[32 buckets][32 channels] += H D with H[bucket][position] = 1 where the position is in the
// bucket, 0 elsewhere, and D = d_out[position][channel], 16 positions at a time.  The products are exact, sums fp32;
// blocks of 32 buckets without a position among the 16 are left out.  In bf16 buckets in any order cost the same (1024 x 1024 x 128: 54.9 us in the
// order of a sequence, 56.0 mixed); in fp32, where a product takes eight times the instructions, mixed ones twice as much (93 and 187).  A wave has 64 channels, two neighbouring ones
// per lane (a load of the wave is two positions' 128 or 256 bytes),
// and every 8th batch of 16 positions; its sums stay in registers.
// 0 times infinity is NaN: a value that is not finite makes sums of other buckets NaN too, and a workgroup that finds such a sum in the
// end forms all of its sums again without products, position by position: with one NaN 384 x 384 x 128 takes 0.56 ms instead of 0.02, 1024 x 1024 x 128 4.5
// instead of 0.05.
// ---------------------------------------------------------------------------------------------------------------------
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32_any __attribute__((aligned(2)));
// Two channels of 8 positions of a lane: their products with H, given the positions' buckets as bytes
template <typename T> struct RpPairs;
template <> struct RpPairs<bf16> {
  static constexpr int DEPTH = 4;         // batches in flight
  uint32_t x[8];
  template <bool NT> PE_DEV void load(int i, const bf16* p) { x[i] = load_as<NT>(reinterpret_cast<const u32_any*>(p)); }
  PE_DEV void add(f32x16 (&acc)[2], uint2 bytes, uint32_t row) const {
    const uint32_t y[2] = {bytes.x ^ (row * 0x01010101u), bytes.y ^ (row * 0x01010101u)};      // 0 where the bucket is this row's
    union { uint32_t u[4]; bf16x8 f; } h, lo, hi;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const uint32_t two = __builtin_amdgcn_perm(0u, y[i >> 1], (i & 1) ? 0x0c030c02u : 0x0c010c00u);   // two bytes as 16-bit halves
      const u16x2 off = __builtin_elementwise_min(__builtin_bit_cast(u16x2, two), u16x2{1, 1});
      h.u[i] = __builtin_bit_cast(uint32_t, (u16x2)(u16x2{0x3f80, 0x3f80} - off * (uint16_t)0x3f80));   // 1.0 or 0
      lo.u[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x05040100u);
      hi.u[i] = __builtin_amdgcn_perm(x[2 * i + 1], x[2 * i], 0x07060302u);
    }
    Mma<bf16>::mma(acc[0], h.f, lo.f);
    Mma<bf16>::mma(acc[1], h.f, hi.f);
  }
};
template <> struct RpPairs<float> {
  static constexpr int DEPTH = 2;
  f32x2 x[8];
  template <bool NT> PE_DEV void load(int i, const float* p) { x[i] = load_as<NT>(reinterpret_cast<const f32x2_any*>(p)); }
  PE_DEV void add(f32x16 (&acc)[2], uint2 bytes, uint32_t row) const {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const uint32_t b = ((i < 4 ? bytes.x : bytes.y) >> (8 * (i & 3))) & 255u;
      const float h = b == row ? 1.0f : 0.0f;
      Mma<float>::mma(acc[0], h, x[i][0]);
      Mma<float>::mma(acc[1], h, x[i][1]);
    }
  }
};

// NB: blocks of 32 buckets, from 32 NB blockIdx.z on (what a wave's registers hold: more than 128 buckets are two workgroups' that both read
// d_out: 201 buckets over 384 x 384 x 128 with the sums 40 us, by the kernel above 66).  LDS: [4][NB * 32][64] sums, 64 bytes of buckets per wave, the edges.  c >= 2, n_q n_k >= 16.
template <typename T, int NB, int MODE, bool NT>
__global__ __launch_bounds__(512) void relpos_pair_bwd_mm_kernel(const RpArgs a) {
  extern __shared__ float lds[];
  constexpr int ROWS = NB * 32, D = RpPairs<T>::DEPTH;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, half = lane >> 5;
  uint8_t* bytes = reinterpret_cast<uint8_t*>(lds + 4 * ROWS * 64) + wave * 64;
  int* edges = reinterpret_cast<int*>(lds + 4 * ROWS * 64 + 128);
  const int b0 = ROWS * blockIdx.z, nb = min(ROWS, a.nb - b0);
  const int ch0 = blockIdx.y * 64, ch = min(ch0 + 2 * col, a.c - 2);           // lanes behind the last channels load those two
  const long long n = (long long)a.n_q * a.n_k;
  const int* seg_q = a.seg_q ? a.seg_q : a.pos_q;            // without segments: loaded and not used
  const int* seg_k = a.seg_q ? a.seg_k : a.pos_k;
  // The workgroups take 128 positions (16 per wave) in turn.  A wave's round is four of its batches; lane l has the place of position
  // l % 16 of batch l / 16, and steps from round to round without a division.
  const int apart = 128 * gridDim.x, step = 4 * apart;
  const long long p0 = 128LL * blockIdx.x;
  long long p = p0 + 16 * wave;
  const int mine_at = apart * (lane >> 4) + (lane & 15);
  int q, k;
  {
    const long long q0 = min(p, n - 1) / a.n_k, over = min(p, n - 1) - q0 * a.n_k + mine_at;
    const int dq = (int)(over / a.n_k);
    q = (int)q0 + dq;
    k = (int)(over - (long long)dq * a.n_k);
  }
  const int step_q = step / a.n_k, step_k = step % a.n_k;
  struct Places { int pq, pk, sq, sk; };
  auto places = [&]() {                                      // q may be behind the end: any place then
    const int r = min(q, a.n_q - 1);
    return Places{a.pos_q[r], a.pos_k[k], seg_q[r], seg_k[k]};
  };
  // A batch's positions, of which lane half h has 8 h + 0..7.  A batch that reaches behind the end is the last 16 positions instead.  Every
  // round issues the same loads, needed or not: after a load under a condition the compiler waits for all that came before it, and
  // the batches in flight are lost.
  RpPairs<T> v[D];
  const uint32_t lane_bytes = (uint32_t)(8 * half * a.c + ch) * (uint32_t)sizeof(T);
  auto load = [&](RpPairs<T>& to, long long p) {
    const char* at = (const char*)a.d_out + min(p, n - 16) * a.c * (long long)sizeof(T);
#pragma unroll
    for (int i = 0; i < 8; i++) to.template load<NT>(i, reinterpret_cast<const T*>(at + (long long)(i * a.c) * (int)sizeof(T) + lane_bytes));
  };
  // requested in the order in which the loop requests them, which the compiler is held to: what it waits for at the top of a round
  // is what has to be there in every round (with the places requested last it waited for all loads, every round)
  Places now = places();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int j = 0; j < D; j++) load(v[j], p + apart * j);
  asm volatile("" ::: "memory");
  if constexpr (MODE != RP_DENSE) {
    RpBuckets<MODE>::fill(edges, a);
    __syncthreads();
  }
  const RpBuckets<MODE> rb(edges, a);
  f32x16 acc[NB][2];
#pragma unroll
  for (int k = 0; k < NB; k++)
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int e = 0; e < 16; e++) acc[k][t][e] = 0.0f;
  for (; p < n; p += step) {
    const bool in = p + mine_at < n;
    const int b = rb.of(now.pq, now.pk, a.seg_q ? now.sq : 0, a.seg_q ? now.sk : 0) - b0;      // as a byte outside of 0..127: no row here
    const long long behind = p + apart * (lane >> 4) + 16 - n;
    const int shift = behind > 0 ? (int)min(behind, 16LL) : 0;                 // places that the batch was moved down by
    bytes[lane] = 255;                                       // no row
    RowsPiece::phase();
    if (in && (lane & 15) + shift < 16) bytes[lane + shift] = (uint8_t)b;
    uint64_t has[NB];
#pragma unroll
    for (int k = 0; k < NB; k++) has[k] = __ballot(in && (b >> 5) == k);
    q += step_q;
    k += step_k;
    if (k >= a.n_k) { k -= a.n_k; q++; }
    now = places();
    asm volatile("" ::: "memory");
    RowsPiece::phase();                                      // the bytes are in LDS before they are read
#pragma unroll
    for (int j = 0; j < 4; j++) {
      RpPairs<T>& d = v[j % D];
      const uint2 bb = *reinterpret_cast<const uint2*>(bytes + 16 * j + 8 * half);
#pragma unroll
      for (int k = 0; k < NB; k++)
        if ((has[k] >> (16 * j)) & 0xffff) d.add(acc[k], bb, 32 * k + col);
      load(d, p + apart * (j + D));
    }
    RowsPiece::phase();                                      // ... and read before the next ones
  }
  bool odd = false;
#pragma unroll
  for (int k = 0; k < NB; k++)
#pragma unroll
    for (int t = 0; t < 2; t++)
#pragma unroll
      for (int e = 0; e < 16; e++) odd = odd || (__float_as_uint(acc[k][t][e]) & 0x7f800000u) == 0x7f800000u;
  // the upper four waves' sums go to LDS, the lower four add theirs, then one sum over four
  float* sums = lds + (wave & 3) * ROWS * 64;
  auto at = [&](int k, int t, int e) { return (32 * k + acc_row(half, e)) * 64 + ch + t - ch0; };
  // lanes behind the last channel have none of their own; of an odd number of channels the last lane has the second of its pair
  const bool mine[2] = {ch == ch0 + 2 * col, ch == ch0 + 2 * col || ch0 + 2 * col == a.c - 1};
  for (int up = 1; up >= 0; up--) {
    if (wave >> 2 == up)
#pragma unroll
      for (int k = 0; k < NB; k++)
#pragma unroll
        for (int t = 0; t < 2; t++)
          if (mine[t])
#pragma unroll
            for (int e = 0; e < 16; e++) {
              float* to = sums + at(k, t, e);
              *to = up ? acc[k][t][e] : acc[k][t][e] + *to;
            }
    __syncthreads();
  }
  float* part = a.part + ((long long)blockIdx.x * a.nb + b0) * a.c + ch0;
  auto each = [&](auto&& f) {
    for (int i = threadIdx.x; i < nb * 64; i += 512) if (ch0 + (i & 63) < a.c) f(i, part + (long long)(i >> 6) * a.c + (i & 63));
  };
  each([&](int i, float* to) { *to = (lds[i] + lds[i + ROWS * 64]) + (lds[i + 2 * ROWS * 64] + lds[i + 3 * ROWS * 64]); });
  if (!__syncthreads_or(odd)) return;
  // again, lane = channel: every wave goes through all positions and adds those of its buckets (every 8th) to words that are its alone
  for (int i = threadIdx.x; i < ROWS * 64; i += 512) lds[i] = 0.0f;
  __syncthreads();
  const T* column = (const T*)a.d_out + min(ch0 + lane, a.c - 1);
  for (long long from = p0; from < n; from += apart)
    for (p = from; p < min(n, from + 128); p++) {
      const int pos = (int)(p / a.n_k), other = (int)(p - (long long)pos * a.n_k);
      const int b = rb.of(a.pos_q[pos], a.pos_k[other], a.seg_q ? a.seg_q[pos] : 0, a.seg_q ? a.seg_k[other] : 0) - b0;
      if (b >= 0 && b < nb && (b & 7) == wave) lds_add(lds + b * 64 + lane, (float)column[p * a.c]);
    }
  __syncthreads();
  each([&](int i, float* to) { *to = lds[i]; });
}

// ---------------------------------------------------------------------------------------------------------------------
// HEADS, backward.  Lane = V positions k; a wave walks over rows q of one head, U at a time, spread over all rows so that every wave has its
// share of those near its positions (which cost several times the others), and adds to the LDS words
// [bucket][lane] of its own accumulators (bank = lane whatever the buckets are).  Most lanes' positions are all farther than the outermost
// edges, which their extremes tell: V elements are then one addition to LDS and no bucket is looked up.
// ---------------------------------------------------------------------------------------------------------------------
template <typename T, int V, bool WHOLE, int U, int MODE, bool NT>
__global__ __launch_bounds__(512) void relpos_heads_bwd_kernel(const RpArgs a) {
  extern __shared__ float acc[];       // [waves][nb][64], then the edges
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  int* edges = reinterpret_cast<int*>(acc + waves * a.nb * 64);
  float* mine = acc + wave * a.nb * 64 + lane;
  RpBuckets<MODE>::fill(edges, a);
  for (int i = threadIdx.x; i < waves * a.nb * 64; i += blockDim.x) acc[i] = 0.0f;
  __syncthreads();
  const RpBuckets<MODE> rb(edges, a);
  const int h = blockIdx.z;
  const Slot<V, WHOLE> sl(blockIdx.x * 64 + lane, a.n_k);
  const int step = gridDim.y * waves;                      // rows between a wave's
  if (sl.in) {
    const RpLane<V> at(a, sl.at);
    const T* g = (const T*)a.d_out + (long long)h * a.n_q * a.ld;
    Raw<T, V> next[U];
    auto fetch = [&](int q) {
#pragma unroll
      for (int u = 0; u < U; u++) next[u] = sl.template load<NT>(g + (long long)min(q + u * step, a.n_q - 1) * a.ld);
    };
    int q = blockIdx.y * waves + wave;
    if (q < a.n_q) fetch(q);
    for (; q < a.n_q; q += U * step) {
      Raw<T, V> v[U];
#pragma unroll
      for (int u = 0; u < U; u++) v[u] = next[u];
      if (q + U * step < a.n_q) fetch(q + U * step);
#pragma unroll
      for (int u = 0; u < U; u++) {
        const int qu = q + u * step;
        if (qu >= a.n_q) break;
        const int pq = a.pos_q[qu], sq = a.seg_q ? a.seg_q[qu] : 0;
        const int far = at.far(rb, pq, sq);
        if (far >= 0) {
          float sum = sl.has(0) ? v[u].get(0) : 0.0f;
#pragma unroll
          for (int i = 1; i < V; i++) sum += sl.has(i) ? v[u].get(i) : 0.0f;
          lds_add(mine + far * 64, sum);
        } else {
          int b[V];
#pragma unroll
          for (int i = 0; i < V; i++) b[i] = rb.of(pq, at.pos[i], sq, at.seg[i]);
#pragma unroll
          for (int i = 0; i < V; i++) lds_add(mine + b[i] * 64, sl.has(i) ? v[u].get(i) : 0.0f);
        }
      }
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
