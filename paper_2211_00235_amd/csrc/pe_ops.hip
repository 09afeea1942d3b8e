// Operators around the block: layer norm, relative position embedding, activation checkpoints in 8 bits (see include/pe.h).
// Host side: argument checks, the choice of kernel variants, launches.
#include <stdio.h>
#include <string.h>
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "pe_ckpt.h"
#include "pe_handle.h"
#include "pe_ln.h"
#include "pe_ops.h"
#include "pe_relpos.h"

namespace {

// One call of an operator: refusals with a text, launches with the handle's timing and checking options.
struct OpCall {
  pe_handle* h;
  hipStream_t st;
  int err = PE_OK;
  int refuse(int code, const char* text) {
    h->last_error = text;
    return code;
  }
  // the current device is the handle's: the kernels are launched there, on a stream of it
  bool device_ok() {
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) { (void)hipGetLastError(); return false; }
    return dev == h->device;
  }
  hipEvent_t event() {
    hipEvent_t e;
    if (!h->ev_pool.empty()) { e = h->ev_pool.back(); h->ev_pool.pop_back(); return e; }
    if (hipEventCreate(&e) != hipSuccess) return nullptr;
    return e;
  }
  template <typename F> void launch(const char* label, const char* kern, double flops, double bytes, F&& f) {
    if (err) return;
    hipEvent_t e0 = nullptr, e1 = nullptr;
    if (h->timing && (e0 = event())) (void)hipEventRecord(e0, st);
    f();
    if (e0 && (e1 = event())) {
      (void)hipEventRecord(e1, st);
      h->recs.push_back(ProfRec{label, kern, flops, bytes, e0, e1});
    }
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && h->sync_debug) e = hipStreamSynchronize(st);
    if (e != hipSuccess) {
      err = PE_ERR_HIP;
      h->last_error = std::string(label) + ": " + hipGetErrorString(e);
    }
  }
};

// An entry point's body: nothing thrown (the host has run out of memory) passes the C boundary
template <typename F> int guarded(F&& f) {
  try { return f(); } catch (...) { return PE_ERR_HIP; }
}

size_t elem(int dtype) { return dtype == PE_BF16 ? 2 : 4; }
bool type_ok(int dtype) { return dtype == PE_F32 || dtype == PE_BF16; }
size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }
bool aligned(const void* p, size_t a) { return ((uintptr_t)p) % a == 0; }
// bytes from the first to the last element of [rows][c] with row stride ld
size_t span(long long rows, long long c, long long ld, size_t e) { return rows > 0 && c > 0 ? ((size_t)(rows - 1) * ld + c) * e : 0; }

// WHOLE: rows of whole 8-element vectors, all of them aligned for 16-byte accesses
struct Whole {
  bool ok;
  size_t e;
  Whole(long long c, size_t elem_bytes) : ok(c % 8 == 0), e(elem_bytes) {}
  Whole& take(const void* p, long long ld, long long rows) {
    if (p && (!aligned(p, 16) || (rows > 1 && (ld * (long long)e) % 16))) ok = false;
    return *this;
  }
};
// calls `f` with V and WHOLE as template arguments: rows of fewer than 8 elements an element at a time
template <typename F> void width_dispatch(long long c, bool whole, F&& f) {
  if (c < 8) f(std::integral_constant<int, 1>{}, std::true_type{});
  else if (whole) f(std::integral_constant<int, 8>{}, std::true_type{});
  else f(std::integral_constant<int, 8>{}, std::false_type{});
}
// Non-temporal loads of a tensor that a call reads once: from 32 MB on (an eighth of the memory-side cache).  With and without, us:
// relpos pair backward 17 MB of gradients 12.9 and 11.5.  Behind a forward pass, which in turn finds less of itself in the cache: 67 MB
// backward 18.2 and 23.7, forward 26.4 and 23.9, 268 MB 50.8 and 80.4, 91.8 and 78.9; both passes and the sums 38 MB 31.9 and 36.8, 67 MB 49.1 and 51.6,
// 134 MB 81.5 and 88.1, 268 MB 146 and 160.  Heads 134 MB, both passes, 64.3 and 68.2; packing and restoring 17 MB 13.5 and
// 13.1, 126 MB 65.0 and 74.2, 252 MB 134 and 141.  Layer norm stays without: its backward pass finds part of what the forward pass has read (29 MB fp32,
// both passes, 38.2 and 34.5, 67 MB bf16 90.1 and 87.6).
template <typename F> void stream_dispatch(double bytes, F&& f) {
  if (bytes >= 32e6) f(std::true_type{}); else f(std::false_type{});
}
template <typename F> void type_dispatch(int dtype, F&& f) {
  if (dtype == PE_BF16) f(bf16{}); else f(float{});
}

constexpr int LN_MAX_C = 16384;
constexpr long long MAX_ROWS = 1LL << 40;
constexpr int CK_MAX_C = 1 << 20;

// ---------------------------------------------------------------------------------------------------------------------
// 8-bit checkpoints
// ---------------------------------------------------------------------------------------------------------------------
long long ck_groups(int c) { return (c + CK_GROUP - 1) / CK_GROUP; }
size_t ck_bytes(long long rows, int c) { return up256((size_t)rows * c) + (size_t)rows * ck_groups(c); }

template <bool PACK> void ck_run(hipStream_t st, int dtype, bool whole, const void* x, long long ld, void* ckpt, void* y, long long rows, int c) {
  type_dispatch(dtype, [&](auto t) {
    using T = decltype(t);
    width_dispatch(c, whole, [&](auto v, auto w) {
      constexpr int V = v.value, U = 4;
      const int per_row = V == 8 ? (int)ck_groups(c) * 4 : 8;
      const long long items = rows * per_row, blocks = (items + 256 * U - 1) / (256 * U);
      const dim3 grid((unsigned)std::min<long long>(blocks, CK_GRID_X), (unsigned)((blocks + CK_GRID_X - 1) / CK_GRID_X));
      auto launch = [&](auto nt) {
        hipLaunchKernelGGL((ckpt_kernel<T, V, w.value, U, PACK, nt.value>), grid, dim3(256), 0, st, (const T*)x, ld, (int8_t*)ckpt,
                           (uint8_t*)ckpt + up256((size_t)rows * c), (T*)y, rows, c, per_row, (int)(c % CK_GROUP == 0 && (ld == c || rows == 1)));
      };
      if constexpr (PACK) stream_dispatch((double)rows * c * sizeof(T), launch); else launch(std::false_type{});
    });
  });
}

int ck_call(pe_handle* h, long long rows, int c, int dtype, const void* t, long long ld, const void* ckpt, bool pack, void* stream) {
  if (!h) return PE_ERR_NULL;
  OpCall op{h, (hipStream_t)stream};
  if (rows < 0 || rows > MAX_ROWS || c < 1 || c > CK_MAX_C || !type_ok(dtype) || (double)rows * c > 1e12)
    return op.refuse(PE_ERR_DIMS, "checkpoint: rows in [0, 2^40], c in [1, 2^20], rows * c up to 10^12, dtype PE_F32 or PE_BF16");
  if (ld < c) return op.refuse(PE_ERR_ARG, "checkpoint: a row stride is less than c");
  if (rows == 0) return PE_OK;
  if (!t || !ckpt) return op.refuse(PE_ERR_NULL, "checkpoint: null tensor");
  const size_t e = elem(dtype);
  if (!aligned(t, e) || !aligned(ckpt, 256)) return op.refuse(PE_ERR_ARG, "checkpoint: a tensor is not aligned to its elements, or the checkpoint not to 256 bytes");
  const Region rg[] = {{t, span(rows, c, ld, e), !pack}, {ckpt, ck_bytes(rows, c), pack}};
  if (any_alias(rg, 2)) return op.refuse(PE_ERR_ALIAS, "checkpoint: tensor and checkpoint overlap");
  if (!op.device_ok()) return op.refuse(PE_ERR_ARG, "checkpoint: the handle belongs to another device than the current one");
  const bool whole = Whole(c, e).take(t, ld, rows).ok;
  const double n = (double)rows * c;
  op.launch(pack ? "ckpt pack" : "ckpt unpack", "ckpt_kernel", 2 * n, n * e + ck_bytes(rows, c), [&] {
    if (pack) ck_run<true>(op.st, dtype, whole, t, ld, const_cast<void*>(ckpt), nullptr, rows, c);
    else ck_run<false>(op.st, dtype, whole, nullptr, ld, const_cast<void*>(ckpt), const_cast<void*>(t), rows, c);
  });
  return op.err;
}

// ---------------------------------------------------------------------------------------------------------------------
// Layer norm
// ---------------------------------------------------------------------------------------------------------------------
// Lanes and vectors per lane of a row of c channels
struct LnPlan { int l, nv; int rows() const { return l > 256 ? 1 : 256 / l; } };
LnPlan ln_plan(int c) {
  if (c < 8) return {8, 1};
  const int n = (c + 7) / 8;
  if (n <= 4) return {4, 1};
  if (n <= 8) return {8, 1};
  if (n <= 16) return {16, 1};
  if (n <= 32) return {32, 1};
  if (n <= 64) return {64, 1};
  if (n <= 128) return {64, 2};
  if (n <= 512) return {256, 2};
  if (n <= 1024) return {512, 2};
  return {1024, 2};
}
// Most workgroups of a launch: they walk over the rows.  Forward with 1024, 2048 and 4096, us: 28677 x 256 fp32 11.9, 11.6 and 11.2, 196608 x 256 bf16
// 40.1, 39.6 and 39.6; rows of whole workgroups, which load gain and offset for a few rows only, 4096 x 8192 30.4, 31.0 and 35.8, 2048 x 16384 38.2,
// 41.5 and 41.7.  Backward, each writes 8 c bytes of partial sums: four per CU of rows within waves (the chip holds as many up to 512 channels; of
// 64 lanes with two vectors each, 159 and 186 registers, three in bf16 and two in fp32), two or one of rows of whole workgroups (4096 x 8192 with 512 of
// them 60 us and 11 for the sums, with 256 49 and 7).
constexpr int LN_FWD_WG = 2048, LN_BWD_WG = 1024;
long long ln_bwd_groups(long long rows, int c) {
  const LnPlan p = ln_plan(c);
  return std::min<long long>((rows + p.rows() - 1) / p.rows(), p.l <= 64 ? LN_BWD_WG : p.l == 256 ? 512 : 256);
}

// calls `f` with the plan's template arguments
template <typename F> void ln_dispatch(const LnPlan& p, F&& f) {
#define PE_LN_CASE(L, NV) if (p.l == L && p.nv == NV) return f(std::integral_constant<int, L>{}, std::integral_constant<int, NV>{})
  PE_LN_CASE(4, 1); PE_LN_CASE(8, 1); PE_LN_CASE(16, 1); PE_LN_CASE(32, 1); PE_LN_CASE(64, 1);
  PE_LN_CASE(64, 2); PE_LN_CASE(256, 2); PE_LN_CASE(512, 2); PE_LN_CASE(1024, 2);
#undef PE_LN_CASE
}
template <typename T, int V, bool WHOLE> void ln_fwd_run(hipStream_t st, const LnArgs& a) {
  auto launch = [&](auto l, auto nv) {
    constexpr int L = l.value;
    const long long wg = (a.rows + LnShape<L>::ROWS - 1) / LnShape<L>::ROWS;
    hipLaunchKernelGGL((ln_op_fwd_kernel<T, V, WHOLE, L, nv.value>), dim3((unsigned)std::min<long long>(wg, LN_FWD_WG)), dim3(LnShape<L>::THREADS), 0, st, a);
  };
  if constexpr (V == 1) launch(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
  else ln_dispatch(ln_plan(a.c), launch);
}
template <typename T, int V, bool WHOLE> void ln_bwd_run(hipStream_t st, const LnArgs& a, unsigned wg) {
  auto launch = [&](auto l, auto nv) {
    constexpr int L = l.value;
    if (a.codes) hipLaunchKernelGGL((ln_op_bwd_kernel<T, V, WHOLE, L, nv.value, true>), dim3(wg), dim3(LnShape<L>::THREADS), 0, st, a);
    else hipLaunchKernelGGL((ln_op_bwd_kernel<T, V, WHOLE, L, nv.value, false>), dim3(wg), dim3(LnShape<L>::THREADS), 0, st, a);
  };
  if constexpr (V == 1) launch(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
  else ln_dispatch(ln_plan(a.c), launch);
}
void columns_sum(OpCall& op, const char* label, const float* part, long long n_part, int cols, float* o0, float* o1, int split, bool acc) {
  op.launch(label, "columns_sum_kernel", (double)n_part * cols, 4.0 * ((double)n_part * cols + cols), [&] {
    hipLaunchKernelGGL(columns_sum_kernel, dim3((unsigned)((cols + 15) / 16)), dim3(1024), 0, op.st, part, (int)n_part, cols, o0, o1, split, (int)acc);
  });
}

// ---------------------------------------------------------------------------------------------------------------------
// Relative positions
// ---------------------------------------------------------------------------------------------------------------------
int rp_buckets(const pe_relpos& p) { return p.n_edges + 1 + (p.segments ? 1 : 0); }
const char* rp_why(const pe_relpos& p) {
  if (p.n_q < 0 || p.n_k < 0 || p.n_q > (1 << 24) || p.n_k > (1 << 24)) return "relative positions: n_q and n_k in [0, 2^24]";
  if (p.c < 1 || p.c > 1024) return "relative positions: c in [1, 1024]";
  if ((double)p.n_q * p.n_k * p.c > 1e12) return "relative positions: n_q * n_k * c up to 10^12";
  if (p.n_edges < 0 || p.n_edges > RP_MAX_EDGES) return "relative positions: n_edges in [0, 254]";
  if (p.layout != PE_RELPOS_PAIR && p.layout != PE_RELPOS_HEADS) return "relative positions: layout PE_RELPOS_PAIR or PE_RELPOS_HEADS";
  if (p.segments != 0 && p.segments != 1) return "relative positions: segments 0 or 1";
  if (!type_ok(p.dtype)) return "relative positions: dtype PE_F32 or PE_BF16";
  if (p.ld < 0) return "relative positions: ld at least 0";
  return nullptr;
}
long long rp_row(const pe_relpos& p) { return p.layout == PE_RELPOS_PAIR ? (long long)p.n_k * p.c : p.n_k; }
long long rp_ld(const pe_relpos& p) { return p.ld ? p.ld : rp_row(p); }

// waves per workgroup of the backward kernels: each has accumulators of its own, [buckets][64] in LDS (160 KB, of which the edges
// take up to 4)
int rp_waves(int nb) { return std::max(1, std::min(8, (int)(150 * 1024 / (nb * 256)))); }
size_t rp_lds(int nb, int waves, int mode) { return (size_t)waves * nb * 256 + 4 * rp_lds_words(mode); }
// PAIR: position groups, so many that with slabs of 64 channels there are 256 workgroups.  Partial sums cost 8 bytes per group, bucket
// and channel: a group has at least 512 positions.
long long rp_pair_groups(const pe_relpos& p) {
  const long long n = (long long)p.n_q * p.n_k;
  return std::max<long long>(1, std::min<long long>(256 / ((p.c + 63) / 64), (n + 511) / 512));
}
// HEADS: 64 vectors of 8 positions k (fewer than 8: of one) per workgroup; so many workgroups share the rows q of those and of a head
// that there are about 512, with a row per wave at least.  That is one round of the chip where two fit a CU's LDS, up to about 38 buckets (2048 x 2048 x 16
// with 32 buckets 33 us with the sums); with more there is one per CU, and two rounds or three (65 buckets 37.5; 1021 x 1021 x 12 30.4).
long long rp_heads_tiles(const pe_relpos& p) { return ((p.n_k < 8 ? p.n_k : (p.n_k + 7) / 8) + 63LL) / 64; }
int rp_heads_split(const pe_relpos& p) {
  const long long all = rp_heads_tiles(p) * p.c;
  return (int)std::min<long long>((p.n_q + 7) / 8, std::max<long long>(1, (512 + all - 1) / all));
}
long long rp_heads_groups(const pe_relpos& p) { return rp_heads_tiles(p) * rp_heads_split(p); }
size_t rp_workspace(const pe_relpos& p) {
  if (p.n_q == 0 || p.n_k == 0) return 256;
  return up256((size_t)(p.layout == PE_RELPOS_PAIR ? rp_pair_groups(p) : rp_heads_groups(p)) * rp_buckets(p) * p.c * 4);
}

// The checks that forward and backward share; on PE_OK `a` is filled but for the tensors of the direction
int rp_check(OpCall& op, const pe_relpos* p, const int* edges, const int* pos_q, const int* pos_k, const int* seg_q, const int* seg_k, RpArgs& a) {
  if (!p) return op.refuse(PE_ERR_NULL, "relative positions: null description");
  if (const char* why = rp_why(*p)) return op.refuse(PE_ERR_DIMS, why);
  if (p->ld && p->ld < rp_row(*p)) return op.refuse(PE_ERR_ARG, "relative positions: ld is less than a row");
  if (p->n_edges && !edges) return op.refuse(PE_ERR_NULL, "relative positions: null edges");
  bool dense = true;
  for (int i = 0; i < p->n_edges; i++) {
    if (edges[i] == -2147483647 - 1 || (i && edges[i] <= edges[i - 1])) return op.refuse(PE_ERR_ARG, "relative positions: edges have to ascend, the first above -2^31");
    if (i && edges[i] != edges[i - 1] + 1) dense = false;
    a.edges[i] = edges[i];
  }
  a.lo = p->n_edges ? edges[0] - 1 : 0;
  a.hi = p->n_edges ? edges[p->n_edges - 1] : 0;        // without edges both are 0: every distance is in bucket 0
  a.mode = dense ? RP_DENSE : (long long)a.hi - a.lo < RP_LUT ? RP_LUTS : RP_SEARCH;
  const bool some = p->n_q > 0 && p->n_k > 0;
  if (some && (!pos_q || !pos_k || (p->segments && (!seg_q || !seg_k)))) return op.refuse(PE_ERR_NULL, "relative positions: null positions or segments");
  if (!aligned(pos_q, 4) || !aligned(pos_k, 4) || !aligned(seg_q, 4) || !aligned(seg_k, 4)) return op.refuse(PE_ERR_ARG, "relative positions: a tensor is not aligned to its elements");
  a.pos_q = pos_q; a.pos_k = pos_k;
  a.seg_q = p->segments ? seg_q : nullptr; a.seg_k = p->segments ? seg_k : nullptr;
  a.table = nullptr; a.add = nullptr; a.out = nullptr; a.d_out = nullptr; a.part = nullptr;
  a.ld = rp_ld(*p);
  a.n_q = p->n_q; a.n_k = p->n_k; a.c = p->c; a.nb = rp_buckets(*p); a.n_edges = p->n_edges;
  return PE_OK;
}
size_t rp_span(const pe_relpos& p) {
  return p.layout == PE_RELPOS_PAIR ? span(p.n_q, rp_row(p), rp_ld(p), elem(p.dtype))
                                    : span((long long)p.n_q * p.c, rp_row(p), rp_ld(p), elem(p.dtype));
}

// calls `f` with the mode as a template argument; few: a lane looks up fewer than ten distances
template <typename F> void rp_dispatch(int mode, bool few, F&& f) {
  if (mode == RP_DENSE) f(std::integral_constant<int, RP_DENSE>{});
  else if (mode == RP_LUTS && !few) f(std::integral_constant<int, RP_LUTS>{});
  else f(std::integral_constant<int, RP_SEARCH>{});
}
// the same for kernels whose lanes always look up few
template <typename F> void rp_dispatch_few(int mode, F&& f) {
  if (mode == RP_DENSE) f(std::integral_constant<int, RP_DENSE>{}); else f(std::integral_constant<int, RP_SEARCH>{});
}
template <typename T, int V, bool WHOLE> void rp_pair_fwd(hipStream_t st, const RpArgs& a) {
  constexpr int U = V == 8 ? 4 : 8;
  const int vecs = (a.c + V - 1) / V;
  const int tile = 256 * U / vecs;                       // vecs <= 128 (c <= 1024): several positions
  const unsigned magic = vecs == 1 ? 0u : (unsigned)(((1ull << 32) + vecs - 1) / vecs);     // exact for vectors up to 2^11
  const unsigned gx = (unsigned)((a.n_k + tile - 1) / tile), gy = (unsigned)std::min(a.n_q, 65535), gz = (unsigned)((a.n_q + 65534) / 65535);
  rp_dispatch_few(a.mode, [&](auto m) { hipLaunchKernelGGL((relpos_pair_fwd_kernel<T, V, WHOLE, U, m.value>), dim3(gx, gy, gz), dim3(256), 0, st, a, tile, vecs, magic); });
}
template <typename T, int V, bool WHOLE> void rp_heads_fwd(hipStream_t st, const RpArgs& a) {
  // heads per workgroup: what 32 KB of LDS hold, and few enough that the chip is filled
  const long long tiles = (a.n_k + 256LL * V - 1) / (256LL * V);
  int heads = std::max(1, std::min(a.c, 32 * 1024 / (a.nb * 4)));
  while (heads > 1 && tiles * a.n_q * ((a.c + heads - 1) / heads) < 512) heads = (heads + 1) / 2;
  const unsigned gz = (unsigned)((a.c + heads - 1) / heads);
  // rows per workgroup: the table's copy in LDS is shared by as many rows as leave 512 workgroups
  const long long all = tiles * gz;
  const int rows = (int)std::max<long long>((a.n_q + 65534) / 65535, std::min<long long>(16, a.n_q * all / 512));
  rp_dispatch(a.mode, rows * V < 10, [&](auto m) {
    hipLaunchKernelGGL((relpos_heads_fwd_kernel<T, V, WHOLE, m.value>), dim3((unsigned)tiles, (unsigned)((a.n_q + rows - 1) / rows), gz), dim3(256),
                       (size_t)heads * a.nb * 4, st, a, heads, rows);
  });
}
// Dynamic LDS above 64 KB has to be allowed once per kernel and device; what is left of a CU's 160 KB is for static LDS
constexpr int RP_LDS_MOST = 156 * 1024;
template <typename K> void allow_lds(K kern, int device, std::atomic<unsigned long long>& done) {
  const unsigned long long bit = 1ull << (device & 63);
  if (done.load() & bit) return;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, RP_LDS_MOST) == hipSuccess) done |= bit;
  else (void)hipGetLastError();      // the launch is refused then, and says so
}
template <typename T, int S, int U> void rp_pair_bwd(hipStream_t st, int device, const RpArgs& a, long long groups) {
  const int waves = rp_waves(a.nb);
  rp_dispatch_few(a.mode, [&](auto m) {
    auto launch = [&](auto near) {
      static std::atomic<unsigned long long> done{0};
      allow_lds(&relpos_pair_bwd_kernel<T, S, U, m.value, near.value>, device, done);
      hipLaunchKernelGGL((relpos_pair_bwd_kernel<T, S, U, m.value, near.value>), dim3((unsigned)groups, (unsigned)((a.c + 63) / 64)),
                         dim3(64 * waves), rp_lds(a.nb, waves, m.value), st, a);
    };
    if ((double)a.n_q * (double)a.ld * sizeof(T) < 4e9) launch(std::true_type{}); else launch(std::false_type{});
  });
}
template <typename T, int V, bool WHOLE> void rp_heads_bwd(hipStream_t st, int device, const RpArgs& a, int split) {
  constexpr int U = V == 8 ? 4 : 8;
  const int waves = rp_waves(a.nb);
  rp_dispatch(a.mode, (long long)V * a.n_q < 10LL * split * waves, [&](auto m) {
    stream_dispatch((double)a.n_q * a.n_k * a.c * sizeof(T), [&](auto nt) {
      static std::atomic<unsigned long long> done{0};
      allow_lds(&relpos_heads_bwd_kernel<T, V, WHOLE, U, m.value, nt.value>, device, done);
      hipLaunchKernelGGL((relpos_heads_bwd_kernel<T, V, WHOLE, U, m.value, nt.value>), dim3((unsigned)(((a.n_k + V - 1) / V + 63) / 64), (unsigned)split, (unsigned)a.c),
                         dim3(64 * waves), rp_lds(a.nb, waves, m.value), st, a);
    });
  });
}
// The matrix unit's kernel: rows without gaps, more than 16 channels, a batch of positions at least.  384 x 384 positions with the sums, by it and by the
// kernel without, us: bf16 8 channels 12.0 and 10.7, 16 12.3 and 11.7, 24 12.7 and 16.6, 32 12.7 and 16.3, 48 13.6 and 15.9, 128 19.2 and 21.3, with positions in
// any order 19.7 and 29.4.  fp32 16 channels 18.0 and 11.9, 32 18.0 and 16.5, 128 26.0 and 23.7 (1024 x 1024: 93 and 98), in any order 39.0 and 30.2:
// there the two are near one another where neighbours' distances are alike, and the kernel without is the faster one where they are not.
bool rp_pair_mm(const RpArgs& a) { return a.c > 16 && a.ld == (long long)a.n_k * a.c && (long long)a.n_q * a.n_k >= 16; }
template <typename T, int NB> void rp_pair_bwd_mm(hipStream_t st, int device, const RpArgs& a, long long groups) {
  rp_dispatch_few(a.mode, [&](auto m) {
    stream_dispatch((double)a.n_q * a.n_k * a.c * sizeof(T), [&](auto nt) {
      static std::atomic<unsigned long long> done{0};
      allow_lds(&relpos_pair_bwd_mm_kernel<T, NB, m.value, nt.value>, device, done);
      const size_t lds = (size_t)4 * NB * 32 * 64 * 4 + 512 + 4 * rp_lds_words(m.value);
      hipLaunchKernelGGL((relpos_pair_bwd_mm_kernel<T, NB, m.value, nt.value>), dim3((unsigned)groups, (unsigned)((a.c + 63) / 64), (unsigned)((a.nb + 32 * NB - 1) / (32 * NB))),
                         dim3(512), lds, st, a);
    });
  });
}
template <typename T> void rp_pair_bwd_run(hipStream_t st, int device, const RpArgs& a, long long groups) {
  if (rp_pair_mm(a)) {
    if (a.nb <= 32) rp_pair_bwd_mm<T, 1>(st, device, a, groups);
    else if (a.nb <= 64) rp_pair_bwd_mm<T, 2>(st, device, a, groups);
    else if (a.nb <= 96) rp_pair_bwd_mm<T, 3>(st, device, a, groups);
    else rp_pair_bwd_mm<T, 4>(st, device, a, groups);
  } else if (a.c > 32) rp_pair_bwd<T, 1, 32>(st, device, a, groups);
  else if (a.c > 16) rp_pair_bwd<T, 2, 16>(st, device, a, groups);
  else if (a.c > 8) rp_pair_bwd<T, 4, 16>(st, device, a, groups);
  else rp_pair_bwd<T, 8, 8>(st, device, a, groups);
}

}  // namespace

int ckpt_launch(pe_handle* h, hipStream_t st, bool pack, int dtype, void* x, void* ckpt, long long rows, int c) {
  OpCall op{h, st};
  const double n = (double)rows * c;
  op.launch(pack ? "ckpt pack" : "ckpt unpack", "ckpt_kernel", 2 * n, n * elem(dtype) + ck_bytes(rows, c), [&] {
    if (pack) ck_run<true>(st, dtype, true, x, c, ckpt, nullptr, rows, c); else ck_run<false>(st, dtype, true, nullptr, c, ckpt, x, rows, c);
  });
  return op.err;
}

extern "C" {

int pe_handle_device(const pe_handle* h) { return h ? h->device : PE_ERR_NULL; }

size_t pe_ckpt_bytes(long long rows, int c) {
  if (rows < 0 || rows > MAX_ROWS || c < 1 || c > CK_MAX_C || (double)rows * c > 1e12) return 0;
  return ck_bytes(rows, c);
}
int pe_ckpt_pack(pe_handle* h, long long rows, int c, int dtype, const void* x, long long ld_x, void* ckpt, void* stream) {
  return guarded([&] { return ck_call(h, rows, c, dtype, x, ld_x, ckpt, true, stream); });
}
int pe_ckpt_unpack(pe_handle* h, long long rows, int c, int dtype, const void* ckpt, void* y, long long ld_y, void* stream) {
  return guarded([&] { return ck_call(h, rows, c, dtype, y, ld_y, ckpt, false, stream); });
}

size_t pe_layernorm_workspace_bytes(long long rows, int c) {
  if (rows < 0 || rows > MAX_ROWS || c < 1 || c > LN_MAX_C) return 0;
  return up256((size_t)std::max(1LL, ln_bwd_groups(rows, c)) * 2 * c * 4);
}

int pe_layernorm_fwd(pe_handle* h, long long rows, int c, int dtype, const void* x, long long ld_x, const void* add, long long ld_add,
                     const float* gain, const float* offset, float eps, void* y, long long ld_y, float* stats, void* ckpt, void* stream) {
  return guarded([&]() -> int {
    if (!h) return PE_ERR_NULL;
    OpCall op{h, (hipStream_t)stream};
    if (rows < 0 || rows > MAX_ROWS || c < 1 || c > LN_MAX_C || !type_ok(dtype))
      return op.refuse(PE_ERR_DIMS, "layer norm: rows in [0, 2^40], c in [1, 16384], dtype PE_F32 or PE_BF16");
    if (!(eps > 0.0f)) return op.refuse(PE_ERR_DIMS, "layer norm: eps has to be positive");
    if (ld_x < c || ld_y < c || (add && ld_add < c)) return op.refuse(PE_ERR_ARG, "layer norm: a row stride is less than c");
    if (rows == 0) return PE_OK;
    if (!x || !y) return op.refuse(PE_ERR_NULL, "layer norm: null tensor");
    const size_t e = elem(dtype);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(add, e) || !aligned(gain, 4) || !aligned(offset, 4) || !aligned(stats, 8) || !aligned(ckpt, 256))
      return op.refuse(PE_ERR_ARG, "layer norm: a tensor is not aligned to its elements, stats not to 8 bytes, or the checkpoint not to 256");
    const bool in_place = add == y && ld_add == ld_y;      // y = y + LN(x): every element is read by the lane that writes it
    const Region rg[] = {{x, span(rows, c, ld_x, e), false}, {in_place ? nullptr : add, span(rows, c, ld_add, e), false},
                         {gain, (size_t)c * 4, false}, {offset, (size_t)c * 4, false}, {y, span(rows, c, ld_y, e), true},
                         {stats, (size_t)rows * 8, true}, {ckpt, ck_bytes(rows, c), true}};
    if (any_alias(rg, 7)) return op.refuse(PE_ERR_ALIAS, "layer norm: a buffer that is written overlaps another one");
    if (!op.device_ok()) return op.refuse(PE_ERR_ARG, "layer norm: the handle belongs to another device than the current one");
    LnArgs a{};
    a.x = x; a.ld_x = ld_x; a.add = add; a.ld_add = ld_add; a.out = y; a.ld_out = ld_y; a.gain = gain; a.offset = offset; a.stats = stats;
    a.rows = rows; a.c = c; a.eps = eps;
    if (ckpt) { a.k_codes = (int8_t*)ckpt; a.k_scales = (uint8_t*)ckpt + up256((size_t)rows * c); }
    const bool whole = Whole(c, e).take(x, ld_x, rows).take(add, ld_add, rows).take(y, ld_y, rows).ok;
    const double n = (double)rows * c;
    op.launch("layernorm fwd", "ln_op_fwd_kernel", 9 * n, n * e * (add ? 3 : 2) + (ckpt ? (double)ck_bytes(rows, c) : 0.0), [&] {
      type_dispatch(dtype, [&](auto t) { width_dispatch(c, whole, [&](auto v, auto w) { ln_fwd_run<decltype(t), v.value, w.value>(op.st, a); }); });
    });
    return op.err;
  });
}

int pe_layernorm_bwd(pe_handle* h, long long rows, int c, int dtype, int x_type, const void* x, long long ld_x, const float* stats,
                     const float* gain, const void* dy, long long ld_dy, const void* add, long long ld_add, void* dx, long long ld_dx,
                     float* d_gain, float* d_offset, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!h) return PE_ERR_NULL;
    OpCall op{h, (hipStream_t)stream};
    if (rows < 0 || rows > MAX_ROWS || c < 1 || c > LN_MAX_C || !type_ok(dtype))
      return op.refuse(PE_ERR_DIMS, "layer norm: rows in [0, 2^40], c in [1, 16384], dtype PE_F32 or PE_BF16");
    const bool kept = x_type == PE_CKPT;
    if (!kept && x_type != dtype) return op.refuse(PE_ERR_ARG, "layer norm: x is of the type dtype or a checkpoint (PE_CKPT)");
    if ((!kept && ld_x < c) || ld_dy < c || (add && dx && ld_add < c) || (dx && ld_dx < c)) return op.refuse(PE_ERR_ARG, "layer norm: a row stride is less than c");
    const bool params = d_gain || d_offset;
    if (rows && (!x || !stats || !dy)) return op.refuse(PE_ERR_NULL, "layer norm: null tensor");
    if (params && !workspace) return op.refuse(PE_ERR_NULL, "layer norm: the gradients of gain and offset need a workspace");
    if (!dx) add = nullptr;
    const size_t e = elem(dtype);
    if (!aligned(x, kept ? 256 : e) || !aligned(dy, e) || !aligned(add, e) || !aligned(dx, e) || !aligned(gain, 4) || !aligned(stats, 8) ||
        !aligned(d_gain, 4) || !aligned(d_offset, 4) || !aligned(workspace, 256))
      return op.refuse(PE_ERR_ARG, "layer norm: a tensor is not aligned to its elements, stats not to 8 bytes, or the checkpoint or workspace not to 256");
    const size_t need = params ? pe_layernorm_workspace_bytes(rows, c) : 0;
    if (params && workspace_bytes < need) return op.refuse(PE_ERR_WORKSPACE, "layer norm: the workspace is smaller than pe_layernorm_workspace_bytes");
    const bool in_place = add == dx && ld_add == ld_dx;    // dx = dx + ...
    const Region rg[] = {{x, kept ? ck_bytes(rows, c) : span(rows, c, ld_x, e), false}, {stats, (size_t)rows * 8, false}, {gain, (size_t)c * 4, false},
                         {dy, span(rows, c, ld_dy, e), false}, {in_place ? nullptr : add, span(rows, c, ld_add, e), false},
                         {dx, span(rows, c, ld_dx, e), true}, {d_gain, (size_t)c * 4, true}, {d_offset, (size_t)c * 4, true},
                         {params ? workspace : nullptr, need, true}};
    if (any_alias(rg, 9)) return op.refuse(PE_ERR_ALIAS, "layer norm: a buffer that is written overlaps another one");
    if (!op.device_ok()) return op.refuse(PE_ERR_ARG, "layer norm: the handle belongs to another device than the current one");
    long long groups = 0;
    if (rows && (dx || params)) {
      LnArgs a{};
      if (kept) { a.codes = (const int8_t*)x; a.scales = (const uint8_t*)x + up256((size_t)rows * c); }
      else { a.x = x; a.ld_x = ld_x; }
      a.add = add; a.ld_add = ld_add; a.dy = dy; a.ld_dy = ld_dy; a.out = dx; a.ld_out = ld_dx; a.gain = gain; a.stats_in = stats;
      a.part = params ? (float*)workspace : nullptr;
      a.rows = rows; a.c = c;
      const bool whole = Whole(c, e).take(a.x, ld_x, rows).take(dy, ld_dy, rows).take(add, ld_add, rows).take(dx, ld_dx, rows).ok;
      groups = ln_bwd_groups(rows, c);
      const unsigned wg = (unsigned)groups;
      const double n = (double)rows * c;
      op.launch("layernorm bwd", "ln_op_bwd_kernel", 15 * n, n * e * (1 + (dx ? 1 : 0) + (add ? 1 : 0)) + (kept ? (double)ck_bytes(rows, c) : n * e), [&] {
        type_dispatch(dtype, [&](auto t) { width_dispatch(c, whole, [&](auto v, auto w) { ln_bwd_run<decltype(t), v.value, w.value>(op.st, a, wg); }); });
      });
    }
    if (params && (groups || !accumulate)) columns_sum(op, "layernorm sums", (const float*)workspace, groups, 2 * c, d_gain, d_offset, c, accumulate != 0);
    return op.err;
  });
}

size_t pe_relpos_workspace_bytes(const pe_relpos* p) {
  if (!p || rp_why(*p)) return 0;
  return rp_workspace(*p);
}

int pe_relpos_fwd(pe_handle* h, const pe_relpos* p, const int* edges, const int* pos_q, const int* pos_k, const int* seg_q, const int* seg_k,
                  const float* table, const void* add, void* out, void* stream) {
  return guarded([&]() -> int {
    if (!h) return PE_ERR_NULL;
    OpCall op{h, (hipStream_t)stream};
    RpArgs a;
    int rc = rp_check(op, p, edges, pos_q, pos_k, seg_q, seg_k, a);
    if (rc) return rc;
    if (p->n_q == 0 || p->n_k == 0) return PE_OK;
    if (!table || !out) return op.refuse(PE_ERR_NULL, "relative positions: null tensor");
    const size_t e = elem(p->dtype);
    if (!aligned(table, 4) || !aligned(add, e) || !aligned(out, e)) return op.refuse(PE_ERR_ARG, "relative positions: a tensor is not aligned to its elements");
    const Region rg[] = {{pos_q, (size_t)p->n_q * 4, false}, {pos_k, (size_t)p->n_k * 4, false}, {a.seg_q, (size_t)p->n_q * 4, false},
                         {a.seg_k, (size_t)p->n_k * 4, false}, {table, (size_t)a.nb * p->c * 4, false},
                         {add == out ? nullptr : add, rp_span(*p), false}, {out, rp_span(*p), true}};
    if (any_alias(rg, 7)) return op.refuse(PE_ERR_ALIAS, "relative positions: the output overlaps another buffer");
    if (!op.device_ok()) return op.refuse(PE_ERR_ARG, "relative positions: the handle belongs to another device than the current one");
    a.table = table; a.add = add; a.out = out;
    const bool pair = p->layout == PE_RELPOS_PAIR;
    const bool whole = Whole(pair ? p->c : p->n_k, e).take(add, a.ld, 2).take(out, a.ld, 2).ok;
    const double n = (double)p->n_q * p->n_k * p->c;
    op.launch("relpos fwd", pair ? "relpos_pair_fwd_kernel" : "relpos_heads_fwd_kernel", n, n * e * (add ? 2 : 1), [&] {
      type_dispatch(p->dtype, [&](auto t) {
        using T = decltype(t);
        // little to write: a position per lane, so that eight times the workgroups share it.  By positions and by vectors, us: 1 x 8191 x 8 fp32
        // 2.9 and 6.6, 1 x 32768 x 8 3.2 and 6.3; beyond the border, where vectors are taken, 1 x 65536 x 8 3.4 and 6.6, 256 x 512 x 16 bf16 4.9 and 7.6,
        // 1 x 524288 x 8 7.9 and 9.3
        if (!pair && n < (1 << 19)) rp_heads_fwd<T, 1, true>(op.st, a);
        else width_dispatch(pair ? p->c : p->n_k, whole, [&](auto v, auto w) {
          if (pair) rp_pair_fwd<T, v.value, w.value>(op.st, a); else rp_heads_fwd<T, v.value, w.value>(op.st, a);
        });
      });
    });
    return op.err;
  });
}

int pe_relpos_bwd(pe_handle* h, const pe_relpos* p, const int* edges, const int* pos_q, const int* pos_k, const int* seg_q, const int* seg_k,
                  const void* d_out, float* d_table, int accumulate, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!h) return PE_ERR_NULL;
    OpCall op{h, (hipStream_t)stream};
    RpArgs a;
    int rc = rp_check(op, p, edges, pos_q, pos_k, seg_q, seg_k, a);
    if (rc) return rc;
    const bool some = p->n_q > 0 && p->n_k > 0;
    if (!d_table || !workspace || (some && !d_out)) return op.refuse(PE_ERR_NULL, "relative positions: null tensor or workspace");
    const size_t e = elem(p->dtype), need = rp_workspace(*p);
    if (!aligned(d_out, e) || !aligned(d_table, 4) || !aligned(workspace, 256))
      return op.refuse(PE_ERR_ARG, "relative positions: a tensor is not aligned to its elements, or the workspace not to 256 bytes");
    if (workspace_bytes < need) return op.refuse(PE_ERR_WORKSPACE, "relative positions: the workspace is smaller than pe_relpos_workspace_bytes");
    const Region rg[] = {{pos_q, (size_t)p->n_q * 4, false}, {pos_k, (size_t)p->n_k * 4, false}, {a.seg_q, (size_t)p->n_q * 4, false},
                         {a.seg_k, (size_t)p->n_k * 4, false}, {d_out, rp_span(*p), false}, {d_table, (size_t)a.nb * p->c * 4, true},
                         {workspace, need, true}};
    if (any_alias(rg, 7)) return op.refuse(PE_ERR_ALIAS, "relative positions: a buffer that is written overlaps another one");
    if (!op.device_ok()) return op.refuse(PE_ERR_ARG, "relative positions: the handle belongs to another device than the current one");
    a.d_out = d_out; a.part = (float*)workspace;
    const bool pair = p->layout == PE_RELPOS_PAIR;
    long long groups = 0;
    if (some) {
      const bool whole = Whole(p->n_k, e).take(d_out, a.ld, 2).ok;
      groups = pair ? rp_pair_groups(*p) : rp_heads_groups(*p);
      const double n = (double)p->n_q * p->n_k * p->c;
      op.launch("relpos bwd", pair ? rp_pair_mm(a) ? "relpos_pair_bwd_mm_kernel" : "relpos_pair_bwd_kernel" : "relpos_heads_bwd_kernel", n, n * e, [&] {
        type_dispatch(p->dtype, [&](auto t) {
          using T = decltype(t);
          if (pair) rp_pair_bwd_run<T>(op.st, h->device, a, groups);
          else width_dispatch(p->n_k, whole, [&](auto v, auto w) { rp_heads_bwd<T, v.value, w.value>(op.st, h->device, a, rp_heads_split(*p)); });
        });
      });
    }
    const int cols = a.nb * p->c;
    if (groups || !accumulate) columns_sum(op, "relpos sums", (const float*)workspace, groups, cols, d_table, nullptr, cols, accumulate != 0);
    return op.err;
  });
}

}  // extern "C"
