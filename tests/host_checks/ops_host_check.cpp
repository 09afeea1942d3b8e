// Refusals of the operators around the trunk, on the CPU under the address and undefined-behaviour sanitizers: every call here has
// to return before anything is launched.  The handle is made by hand (pe_create needs a device).  Prints "ok <checks>" on success.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include "../../paper_2211_00235_amd/csrc/pe_handle.h"

static int checks = 0;
#define REQUIRE(c) do { checks++; if (!(c)) { fprintf(stderr, "FAILED line %d: %s\n", __LINE__, #c); exit(1); } } while (0)

static char* at(size_t mib) { return reinterpret_cast<char*>(((uintptr_t)1 << 44) + (mib << 20)); }   // never dereferenced
static pe_handle* h;

struct Ln {
  long long rows = 100; int c = 64, dtype = PE_BF16;
  void* x = at(1); long long ld_x = 64; void* add = at(2); long long ld_add = 64; float *gain = (float*)at(3), *offset = (float*)at(4); float eps = 1e-5f;
  void* y = at(5); long long ld_y = 64; float* stats = (float*)at(6); void* ckpt = at(7);
  int fwd() const { return pe_layernorm_fwd(h, rows, c, dtype, x, ld_x, add, ld_add, gain, offset, eps, y, ld_y, stats, ckpt, nullptr); }
};
struct LnB {
  long long rows = 100; int c = 64, dtype = PE_BF16, x_type = PE_BF16;
  void* x = at(1); long long ld_x = 64; float *stats = (float*)at(2), *gain = (float*)at(3); void* dy = at(4); long long ld_dy = 64;
  void* add = at(5); long long ld_add = 64; void* dx = at(6); long long ld_dx = 64; float *dg = (float*)at(7), *db = (float*)at(8);
  void* ws = at(9); size_t n = 1 << 20;
  int bwd() const { return pe_layernorm_bwd(h, rows, c, dtype, x_type, x, ld_x, stats, gain, dy, ld_dy, add, ld_add, dx, ld_dx, dg, db, 0, ws, n, nullptr); }
};
struct Ck {
  long long rows = 100; int c = 64, dtype = PE_F32; void* t = at(1); long long ld = 64; void* k = at(2);
  int pack() const { return pe_ckpt_pack(h, rows, c, dtype, t, ld, k, nullptr); }
  int unpack() const { return pe_ckpt_unpack(h, rows, c, dtype, k, t, ld, nullptr); }
};
static const int EDGES[3] = {-1, 0, 5};
struct Rp {
  pe_relpos p{10, 12, 8, 3, 1, PE_RELPOS_PAIR, PE_BF16, 0};
  const int* edges = EDGES; int *pq = (int*)at(1), *pk = (int*)at(2), *sq = (int*)at(3), *sk = (int*)at(4);
  float* table = (float*)at(5); void* add = at(6); void* out = at(7); void* ws = at(8); size_t n = 1 << 20;
  int fwd() const { return pe_relpos_fwd(h, &p, edges, pq, pk, sq, sk, table, add, out, nullptr); }
  int bwd() const { return pe_relpos_bwd(h, &p, edges, pq, pk, sq, sk, out, table, 0, ws, n, nullptr); }
};
template <typename C, typename F> static C with(F&& f) { C c; f(c); return c; }
#define LN(code, ...) REQUIRE(with<Ln>([](Ln& a) { __VA_ARGS__; }).fwd() == code && h->last_error.size() > 0)
#define LNB(code, ...) REQUIRE(with<LnB>([](LnB& a) { __VA_ARGS__; }).bwd() == code && h->last_error.size() > 0)
#define CK(code, ...) do { REQUIRE(with<Ck>([](Ck& a) { __VA_ARGS__; }).pack() == code); REQUIRE(with<Ck>([](Ck& a) { __VA_ARGS__; }).unpack() == code); } while (0)
#define RP(code, ...) do { REQUIRE(with<Rp>([](Rp& a) { __VA_ARGS__; }).fwd() == code); REQUIRE(with<Rp>([](Rp& a) { __VA_ARGS__; }).bwd() == code); } while (0)

int main() {
  h = new pe_handle();
  h->device = -5;               // no current device is this one: a call that passes every other check is refused for it
  // layer norm, forward
  LN(PE_ERR_ARG, );             // the device
  REQUIRE(h->last_error.find("device") != std::string::npos);
  LN(PE_ERR_DIMS, a.rows = -1); LN(PE_ERR_DIMS, a.rows = 1LL << 41); LN(PE_ERR_DIMS, a.c = 0); LN(PE_ERR_DIMS, a.c = 16385); LN(PE_ERR_DIMS, a.dtype = PE_CKPT);
  LN(PE_ERR_DIMS, a.eps = 0.0f); LN(PE_ERR_DIMS, a.eps = -1.0f); LN(PE_ERR_DIMS, a.eps = __builtin_nanf(""));
  LN(PE_ERR_ARG, a.ld_x = 63); LN(PE_ERR_ARG, a.ld_y = 0); LN(PE_ERR_ARG, a.ld_add = -64);
  LN(PE_ERR_NULL, a.x = nullptr); LN(PE_ERR_NULL, a.y = nullptr);
  LN(PE_ERR_ARG, a.x = at(1) + 1); LN(PE_ERR_ARG, a.stats = (float*)(at(6) + 4)); LN(PE_ERR_ARG, a.ckpt = at(7) + 128); LN(PE_ERR_ARG, a.gain = (float*)(at(3) + 2));
  LN(PE_ERR_ALIAS, a.y = a.x); LN(PE_ERR_ALIAS, a.y = at(1) + 2 * (99 * 64 + 63)); LN(PE_ERR_ALIAS, a.stats = (float*)a.y); LN(PE_ERR_ALIAS, a.ckpt = a.x);
  LN(PE_ERR_ALIAS, a.add = a.y; a.ld_add = 65); LN(PE_ERR_ALIAS, a.gain = (float*)a.stats);
  REQUIRE(with<Ln>([](Ln& a) { a.add = a.y; }).fwd() == PE_ERR_ARG && h->last_error.find("device") != std::string::npos);    // in place is allowed
  REQUIRE(with<Ln>([](Ln& a) { a.y = at(1) + 2 * 100 * 64; }).fwd() == PE_ERR_ARG && h->last_error.find("device") != std::string::npos);   // next to each other
  REQUIRE(with<Ln>([](Ln& a) { a.rows = 0; a.x = a.y = nullptr; }).fwd() == PE_OK);
  // layer norm, backward
  LNB(PE_ERR_ARG, );
  LNB(PE_ERR_DIMS, a.rows = -1); LNB(PE_ERR_DIMS, a.c = 0); LNB(PE_ERR_DIMS, a.dtype = 7);
  LNB(PE_ERR_ARG, a.x_type = PE_F32); LNB(PE_ERR_ARG, a.x_type = 9); LNB(PE_ERR_ARG, a.ld_x = 1); LNB(PE_ERR_ARG, a.ld_dy = 1); LNB(PE_ERR_ARG, a.ld_dx = 1); LNB(PE_ERR_ARG, a.ld_add = 1);
  LNB(PE_ERR_NULL, a.x = nullptr); LNB(PE_ERR_NULL, a.stats = nullptr); LNB(PE_ERR_NULL, a.dy = nullptr); LNB(PE_ERR_NULL, a.ws = nullptr);
  LNB(PE_ERR_ARG, a.x_type = PE_CKPT; a.x = at(1) + 64); LNB(PE_ERR_ARG, a.ws = at(9) + 128); LNB(PE_ERR_ARG, a.dg = (float*)(at(7) + 1));
  LNB(PE_ERR_WORKSPACE, a.n = pe_layernorm_workspace_bytes(100, 64) - 1);
  LNB(PE_ERR_ALIAS, a.dx = a.dy); LNB(PE_ERR_ALIAS, a.dx = a.x); LNB(PE_ERR_ALIAS, a.dg = a.db); LNB(PE_ERR_ALIAS, a.ws = a.x); LNB(PE_ERR_ALIAS, a.dg = a.gain);
  LNB(PE_ERR_ALIAS, a.add = at(6) + 2; a.ld_add = 64); LNB(PE_ERR_ALIAS, a.x_type = PE_CKPT; a.dx = at(1) + 6400);
  REQUIRE(with<LnB>([](LnB& a) { a.add = a.dx; }).bwd() == PE_ERR_ARG && h->last_error.find("device") != std::string::npos);
  REQUIRE(with<LnB>([](LnB& a) { a.dg = a.db = nullptr; a.ws = nullptr; a.n = 0; }).bwd() == PE_ERR_ARG && h->last_error.find("device") != std::string::npos);
  // checkpoints
  CK(PE_ERR_ARG, );
  CK(PE_ERR_DIMS, a.rows = -1); CK(PE_ERR_DIMS, a.c = 0); CK(PE_ERR_DIMS, a.c = (1 << 20) + 1); CK(PE_ERR_DIMS, a.dtype = PE_CKPT); CK(PE_ERR_DIMS, a.rows = 1LL << 39; a.c = a.ld = 1024);
  CK(PE_ERR_ARG, a.ld = 63); CK(PE_ERR_NULL, a.t = nullptr); CK(PE_ERR_NULL, a.k = nullptr); CK(PE_ERR_ARG, a.t = at(1) + 2); CK(PE_ERR_ARG, a.k = at(2) + 16);
  CK(PE_ERR_ALIAS, a.k = a.t); CK(PE_ERR_ALIAS, a.t = at(2) + 6400);
  CK(PE_OK, a.rows = 0; a.t = a.k = nullptr);
  // relative positions
  RP(PE_ERR_ARG, );
  RP(PE_ERR_DIMS, a.p.n_q = -1); RP(PE_ERR_DIMS, a.p.n_k = (1 << 24) + 1); RP(PE_ERR_DIMS, a.p.c = 0); RP(PE_ERR_DIMS, a.p.c = 1025); RP(PE_ERR_DIMS, a.p.n_edges = -1);
  RP(PE_ERR_DIMS, a.p.n_edges = 255); RP(PE_ERR_DIMS, a.p.segments = 2); RP(PE_ERR_DIMS, a.p.layout = 2); RP(PE_ERR_DIMS, a.p.dtype = PE_CKPT); RP(PE_ERR_DIMS, a.p.ld = -1);
  RP(PE_ERR_DIMS, a.p.n_q = a.p.n_k = 1 << 24);
  RP(PE_ERR_ARG, a.p.ld = 12 * 8 - 1); RP(PE_ERR_ARG, a.p.layout = PE_RELPOS_HEADS; a.p.ld = 11);
  static const int same[3] = {-1, -1, 5}, down[3] = {0, -1, 5}, least[3] = {-2147483647 - 1, 0, 5};
  RP(PE_ERR_ARG, a.edges = same); RP(PE_ERR_ARG, a.edges = down); RP(PE_ERR_ARG, a.edges = least);
  RP(PE_ERR_NULL, a.edges = nullptr); RP(PE_ERR_NULL, a.pq = nullptr); RP(PE_ERR_NULL, a.sk = nullptr); RP(PE_ERR_NULL, a.table = nullptr); RP(PE_ERR_NULL, a.out = nullptr);
  RP(PE_ERR_ARG, a.pk = (int*)(at(2) + 2)); RP(PE_ERR_ARG, a.out = at(7) + 1); RP(PE_ERR_ARG, a.table = (float*)(at(5) + 2));
  REQUIRE(with<Rp>([](Rp& a) { a.out = a.table; }).fwd() == PE_ERR_ALIAS);
  REQUIRE(with<Rp>([](Rp& a) { a.add = at(7) + 2; }).fwd() == PE_ERR_ALIAS);
  REQUIRE(with<Rp>([](Rp& a) { a.add = a.out; }).fwd() == PE_ERR_ARG && h->last_error.find("device") != std::string::npos);
  REQUIRE(with<Rp>([](Rp& a) { a.ws = nullptr; }).bwd() == PE_ERR_NULL);
  REQUIRE(with<Rp>([](Rp& a) { a.ws = at(8) + 8; }).bwd() == PE_ERR_ARG);
  REQUIRE(with<Rp>([](Rp& a) { a.n = pe_relpos_workspace_bytes(&a.p) - 1; }).bwd() == PE_ERR_WORKSPACE);
  REQUIRE(with<Rp>([](Rp& a) { a.ws = a.out; }).bwd() == PE_ERR_ALIAS);
  REQUIRE(with<Rp>([](Rp& a) { a.p.n_q = 0; a.pq = a.sq = nullptr; a.out = nullptr; }).fwd() == PE_OK);
  REQUIRE(pe_relpos_fwd(h, nullptr, EDGES, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == PE_ERR_NULL);
  REQUIRE(pe_relpos_workspace_bytes(nullptr) == 0);
  delete h;
  printf("ok %d\n", checks);
  return 0;
}
