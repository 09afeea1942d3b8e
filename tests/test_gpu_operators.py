"""The operators around the trunk on the GPU against their float64 definitions (tests/op_reference.py).

Tolerances, elementwise, u = 2^-24 (half a step of fp32), h = half a step of the storage type (fp32 2^-24, bf16 2^-8 of the value):
  a sum of n terms in a fixed tree over lanes, with D additions in a row at most, is off by D u times the sum of the terms' magnitudes.
  layer norm, D = 48 (a lane adds up to 16 elements, 6 steps over lanes, 16 waves, and a handful of products):
    y:      h |y| + D u ((|x| + mean|x|) rstd |gain| + |offset| + |add|)
    dx:     h |dx| + D u rstd (|u| + mean|u| + (|z| + zz) mean|u z| + ...), zz = (|x| + |mean|) rstd, the size of the terms of z
    d_gain: D' u sum |dy| zz, D' = 64 + rows / 64 (a lane adds one row in 64 or fewer)
  the gradient of the table: see there."""
import numpy as np
import pytest
import torch

import paper_2211_00235_amd as pe
from tests import op_reference as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16)}      # rounding to nearest is off by half a step
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def h():
    return pe.Handle()


def f64(t):
    return t.detach().cpu().double().numpy()


def rand(rng, shape, dt, scale=1.0):
    return (torch.from_numpy(rng.normal(size=shape)) * scale).to(dt).cuda()


def vec(rng, n, around=0.0):
    return (torch.from_numpy(rng.normal(size=n)) * 0.3 + around).float().cuda()


def bytes_(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


def inside(got, want, tol, what=""):
    got = f64(got)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], np.broadcast_to(tol, want.shape)[bad][:4])


def ln_y_tol(y, x, rstd, gain, offset, add, half):
    a = np.abs(x) + np.abs(x).mean(1, keepdims=True)
    s = a * rstd[:, None] * (np.abs(gain) if gain is not None else 1.0)
    s = s + (np.abs(offset) if offset is not None else 0.0) + (np.abs(add) if add is not None else 0.0)
    return half * np.abs(y) * (1 + 1e-6) + 48 * U * s


def ln_check_bwd(x, stats, gain, dy, add, got, half, rows):
    """x, dy, add: float64; stats: the fp32 statistics that the call was given."""
    mean, rstd = stats[:, 0], stats[:, 1]
    dx, dg, db = ref.layernorm_bwd(x, mean, rstd, gain, dy, add)
    z = (x - mean[:, None]) * rstd[:, None]
    zz = (np.abs(x) + np.abs(mean)[:, None]) * rstd[:, None]
    w = dy if gain is None else dy * gain
    m1, m2 = np.abs(w).mean(1, keepdims=True), (np.abs(w) * zz).mean(1, keepdims=True)
    tol = half * np.abs(dx) * (1 + 1e-6) + 48 * U * (rstd[:, None] * (np.abs(w) + m1 + (np.abs(z) + zz) * m2) + (np.abs(add) if add is not None else 0.0))
    if got[0] is not None:
        inside(got[0], dx, tol, "dx")
    deep = (64 + rows / 64) * U
    if got[1] is not None:
        inside(got[1], dg, deep * (np.abs(dy) * zz).sum(0) + 1e-30, "d_gain")
    if got[2] is not None:
        inside(got[2], db, deep * np.abs(dy).sum(0) + 1e-30, "d_offset")


# every width of access, every number of lanes per row, and the neighbours of the borders between them
CS = [1, 2, 3, 7, 8, 23, 31, 32, 33, 40, 64, 65, 100, 128, 130, 136, 256, 257, 512, 514, 520, 1000, 1024, 1026, 2047, 2048, 2056, 4096,
      4098, 4099, 4104, 8192, 8194, 8200, 16383, 16384]


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("c", CS)
def test_layernorm(h, c, dt):
    rng = np.random.default_rng(c)
    rows = 37 if c > 600 else 301
    x, add, dy = rand(rng, (rows, c), dt, 2.0) + 0.7, rand(rng, (rows, c), dt), rand(rng, (rows, c), dt)
    g, b = vec(rng, c, 1.0), vec(rng, c)
    y, stats, kept = torch.empty_like(x), torch.empty(rows, 2, device="cuda"), bytes_(pe.ckpt_bytes(rows, c))
    pe.layernorm_fwd(h, x, g, b, y, add=add, stats=stats, ckpt=kept)
    X, G, B, A, DY = f64(x), f64(g), f64(b), f64(add), f64(dy)
    want, mean, rstd = ref.layernorm(X, G, B, 1e-5, A)
    inside(y, want, ln_y_tol(want, X, rstd, G, B, A, HALF[dt]), "y")
    inside(stats[:, 0], mean, 48 * U * np.abs(X).mean(1), "mean")
    # the variance is off by the mean's error squared and 48 u of itself; its rounding shows where it is near zero (c = 1)
    inside(stats[:, 1], rstd, rstd * (48 * U + 0.5 * (48 * U * np.abs(X).mean(1) * rstd) ** 2) + 0 * rstd, "rstd")
    codes, scales, back = ref.ckpt(X)
    k = kept.cpu().numpy()
    assert np.array_equal(k[:rows * c].view(np.int8).reshape(rows, c), codes)
    off = -(-rows * c // 256) * 256
    assert np.array_equal(k[off:off + scales.size].reshape(scales.shape), scales)
    ws = bytes_(pe.layernorm_workspace_bytes(rows, c))
    for src, xs in ((x, X), (kept, back)):
        dx, dg, db = torch.empty_like(x), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        pe.layernorm_bwd(h, dy, src, stats, g, dx, dg, db, ws)
        ln_check_bwd(xs, f64(stats), G, DY, None, (dx, dg, db), HALF[dt], rows)


@pytest.mark.parametrize("rows", [0, 1, 2, 3, 63, 64, 65, 1023, 4097, 40000])
@pytest.mark.parametrize("c, dt", [(128, torch.bfloat16), (23, torch.bfloat16), (64, torch.float32), (2048, torch.bfloat16)])
def test_layernorm_row_counts(h, rows, c, dt):
    if rows * c > 9_000_000:
        rows //= 10
    rng = np.random.default_rng(rows + c)
    x, dy, g = rand(rng, (rows, c), dt), rand(rng, (rows, c), dt), vec(rng, c, 1.0)
    y, stats = torch.empty_like(x), torch.empty(rows, 2, device="cuda")
    pe.layernorm_fwd(h, x, g, None, y, stats=stats)
    X, G = f64(x), f64(g)
    want, _, rstd = ref.layernorm(X, G)
    inside(y, want, ln_y_tol(want, X, rstd, G, None, None, HALF[dt]) if rows else 0.0)
    ws = bytes_(pe.layernorm_workspace_bytes(rows, c))
    dx, dg, db = torch.empty_like(x), torch.full((c,), 5.0, device="cuda"), torch.full((c,), 5.0, device="cuda")
    pe.layernorm_bwd(h, dy, x, stats, g, dx, dg, db, ws)
    if rows:
        ln_check_bwd(X, f64(stats), G, f64(dy), None, (dx, dg, db), HALF[dt], rows)
    else:
        assert not dg.any() and not db.any()
        pe.layernorm_bwd(h, dy, x, stats, g, dx, dg.fill_(5.0), db, ws, accumulate=True)
        assert bool((dg == 5.0).all())


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("c, ld, off", [(64, 72, 0), (64, 65, 0), (64, 80, 1), (64, 80, 2), (23, 40, 3), (256, 512, 8), (2048, 2050, 2), (130, 132, 4)])
def test_layernorm_strided_rows_and_gaps(h, c, ld, off, dt):
    """Rows with gaps and odd starts: the gaps, and what lies in front of and behind the rows, stay as they were."""
    rng = np.random.default_rng(ld)
    rows = 29
    mk = lambda: rand(rng, (rows * ld + 64,), dt)
    view = lambda t: torch.as_strided(t, (rows, c), (ld, 1), off)
    bx, ba, by, bdy, bdx = mk(), mk(), mk(), mk(), mk()
    x, add, y, dy, dx = map(view, (bx, ba, by, bdy, bdx))
    before = [t.clone() for t in (bx, ba, by, bdy, bdx)]
    g, b, stats = vec(rng, c, 1.0), vec(rng, c), torch.empty(rows, 2, device="cuda")
    pe.layernorm_fwd(h, x, g, b, y, add=add, stats=stats)
    ws = bytes_(pe.layernorm_workspace_bytes(rows, c))
    dg, db = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    pe.layernorm_bwd(h, dy, x, stats, g, dx, dg, db, ws, add=add)
    X, G, B, A = f64(x), f64(g), f64(b), f64(add)
    want, _, rstd = ref.layernorm(X, G, B, 1e-5, A)
    inside(y, want, ln_y_tol(want, X, rstd, G, B, A, HALF[dt]))
    ln_check_bwd(X, f64(stats), G, f64(dy), A, (dx, dg, db), HALF[dt], rows)
    for t, was, written in zip((bx, ba, by, bdy, bdx), before, (False, False, True, False, True)):
        now = t.clone()
        if written:
            view(now).copy_(view(was))
        assert torch.equal(now, was)


def test_layernorm_in_place_and_optional_arguments(h):
    rng = np.random.default_rng(5)
    rows, c = 77, 256
    x, dy, y0 = (rand(rng, (rows, c), torch.bfloat16) for _ in range(3))
    g, b, stats = vec(rng, c, 1.0), vec(rng, c), torch.empty(rows, 2, device="cuda")
    two, y, dx0 = torch.empty_like(x), y0.clone(), rand(rng, (rows, c), torch.bfloat16)
    pe.layernorm_fwd(h, x, g, b, two, add=y0, stats=stats)
    pe.layernorm_fwd(h, x, g, b, y, add=y)                        # y = y + LN(x)
    assert torch.equal(y, two)
    ws = bytes_(pe.layernorm_workspace_bytes(rows, c))
    dx, dx2, dg, db, dg2 = torch.empty_like(x), dx0.clone(), *(torch.empty(c, device="cuda") for _ in range(3))
    pe.layernorm_bwd(h, dy, x, stats, g, dx, dg, db, ws, add=dx0)
    pe.layernorm_bwd(h, dy, x, stats, g, dx2, None, None, None, add=dx2)
    assert torch.equal(dx, dx2)
    pe.layernorm_bwd(h, dy, x, stats, g, None, dg2, None, ws)     # no input gradient, no offset
    assert torch.equal(dg2, dg)
    pe.layernorm_bwd(h, dy, x, stats, g, None, dg2, None, ws, accumulate=True)
    assert torch.equal(dg2, 2 * dg)
    pe.layernorm_bwd(h, dy, x, stats, g, None, None, None, None)  # nothing wanted
    x3 = x.reshape(7, 11, c)                                      # more than two dimensions
    pe.layernorm_fwd(h, x3, g, b, two.view(7, 11, c), add=y0.view(7, 11, c))
    assert torch.equal(two, y)
    ones, zeros = torch.ones(c, device="cuda"), torch.zeros(c, device="cuda")
    pe.layernorm_fwd(h, x, None, None, y)
    pe.layernorm_fwd(h, x, ones, zeros, two)
    assert torch.equal(y, two)
    pe.layernorm_bwd(h, dy, x, stats, None, dx, dg, db, ws)
    pe.layernorm_bwd(h, dy, x, stats, ones, dx2, dg2, None, ws)
    assert torch.equal(dx, dx2) and torch.equal(dg, dg2)


def test_layernorm_special_values(h):
    """A row with NaN or infinity spoils itself alone; constant rows and rows far from zero keep their precision."""
    rng = np.random.default_rng(6)
    rows, c = 40, 128
    x = rand(rng, (rows, c), torch.float32)
    x[3, 7], x[9, 100], x[20] = float("nan"), float("inf"), 1.5
    x[30:] = x[30:] + 1000.0
    y, stats, kept = torch.empty_like(x), torch.empty(rows, 2, device="cuda"), bytes_(pe.ckpt_bytes(rows, c))
    pe.layernorm_fwd(h, x, None, None, y, stats=stats, ckpt=kept)
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[9]).all()) and not y[20].any()
    fine = [r for r in range(rows) if r not in (3, 9)]
    X = f64(x)[fine]
    want, _, rstd = ref.layernorm(X)
    inside(y[fine], want, ln_y_tol(want, X, rstd, None, None, None, HALF[torch.float32]))
    back = torch.empty_like(x)
    pe.ckpt_unpack(h, kept, back)
    nan = torch.isnan(back).cpu().numpy()
    assert nan[3, :32].all() and nan[9, 96:].all() and nan.sum() == 64
    # a long mean of large equal terms: integers, so that the gradient sums are exact whatever their order
    dy = torch.from_numpy(rng.integers(-8, 9, size=(3000, 64))).float().cuda()
    x = rand(rng, (3000, 64), torch.float32)
    stats, db, dg = torch.tensor([[0.0, 1.0]], device="cuda").repeat(3000, 1), torch.empty(64, device="cuda"), torch.empty(64, device="cuda")
    xi = torch.from_numpy(rng.integers(-4, 5, size=(3000, 64))).float().cuda()
    pe.layernorm_bwd(h, dy, xi, stats, None, None, dg, db, bytes_(pe.layernorm_workspace_bytes(3000, 64)))
    assert torch.equal(db, dy.sum(0)) and torch.equal(dg.double(), (dy.double() * xi.double()).sum(0))


# ---------------------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("rows, c", [(0, 8), (1, 1), (1, 8), (3, 32), (5, 33), (7, 31), (64, 64), (129, 40), (1000, 16), (33, 100), (17, 1026), (3, 5000), (2, 100000),
                                     (4099, 23), (2048, 128)])
def test_ckpt(h, rows, c, dt):
    """Codes, scales and restored values are the definition's, bit for bit."""
    rng = np.random.default_rng(rows + 7 * c)
    x = rng.normal(size=(rows, c)) * np.exp2(rng.integers(-130, 120, size=(rows, 1)).astype(np.float64))
    x[rng.random(x.shape) < 0.05] = 0.0
    if rows > 2:
        x[rows // 2] = 0.0
        x[rows - 1] = 1e-44                                    # below the least scale
        x[0] = 127.0 * 2.0 ** 9 * np.sign(x[0])
        x[1, c // 2] = [np.nan, np.inf, -np.inf][c % 3]
    t = torch.from_numpy(x).to(dt).cuda()
    kept, y = bytes_(pe.ckpt_bytes(rows, c) + 64).fill_(0xA5), torch.full_like(t, 3.0)
    pe.ckpt_pack(h, t, kept)
    pe.ckpt_unpack(h, kept, y)
    codes, scales, back = ref.ckpt(f64(t))
    k, off = kept.cpu().numpy(), -(-rows * c // 256) * 256
    assert np.array_equal(k[:rows * c].view(np.int8).reshape(rows, c), codes)
    assert np.array_equal(k[off:off + scales.size].reshape(scales.shape), scales)
    assert bool((kept[off + scales.size:] == 0xA5).all()) and bool((kept[rows * c:off] == 0xA5).all())
    got = f64(y)
    assert np.array_equal(np.isnan(got), np.isnan(back)) and np.array_equal(got[~np.isnan(got)], back[~np.isnan(back)])
    again = torch.empty_like(kept)
    pe.ckpt_pack(h, y, again)                                   # packing what was restored changes nothing
    assert torch.equal(again[:rows * c], kept[:rows * c])


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("c", [5, 32, 40])
def test_ckpt_largest_numbers(h, c, dt):
    """Numbers up to the type's largest stay numbers, off by at most 1/127 of the largest of their group."""
    top = torch.finfo(dt).max
    x = torch.tensor([[top], [-top], [top * 0.9961], [top * 0.992], [top / 2]], dtype=torch.float64) * torch.linspace(1.0, -1.0, c, dtype=torch.float64)
    t = x.to(dt).cuda()
    kept, y, again = bytes_(pe.ckpt_bytes(5, c)), torch.empty_like(t), bytes_(pe.ckpt_bytes(5, c))
    pe.ckpt_pack(h, t, kept)
    pe.ckpt_unpack(h, kept, y)
    T, Y = f64(t), f64(y)
    assert np.isfinite(Y).all() and np.array_equal(Y, ref.ckpt(T)[2])
    assert (np.abs(Y - T)[:, :32] <= np.abs(T[:, :32]).max(1, keepdims=True) / 127).all()
    pe.ckpt_pack(h, y, again)
    assert torch.equal(again[:5 * c], kept[:5 * c])


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("c, ld, off", [(64, 72, 0), (64, 65, 0), (64, 80, 1), (40, 48, 8), (23, 40, 3), (130, 132, 4)])
def test_ckpt_strided_rows(h, c, ld, off, dt):
    rng = np.random.default_rng(ld)
    rows = 45
    buf, out = rand(rng, (rows * ld + 64,), dt), rand(rng, (rows * ld + 64,), dt)
    view = lambda t: torch.as_strided(t, (rows, c), (ld, 1), off)
    kept, was = bytes_(pe.ckpt_bytes(rows, c)), out.clone()
    pe.ckpt_pack(h, view(buf), kept)
    pe.ckpt_unpack(h, kept, view(out))
    assert np.array_equal(f64(view(out)), ref.ckpt(f64(view(buf)))[2])
    view(out).copy_(view(was))
    assert torch.equal(out, was)


# ---------------------------------------------------------------------------------------------------------------------

CLIP, LOG = list(range(-31, 33)), [-90, -31, -15, -7, -2, -1, 0, 1, 2, 3, 8, 16, 32, 91]
MANY = [3 * i - 381 for i in range(254)]


def rp_inputs(rng, n_q, n_k, edges, segs, c, spread=1.0):
    span = max(4, int(spread * (max(n_q, n_k) + 40)))
    pos = lambda n: torch.from_numpy(np.sort(rng.integers(-span, span, n)) if n % 2 else rng.integers(-span, span, n)).int().cuda()
    seg = lambda n: torch.from_numpy(rng.integers(0, 3, n)).int().cuda()
    pq, pk = pos(n_q), pos(n_k)
    sq, sk = (seg(n_q), seg(n_k)) if segs else (None, None)
    nb = len(edges) + (2 if segs else 1)
    b = ref.buckets(pq.cpu().numpy(), pk.cpu().numpy(), edges, *(t.cpu().numpy() if segs else None for t in (sq, sk)))
    return pq, pk, torch.tensor(edges, dtype=torch.int32), sq, sk, vec(rng, nb * c).view(nb, c), b, nb


@pytest.mark.parametrize("layout", ["pair", "heads"])
@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("n_q, n_k, c, edges, segs", [
    (1, 1, 1, [], False), (1, 1, 8, [0], True), (1, 700, 8, LOG, False), (300, 1, 16, CLIP, True), (33, 47, 128, CLIP, True), (64, 64, 64, LOG, False),
    (50, 50, 23, CLIP, False), (17, 1024, 4, LOG, True), (40, 56, 130, CLIP, True), (21, 88, 1, MANY, True), (9, 72, 40, MANY, False), (5, 16, 1024, CLIP, False),
    (130, 264, 12, CLIP, False), (70, 70, 128, CLIP, True), (90, 41, 96, [3 * i for i in range(100)], True), (61, 77, 24, CLIP, False), (37, 45, 64, list(range(20)), False), (0, 5, 8, CLIP, False), (5, 0, 8, CLIP, True), (3, 2100, 33, [-2147483647, 0, 2147483647], False)])
def test_relpos(h, layout, dt, n_q, n_k, c, edges, segs):
    rng = np.random.default_rng(n_q * 31 + n_k + c)
    pq, pk, ed, sq, sk, table, b, nb = rp_inputs(rng, n_q, n_k, edges, segs, c)
    shape = (n_q, n_k, c) if layout == "pair" else (c, n_q, n_k)
    out, add = torch.full(shape, 7.0, dtype=dt, device="cuda"), rand(rng, shape, dt)
    pe.relpos_fwd(h, pq, pk, ed, table, out, sq, sk, layout=layout)
    T, A = f64(table), f64(add)
    want = ref.relpos(b, T, None, layout)
    assert np.array_equal(f64(out), f64(torch.from_numpy(want).float().to(dt)))          # one rounding of an fp32 number
    pe.relpos_fwd(h, pq, pk, ed, table, out, sq, sk, add=add, layout=layout)
    want = ref.relpos(b, T, A, layout)
    inside(out, want, HALF[dt] * np.abs(want) * (1 + 1e-6) + U * np.abs(want))                # the fp32 sum, then the storage type
    pe.relpos_fwd(h, pq, pk, ed, table, add, sq, sk, add=add, layout=layout)             # in place
    assert torch.equal(add, out)
    ws = bytes_(pe.relpos_workspace_bytes(n_q, n_k, c, nb, layout))
    # whole numbers: every order of summation gives the same sum (n_q n_k 8 < 2^24), so a pair that is missed or doubled shows
    d = torch.from_numpy(rng.integers(-8, 9, size=shape)).to(dt).cuda()
    dt_ = torch.full((nb, c), 3.0, device="cuda")
    pe.relpos_bwd(h, pq, pk, ed, d, dt_, ws, sq, sk, layout=layout)
    exact = ref.relpos_bwd(b, f64(d), nb, layout)
    assert np.array_equal(f64(dt_), exact)
    pe.relpos_bwd(h, pq, pk, ed, d, dt_, ws, sq, sk, layout=layout, accumulate=True)
    assert np.array_equal(f64(dt_), 2 * exact)
    # normal values: a sum of n terms with at most n / 4 + 64 additions in a row
    d = rand(rng, shape, dt)
    pe.relpos_bwd(h, pq, pk, ed, d, dt_, ws, sq, sk, layout=layout)
    inside(dt_, ref.relpos_bwd(b, f64(d), nb, layout), (64 + n_q * n_k / 4) * U * ref.relpos_bwd(b, np.abs(f64(d)), nb, layout))


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("n_q, n_k, c, edges, off", [(20, 30, 65, CLIP, 0), (19, 33, 129, LOG, 1), (31, 17, 191, CLIP, 3), (23, 40, 64, CLIP, 1), (9, 50, 11, LOG, 5)])
def test_relpos_pair_odd_channels_and_alignment(h, n_q, n_k, c, edges, off, dt):
    """Positions whose channels are no whole 16-byte pieces, or start between two; what lies around them stays."""
    rng = np.random.default_rng(n_q + c)
    pq, pk, ed, _, _, table, b, nb = rp_inputs(rng, n_q, n_k, edges, False, c)
    n = n_q * n_k * c
    buf = rand(rng, (off + n + 40,), dt)
    was, view = buf.clone(), buf[off:off + n].view(n_q, n_k, c)
    want = ref.relpos(b, f64(table), f64(view), "pair")
    pe.relpos_fwd(h, pq, pk, ed, table, view, add=view, layout="pair")
    inside(view, want, HALF[dt] * np.abs(want) * (1 + 1e-6) + U * np.abs(want))
    assert torch.equal(buf[:off], was[:off]) and torch.equal(buf[off + n:], was[off + n:])
    view.copy_(torch.from_numpy(rng.integers(-8, 9, size=(n_q, n_k, c))))                  # whole numbers: exact sums
    d = torch.full((nb, c), 5.0, device="cuda")
    pe.relpos_bwd(h, pq, pk, ed, view, d, bytes_(pe.relpos_workspace_bytes(n_q, n_k, c, nb, "pair")), layout="pair")
    assert np.array_equal(f64(d), ref.relpos_bwd(b, f64(view), nb, "pair"))


@pytest.mark.parametrize("layout", ["pair", "heads"])
@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("n_q, n_k, c, edges", [(40, 64, 64, CLIP), (33, 50, 33, LOG), (21, 47, 20, CLIP), (40, 64, 8, CLIP), (17, 90, 48, MANY)])
def test_relpos_gradients_that_are_not_finite(h, layout, dt, n_q, n_k, c, edges):
    """An infinity or NaN shows in the sums of its own bucket and channel, and nowhere else."""
    rng = np.random.default_rng(n_k)
    pq, pk, ed, sq, sk, table, b, nb = rp_inputs(rng, n_q, n_k, edges, True, c)
    shape = (n_q, n_k, c) if layout == "pair" else (c, n_q, n_k)
    d = rng.integers(-8, 9, size=shape).astype(np.float64)
    for i in range(24):
        at = tuple(rng.integers(0, s) for s in shape)
        d[at] = [np.inf, -np.inf, np.nan, np.inf][i % 4]
    t, dtab = torch.from_numpy(d).to(dt).cuda(), torch.empty(nb, c, device="cuda")
    pe.relpos_bwd(h, pq, pk, ed, t, dtab, bytes_(pe.relpos_workspace_bytes(n_q, n_k, c, nb, layout)), sq, sk, layout=layout)
    want, got = ref.relpos_bwd(b, d, nb, layout), f64(dtab)
    assert not np.isfinite(want).all() and np.isfinite(want).any()
    assert np.array_equal(np.isnan(want), np.isnan(got)) and np.array_equal(want[~np.isnan(want)], got[~np.isnan(got)])


@pytest.mark.parametrize("layout", ["pair", "heads"])
@pytest.mark.parametrize("gap", [1, 8, 13])
def test_relpos_rows_with_gaps(h, layout, gap):
    rng = np.random.default_rng(gap)
    n_q, n_k, c = 37, 64, 16
    pq, pk, ed, sq, sk, table, b, nb = rp_inputs(rng, n_q, n_k, CLIP, True, c)
    row = n_k * c if layout == "pair" else n_k
    ld = row + gap
    shape, st = ((n_q, n_k, c), (ld, c, 1)) if layout == "pair" else ((c, n_q, n_k), (n_q * ld, ld, 1))
    n = (n_q if layout == "pair" else n_q * c) * ld + 8
    buf = rand(rng, (n,), torch.bfloat16)
    out, was = torch.as_strided(buf, shape, st), buf.clone()
    pe.relpos_fwd(h, pq, pk, ed, table, out, sq, sk, layout=layout)
    assert np.array_equal(f64(out), f64(torch.from_numpy(ref.relpos(b, f64(table), None, layout)).float().to(torch.bfloat16)))
    d = out
    d.copy_(torch.from_numpy(rng.integers(-8, 9, size=shape)).to(torch.bfloat16))
    dtab = torch.empty(nb, c, device="cuda")
    pe.relpos_bwd(h, pq, pk, ed, d, dtab, bytes_(pe.relpos_workspace_bytes(n_q, n_k, c, nb, layout)), sq, sk, layout=layout)
    assert np.array_equal(f64(dtab), ref.relpos_bwd(b, f64(d), nb, layout))
    out.copy_(torch.as_strided(was, shape, st))
    assert torch.equal(buf, was)


def test_relpos_axes_of_one_element(h):
    """One new position's rows in a longer sequence's bias and pair representation; what lies around them stays."""
    rng = np.random.default_rng(8)
    n, c, at = 72, 16, 29
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    ed, table = torch.tensor(LOG, dtype=torch.int32), vec(rng, (len(LOG) + 1) * c).view(-1, c)
    b = ref.buckets(np.array([at]), np.arange(n), LOG)
    bias, pair = rand(rng, (c, n, n), torch.float32), rand(rng, (n, n, c), torch.float32)
    for layout, whole, view in (("heads", bias, bias[:, at:at + 1]), ("heads", bias, bias[3:4, at:at + 1]), ("pair", pair, pair[at:at + 1]), ("pair", pair, pair[at:at + 1, :, 5:6])):
        cc = view.shape[0] if layout == "heads" else view.shape[2]
        if layout == "pair" and cc == 1:                     # channels of one position each, apart
            with pytest.raises(pe.PEError, match="gaps"):
                pe.relpos_fwd(h, pos[at:at + 1], pos, ed, table[:, :1].contiguous(), view, layout=layout)
            continue
        tab, was, old = table[:, :cc].contiguous(), whole.clone(), view.clone()
        pe.relpos_fwd(h, pos[at:at + 1], pos, ed, tab, view, layout=layout)
        assert np.array_equal(f64(view), ref.relpos(b, f64(tab), None, layout))
        d = torch.empty(len(LOG) + 1, cc, device="cuda")
        view.copy_(torch.from_numpy(rng.integers(-8, 9, size=tuple(view.shape))))
        pe.relpos_bwd(h, pos[at:at + 1], pos, ed, view, d, bytes_(pe.relpos_workspace_bytes(1, n, cc, len(LOG) + 1, layout)), layout=layout)
        assert np.array_equal(f64(d), ref.relpos_bwd(b, f64(view), len(LOG) + 1, layout))
        view.copy_(old)
        assert torch.equal(whole, was)
    column = pair[:, at:at + 1]                              # n_k = 1
    was, want = pair.clone(), ref.relpos(ref.buckets(np.arange(n), np.array([at]), LOG), f64(table), f64(column), "pair")
    pe.relpos_fwd(h, pos, pos[at:at + 1], ed, table, column, add=column)
    inside(column, want, HALF[torch.float32] * np.abs(want) * (1 + 1e-6) + U * np.abs(want))
    pair[:, at] = was[:, at]
    assert torch.equal(pair, was)


def test_relpos_extreme_positions(h):
    """Differences beyond 32 bits fall into the outermost buckets."""
    big = 2147483647
    pq, pk = torch.tensor([big, -big - 1, 0], dtype=torch.int32).cuda(), torch.tensor([big, -big - 1, 0, 5], dtype=torch.int32).cuda()
    for edges in ([-big, 0, big], [0, 1], [], CLIP):
        ed = torch.tensor(edges, dtype=torch.int32)
        table = torch.arange(float(len(edges) + 1), device="cuda").view(-1, 1)
        for layout in ("pair", "heads"):
            out = torch.empty((3, 4, 1) if layout == "pair" else (1, 3, 4), device="cuda")
            pe.relpos_fwd(h, pq, pk, ed, table, out, layout=layout)
            assert np.array_equal(out.cpu().numpy().reshape(3, 4), ref.buckets(pq.cpu().numpy(), pk.cpu().numpy(), edges))


def test_relpos_long_and_offsets_past_32_bits(h):
    """Bias of 33000 x 33000 positions, two heads: offsets beyond 2^31 elements; a few rows against the definition, and the gradient of
    ones, which counts pairs."""
    n, c = 33000, 2
    pos, ed = torch.arange(n, dtype=torch.int32, device="cuda"), torch.tensor(CLIP, dtype=torch.int32)
    table = torch.randn(65, c, device="cuda").bfloat16().float()
    out = torch.empty(c, n, n, dtype=torch.bfloat16, device="cuda")
    pe.relpos_fwd(h, pos, pos, ed, table, out, layout="heads")
    for q in (0, 1, 16500, n - 1):
        b = (q - torch.arange(n, device="cuda") + 32).clamp(0, 64)
        assert torch.equal(out[:, q], table.t()[:, b].to(torch.bfloat16))
    out.fill_(1.0)
    d = torch.empty(65, c, device="cuda")
    pe.relpos_bwd(h, pos, pos, ed, out, d, bytes_(pe.relpos_workspace_bytes(n, n, c, 65, "heads")), layout="heads")
    k = torch.arange(-32, 33, device="cuda").abs().double()
    count = n - k
    count[0] = count[64] = (n - 32) * (n - 31) / 2
    # counts are whole; those above 2^24 lose at most (additions in a row) half steps of the running sum
    assert bool(((d.double() - count[:, None]).abs() <= 1e-5 * count[:, None]).all()), d
    assert torch.equal(d[1:64].double(), count[1:64, None].expand(63, c))


# ---------------------------------------------------------------------------------------------------------------------


def test_refusals_raise(h):
    t, g = torch.zeros(4, 64, device="cuda", dtype=torch.bfloat16), torch.ones(64, device="cuda")
    y, st = torch.empty_like(t), torch.empty(4, 2, device="cuda")
    ws = bytes_(pe.layernorm_workspace_bytes(4, 64))
    bad = [
        (lambda: pe.layernorm_fwd(h, t.cpu(), g, g, y), "device"), (lambda: pe.layernorm_fwd(h, t.half(), g, g, y), "bfloat16"),
        (lambda: pe.layernorm_fwd(h, t, g, g, y[:3]), "differs"), (lambda: pe.layernorm_fwd(h, t, g[:63], g, y), "64 elements"),
        (lambda: pe.layernorm_fwd(h, t.t(), g, g, y), "neighbours"), (lambda: pe.layernorm_fwd(h, t, g, g, t), "overlaps"),
        (lambda: pe.layernorm_fwd(h, t, g, g, y, eps=0.0), "eps"), (lambda: pe.layernorm_fwd(h, t, g, g, y, ckpt=bytes_(255)), "bytes"),
        (lambda: pe.layernorm_bwd(h, t, y, st, g, None, g.clone(), None, ws[:256]), "workspace"),
        (lambda: pe.layernorm_bwd(h, t, y.float(), st, g, None, None, None, None), "differs"),
        (lambda: pe.ckpt_pack(h, t, bytes_(64)), "bytes"), (lambda: pe.ckpt_unpack(h, bytes_(4096)[8:], y), "256"),
        (lambda: pe.relpos_fwd(h, *[torch.zeros(4, dtype=torch.int32, device="cuda")] * 2, torch.tensor([1, 1], dtype=torch.int32), torch.zeros(3, 2, device="cuda"),
                               torch.zeros(4, 4, 2, device="cuda")), "ascend"),
        (lambda: pe.relpos_fwd(h, *[torch.zeros(4, dtype=torch.int32, device="cuda")] * 2, torch.tensor([0, 1], dtype=torch.int32), torch.zeros(3, 2, device="cuda"),
                               torch.zeros(4, 5, 2, device="cuda")), "shape"),
    ]
    for call, word in bad:
        with pytest.raises(pe.PEError, match=word):
            call()


def test_timing_and_checking_options(h):
    """The handle's options hold for the operators: results are the same, and the launches are listed."""
    rng = np.random.default_rng(8)
    x, y, y2, g = rand(rng, (100, 64), torch.bfloat16), *(torch.empty(100, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)), vec(rng, 64, 1.0)
    pe.layernorm_fwd(h, x, g, None, y)
    h2 = pe.Handle()
    h2.set_option(3, 1)
    h2.set_option(2, 1)
    pe.layernorm_fwd(h2, x, g, None, y2)
    assert torch.equal(y, y2)
    t = h2.timing_collect()
    assert [e["name"] for e in t] == ["layernorm fwd"] and t[0]["launches"] == 1 and t[0]["bytes"] == 2 * 2 * 6400


def _step(rng, n_res=40, c=64):
    """What a step has in hand: previous pair representation, positions of two chains, a trainable table and layer norm."""
    dt = torch.bfloat16
    st = dict(prev=rand(rng, (n_res, n_res, c), dt, 3.0), base=rand(rng, (n_res, n_res, c), dt), dy=rand(rng, (n_res, n_res, c), dt), g=vec(rng, c, 1.0), b=vec(rng, c),
              pos=torch.arange(n_res, dtype=torch.int32, device="cuda") % 23, seg=(torch.arange(n_res, device="cuda") // 23).int(), ed=torch.tensor(CLIP, dtype=torch.int32),
              table=vec(rng, 66 * c).view(66, c))
    e = lambda *s: torch.empty(*s, device="cuda")
    st.update(z=torch.empty_like(st["prev"]), stats=e(n_res * n_res, 2), kept=bytes_(pe.ckpt_bytes(n_res * n_res, c)), dprev=torch.empty_like(st["prev"]), dg=e(c), db=e(c),
              dtab=e(66, c), ws=bytes_(pe.layernorm_workspace_bytes(n_res * n_res, c)), ws2=bytes_(pe.relpos_workspace_bytes(n_res, n_res, c, 66)))
    return st


def _run_step(h, s, stream=None):
    """z = base + LN(prev) + relpos, with prev kept in 8 bits; then the gradients."""
    pe.layernorm_fwd(h, s["prev"], s["g"], s["b"], s["z"], add=s["base"], stats=s["stats"], ckpt=s["kept"], stream=stream)
    pe.relpos_fwd(h, s["pos"], s["pos"], s["ed"], s["table"], s["z"], s["seg"], s["seg"], add=s["z"], stream=stream)
    pe.relpos_bwd(h, s["pos"], s["pos"], s["ed"], s["dy"], s["dtab"], s["ws2"], s["seg"], s["seg"], stream=stream)
    pe.layernorm_bwd(h, s["dy"], s["kept"], s["stats"], s["g"], s["dprev"], s["dg"], s["db"], s["ws"], stream=stream)
    return [s[k] for k in ("z", "stats", "kept", "dprev", "dg", "db", "dtab")]


def test_step_repeats_on_other_streams_and_handles(h):
    s = _step(np.random.default_rng(9))
    first = [t.clone() for t in _run_step(h, s)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    h2 = pe.Handle()
    others = [_step(np.random.default_rng(9)) for _ in streams]
    torch.cuda.synchronize()
    for rep in range(3):                 # two handles on two streams at once, with buffers of their own
        for hh, st, o in zip((h, h2), streams, others):
            _run_step(hh, o, st)
    torch.cuda.synchronize()
    for o in others:
        assert all(torch.equal(a, o[k]) for a, k in zip(first, ("z", "stats", "kept", "dprev", "dg", "db", "dtab")))


def test_step_captured_and_replayed(h):
    """Two graphs of the same step on different inputs, with workspaces of their own, replayed in turn between eager work."""
    cases = [_step(np.random.default_rng(k)) for k in (10, 11)]
    want = [[t.clone() for t in _run_step(h, s)] for s in cases]
    torch.cuda.synchronize()
    graphs, st = [], torch.cuda.Stream()
    for s in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            _run_step(h, s, st)
        graphs.append(g)
    other = torch.randn(1 << 20, device="cuda")
    for rep in range(4):
        for s in cases:
            for k in ("z", "stats", "kept", "dprev", "dg", "db", "dtab", "ws", "ws2"):
                s[k].fill_(7)
        other = other * 1.0001 + 1.0
        torch.cuda.synchronize()
        for g in graphs if rep % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for s, w in zip(cases, want):
            assert all(torch.equal(s[k], t) for k, t in zip(("z", "stats", "kept", "dprev", "dg", "db", "dtab"), w)), rep
