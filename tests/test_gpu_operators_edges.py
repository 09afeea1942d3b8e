"""The operators around the trunk at starts, gaps, sizes and arguments beside those of tests/test_gpu_operators.py, against the same
float64 definitions (tests/op_reference.py).  Checkpoints and gradients of whole numbers are compared bit for bit."""
import numpy as np
import pytest
import torch

import paper_2211_00235_amd as pe
from tests import op_reference as ref

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16]


@pytest.fixture(scope="module")
def h():
    return pe.Handle()


def f64(t):
    return t.detach().cpu().double().numpy()


def bytes_(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("off", [1, 3, 8])
@pytest.mark.parametrize("rows, c", [(300, 64), (1, 4096), (1, 100000), (100, 32), (45, 128), (2, 100000), (700, 40), (9, 2)])
def test_ckpt_of_views_without_gaps(h, rows, c, off, dt):
    """Rows without gaps that start anywhere in a buffer, more of them than one wave takes."""
    rng = np.random.default_rng(rows + c + off)
    n = rows * c
    buf = torch.from_numpy(rng.normal(size=n + 32)).to(dt).cuda()
    out = torch.from_numpy(rng.normal(size=n + 32)).to(dt).cuda()
    was, view = out.clone(), lambda t: t[off:off + n].view(rows, c)
    kept = bytes_(pe.ckpt_bytes(rows, c)).fill_(0xA5)
    pe.ckpt_pack(h, view(buf), kept)
    codes, scales, back = ref.ckpt(f64(view(buf)))
    k, at = kept.cpu().numpy(), -(-n // 256) * 256
    assert np.array_equal(k[:n].view(np.int8).reshape(rows, c), codes)
    assert np.array_equal(k[at:at + scales.size].reshape(scales.shape), scales)
    pe.ckpt_unpack(h, kept, view(out))
    assert np.array_equal(f64(view(out)), back)
    assert torch.equal(out[:off], was[:off]) and torch.equal(out[off + n:], was[off + n:])


def _busy(stream):
    """Some milliseconds of work on a stream, in front of what a test queues on it."""
    a = torch.ones(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(20):
            a = a @ a * 2.0 ** -12
    return a


def _chain(h, t):
    """z = x + LN(prev) + table[bucket], kept in 8 bits and restored; gradients of the table and of the layer norm.  No call names a stream."""
    t["x"].copy_(t["x0"], non_blocking=True)
    t["prev"].copy_(t["prev0"], non_blocking=True)
    pe.layernorm_fwd(h, t["prev"], t["g"], t["b"], t["z"], add=t["x"], stats=t["stats"])
    pe.relpos_fwd(h, t["pos"], t["pos"], t["edges"], t["table"], t["z"], add=t["z"])
    pe.ckpt_pack(h, t["z"], t["kept"])
    pe.ckpt_unpack(h, t["kept"], t["back"])
    pe.relpos_bwd(h, t["pos"], t["pos"], t["edges"], t["back"], t["dtab"], t["wt"])
    pe.layernorm_bwd(h, t["back"], t["prev"], t["stats"], t["g"], t["dprev"], t["dg"], t["db"], t["wl"])
    return [t[k] for k in ("z", "stats", "kept", "back", "dtab", "dprev", "dg", "db")]


def _chain_state(seed, n=48, c=64):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    e = lambda *s: torch.zeros(*s, device="cuda")
    t = dict(x0=rnd(n, n, c).bfloat16(), prev0=rnd(n, n, c).bfloat16(), g=1 + 0.1 * rnd(c), b=0.1 * rnd(c), table=rnd(65, c), pos=torch.arange(n, dtype=torch.int32, device="cuda"),
             edges=torch.arange(-31, 33, dtype=torch.int32), stats=e(n * n, 2), dtab=e(65, c), dg=e(c), db=e(c), kept=bytes_(pe.ckpt_bytes(n * n, c)),
             wt=bytes_(pe.relpos_workspace_bytes(n, n, c, 65)), wl=bytes_(pe.layernorm_workspace_bytes(n * n, c)))
    t.update({k: torch.zeros_like(t["x0"]) for k in ("x", "prev", "z", "back", "dprev")})
    return t


def test_operators_without_a_stream_follow_the_current_one(h):
    """Inside torch.cuda.stream(s) the calls run behind what is queued on s."""
    t, s = _chain_state(1), torch.cuda.Stream()
    want = [o.clone() for o in _chain(h, t)]
    for o in _chain(h, t):
        o.zero_()
    t["x"].zero_(), t["prev"].zero_()
    _busy(s)
    with torch.cuda.stream(s):
        got = _chain(h, t)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_operators_without_a_stream_are_captured(h):
    """Inside torch.cuda.graph the current stream is the one that is captured."""
    t = _chain_state(2)
    want = [o.clone() for o in _chain(h, t)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = _chain(h, t)
    other = torch.randn(1 << 20, device="cuda")
    for rep in range(3):
        for o in outs:
            o.fill_(7)
        other = other * 1.0001 + 1.0
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), rep


def test_block_without_streams_follows_the_current_one():
    from oracle.params import param_table
    from paper_2211_00235_amd.harness import BlockRun
    from pe_inputs import dims_for, make_inputs
    dims, mask, seed = dims_for("tiny")
    table, n = param_table(dims)
    run = BlockRun(dims, make_inputs(dims, table, n, mask, seed), two_streams=False)

    def both(**k):
        pe.block_fwd(run.h, dims, run.msa, run.pair, run.msa_mask, run.pair_mask, run.params, run.msa_out, run.pair_out, run.ctx, run.ws, **k)
        pe.block_bwd(run.h, dims, run.msa, run.pair, run.msa_mask, run.pair_mask, run.params, run.d_msa_out, run.d_pair_out, run.d_msa_in, run.d_pair_in, run.d_params,
                     run.ctx, run.ws, **k)
        return [run.msa_out, run.pair_out, run.d_msa_in, run.d_pair_in, run.d_params]
    s = torch.cuda.Stream()
    want = [o.clone() for o in both(stream_msa=s, stream_pair=s) if not s.synchronize()]
    msa, outs = run.msa.clone(), [run.msa_out, run.pair_out, run.d_msa_in, run.d_pair_in, run.d_params]
    for o in [run.msa, *outs]:
        o.zero_()
    _busy(s)
    with torch.cuda.stream(s):
        run.msa.copy_(msa)
        got = both()
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---------------------------------------------------------------------------------------------------------------------
# Relative positions, pair layout, rows with gaps: the gradient's kernel without the matrix unit, whose variants go with the channels
# (9..16: four positions per wave, 17..32: two, more: one and slabs of 64 channels) and whose waves go with the buckets (256: two)
CLIP, LOG = list(range(-31, 33)), [-90, -31, -15, -7, -2, -1, 0, 1, 2, 3, 8, 16, 32, 91]
MANY = [3 * i - 381 for i in range(254)]


def rp_inputs(rng, n_q, n_k, edges, segs, c):
    """Positions in ascending order (runs of a bucket) for odd counts, in any order for even ones."""
    span = max(4, n_q + n_k)
    pos = lambda n: torch.from_numpy(np.sort(rng.integers(-span, span, n)) if n % 2 else rng.integers(-span, span, n)).int().cuda()
    seg = lambda n: torch.from_numpy(rng.integers(0, 3, n)).int().cuda()
    pq, pk = pos(n_q), pos(n_k)
    sq, sk = (seg(n_q), seg(n_k)) if segs else (None, None)
    nb = len(edges) + (2 if segs else 1)
    b = ref.buckets(pq.cpu().numpy(), pk.cpu().numpy(), edges, *(t.cpu().numpy() if segs else None for t in (sq, sk)))
    table = torch.from_numpy(rng.normal(size=(nb, c))).float().cuda()
    return pq, pk, torch.tensor(edges, dtype=torch.int32), sq, sk, table, b, nb


def rp_check(h, dt, rng, inputs, view, c):
    """Forward into the view, in place onto it, and the gradient of what is in it: whole numbers exactly, normal ones as a sum of n
    terms with at most n / 4 + 64 additions in a row."""
    pq, pk, ed, sq, sk, table, b, nb = inputs
    n_q, n_k = b.shape
    T = f64(table)
    pe.relpos_fwd(h, pq, pk, ed, table, view, sq, sk)
    want = ref.relpos(b, T, None, "pair")
    assert np.array_equal(f64(view), f64(torch.from_numpy(want).float().to(dt)))
    A = f64(view)
    pe.relpos_fwd(h, pq, pk, ed, table, view, sq, sk, add=view)
    want, half = ref.relpos(b, T, A, "pair"), torch.finfo(dt).eps / 2
    assert (np.abs(f64(view) - want) <= (half * (1 + 1e-6) + U) * np.abs(want)).all()
    ws, d = bytes_(pe.relpos_workspace_bytes(n_q, n_k, c, nb)), torch.full((nb, c), 3.0, device="cuda")
    view.copy_(torch.from_numpy(rng.integers(-8, 9, size=(n_q, n_k, c))))
    exact = ref.relpos_bwd(b, f64(view), nb)
    pe.relpos_bwd(h, pq, pk, ed, view, d, ws, sq, sk)
    assert np.array_equal(f64(d), exact)
    pe.relpos_bwd(h, pq, pk, ed, view, d, ws, sq, sk, accumulate=True)
    assert np.array_equal(f64(d), 2 * exact)
    view.copy_(torch.from_numpy(rng.normal(size=(n_q, n_k, c))))
    pe.relpos_bwd(h, pq, pk, ed, view, d, ws, sq, sk)
    g = f64(view)
    assert (np.abs(f64(d) - ref.relpos_bwd(b, g, nb)) <= (64 + n_q * n_k / 4) * U * ref.relpos_bwd(b, np.abs(g), nb)).all()


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("edges, segs", [(CLIP, True), (LOG, False), (MANY, True), ([], False)], ids=["clip", "log", "many", "none"])
@pytest.mark.parametrize("c", [9, 16, 17, 24, 32, 33, 64, 65, 130])
def test_relpos_pair_rows_with_gaps(h, c, edges, segs, dt):
    rng = np.random.default_rng(c)
    for n_q, n_k, gap, off in ((37, 64, 13, 0), (130, 41, 8, 0), (19, 67, 1, 3), (3, 5, 16, 1), (9, 1, 40, 0)):
        ld = n_k * c + gap
        buf = torch.from_numpy(rng.normal(size=n_q * ld + off + 8)).to(dt).cuda()
        was, view = buf.clone(), torch.as_strided(buf, (n_q, n_k, c), (ld, c, 1), off)
        rp_check(h, dt, rng, rp_inputs(rng, n_q, n_k, edges, segs, c), view, c)
        view.copy_(torch.as_strided(was, view.shape, view.stride(), off))
        assert torch.equal(buf, was)


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
@pytest.mark.parametrize("n_q, n_k, c", [(1, 1, 17), (1, 15, 40), (15, 1, 65), (3, 5, 130), (1, 16, 17), (4, 4, 64)])
def test_relpos_pair_fewer_positions_than_a_batch(h, n_q, n_k, c, dt):
    """Around 16 positions, where the matrix unit's kernel begins."""
    rng = np.random.default_rng(c)
    rp_check(h, dt, rng, rp_inputs(rng, n_q, n_k, CLIP, True, c), torch.empty(n_q, n_k, c, dtype=dt, device="cuda"), c)


@pytest.mark.parametrize("dt", TYPES, ids=["fp32", "bf16"])
def test_relpos_pair_rows_4_gb_apart(h, dt):
    """Three rows whose offsets pass 32 bits; what lies between them is not touched, so it is not set either."""
    ld = 1_100_000_000 if dt is torch.bfloat16 else 600_000_000
    buf = torch.empty(2 * ld + 40 * 130 + 8, dtype=dt, device="cuda")
    for c in (8, 16, 24, 64, 130):
        rng = np.random.default_rng(c)
        edge = [buf[q * ld + 40 * c:q * ld + 40 * c + 8] for q in range(3)]      # behind the rows
        for e in edge:
            e.fill_(5.0)
        rp_check(h, dt, rng, rp_inputs(rng, 3, 40, CLIP, True, c), torch.as_strided(buf, (3, 40, c), (ld, c, 1)), c)
        assert all(bool((e == 5.0).all()) for e in edge)


def test_ckpt_of_more_workgroups_than_a_grid_row(h):
    """2^29 + 300 rows of one channel: 2^22 workgroups and three more, items past 2^32."""
    rows = 2 ** 29 + 300
    x = torch.randn(rows, 1, dtype=torch.bfloat16, device="cuda")
    y, kept = torch.full_like(x, float("nan")), bytes_(pe.ckpt_bytes(rows, 1)).fill_(0xA5)
    pe.ckpt_pack(h, x, kept)
    pe.ckpt_unpack(h, kept, y)
    at = -(-rows // 256) * 256
    for part in (slice(0, 3000), slice(2 ** 29 - 3000, rows)):
        codes, scales, back = ref.ckpt(f64(x[part]))
        assert np.array_equal(kept[:rows][part].cpu().numpy().view(np.int8), codes[:, 0])
        assert np.array_equal(kept[at:at + rows][part].cpu().numpy(), scales[:, 0])
        assert np.array_equal(f64(y[part]), back)
    for a in range(0, rows, 2 ** 27):                        # all of them: off by at most half a step of 64 to 127
        p, q = x[a:a + 2 ** 27].float(), y[a:a + 2 ** 27].float()
        assert bool(((p - q).abs() <= p.abs() / 127).all()), a
