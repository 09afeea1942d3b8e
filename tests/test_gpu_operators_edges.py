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
