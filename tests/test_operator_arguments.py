"""Arguments of the operators around the trunk from Python, as far as no GPU is needed: what the marshalling itself has to refuse."""
from types import SimpleNamespace

import pytest
import torch

import paper_2211_00235_amd as pe
from paper_2211_00235_amd import binding

WIDE = 2 ** 32 + 64          # 64 in 32 bits
HOST = SimpleNamespace(device=-1)      # a handle for tensors that are on no GPU, for the marshalling alone


def test_size_queries_refuse_sizes_past_32_bits():
    assert pe.ckpt_bytes(1, WIDE) == 0 and pe.layernorm_workspace_bytes(1, WIDE) == 0
    for layout in ("pair", "heads"):
        assert pe.relpos_workspace_bytes(WIDE, 3, 4, 5, layout) == 0 and pe.relpos_workspace_bytes(3, WIDE, 4, 5, layout) == 0
        assert pe.relpos_workspace_bytes(3, 3, WIDE, 5, layout) == 0 and pe.relpos_workspace_bytes(3, 3, 4, WIDE, layout) == 0
        assert pe.relpos_workspace_bytes(3, 3, -WIDE, 5, layout) == 0


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_tensors_with_axes_past_32_bits_are_refused(dt):
    meta = lambda *shape, dtype=dt: torch.empty(*shape, dtype=dtype, device="meta")
    with pytest.raises(pe.PEError, match="channels"):
        binding._rows(HOST, meta(WIDE), "x")
    with pytest.raises(pe.PEError, match="channels"):
        binding._rows(HOST, meta(2, WIDE), "x")
    assert binding._rows(HOST, meta(WIDE, 64), "x")[1:] == (WIDE, 64, 64)      # rows may be as many
    edges = torch.tensor([0], dtype=torch.int32)
    pos = lambda n: meta(n, dtype=torch.int32)
    for n_q, n_k, c in ((WIDE, 1, 1), (1, WIDE, 1), (1, 1, WIDE)):
        with pytest.raises(pe.PEError, match="wanted"):
            binding._relpos(HOST, pos(n_q), pos(n_k), edges, meta(n_q, n_k, c), None, None, "pair", "out")
        with pytest.raises(pe.PEError, match="wanted"):
            binding._relpos(HOST, pos(n_q), pos(n_k), edges, meta(c, n_q, n_k), None, None, "heads", "out")


class _Recorder:
    """In the library's place: every call's arguments, nothing run."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 0
        return call


def _streams(args):
    return [getattr(a, "value", a) or None for a in args[-2:]]


def test_calls_without_a_stream_run_on_the_current_one(monkeypatch):
    """None is torch's current stream on the handle's device, 0 the default stream, and a stream that is given is that stream."""
    seen, rec = [], _Recorder()
    monkeypatch.setattr(binding, "_current_stream", lambda device: seen.append(device) or 4096, raising=False)
    monkeypatch.setattr(binding, "lib", lambda: rec)
    h = SimpleNamespace(device=-1, _h=None, last_error=lambda: "")
    f = lambda *shape: torch.zeros(*shape)
    i = lambda n: torch.zeros(n, dtype=torch.int32)
    x, kept, st, ws = f(4, 8), torch.zeros(512, dtype=torch.uint8), f(4, 2), torch.zeros(4096, dtype=torch.uint8)
    dims = dict(s=1, r=1, c_m=8, c_z=8, h_msa=1, d_msa=8, h_pair=1, d_pair=8, c_tri=8, c_opm=8, n_trans=1, col_global=0, dtype=0, ln_eps=1e-5, opm_eps=1e-3)
    p = [16] * 9
    one = [lambda **k: pe.layernorm_fwd(h, x, None, None, f(4, 8), **k), lambda **k: pe.layernorm_bwd(h, x, x, st, None, f(4, 8), None, None, None, **k),
           lambda **k: pe.ckpt_pack(h, x, kept, **k), lambda **k: pe.ckpt_unpack(h, kept, x, **k),
           lambda **k: pe.relpos_fwd(h, i(4), i(3), i(1), f(2, 8), f(4, 3, 8), **k), lambda **k: pe.relpos_bwd(h, i(4), i(3), i(1), f(4, 3, 8), f(2, 8), ws, **k)]
    for call in one:
        for k, want in (({}, 4096), ({"stream": 0}, None), ({"stream": SimpleNamespace(cuda_stream=77)}, 77)):
            call(**k)
            assert _streams(rec.calls[-1][1])[-1] == want, rec.calls[-1][0]
    for call in (lambda *s: pe.block_fwd(h, dims, *p[:5], *p[:2], None, ws, *s), lambda *s: pe.block_bwd(h, dims, *p, None, None, ws, *s),
                 lambda *s: pe.block_fwd_static(h, dims, *p[:7], *s), lambda *s: pe.stack_fwd_bwd(h, 0, None, 1, dims, *p, *p[:6], ws, *s)):
        for s, want in (((), [4096, 4096]), ((5, 6), [5, 6]), ((0, 0), [None, None])):
            call(*s)
            assert _streams(rec.calls[-1][1])[-2:] == want, rec.calls[-1][0]
    assert set(seen) == {-1}


def test_relpos_backward_without_a_workspace_is_refused():
    i = lambda n: torch.zeros(n, dtype=torch.int32)
    with pytest.raises(pe.PEError, match="workspace"):
        pe.relpos_bwd(HOST, i(4), i(3), i(1), torch.zeros(4, 3, 8), torch.zeros(2, 8), None)


def test_relpos_add_laid_out_as_out(monkeypatch):
    """One row of a bias, [c][1][k] with gaps between the heads: the stride of the axis of one element may be any."""
    rec = _Recorder()
    monkeypatch.setattr(binding, "lib", lambda: rec)
    h = SimpleNamespace(device=-1, _h=None, last_error=lambda: "")
    i, bias = (lambda n: torch.zeros(n, dtype=torch.int32)), torch.zeros(6, 5, 40)
    call = lambda out, add: pe.relpos_fwd(h, i(out.shape[1]), i(40), i(1), torch.zeros(2, 6), out, add=add, layout="heads")
    row, same = bias[:, 2:3], torch.zeros(6, 200)[:, :40].as_strided((6, 1, 40), (200, 200, 1))
    assert row.stride() != same.stride()
    call(row, same)
    call(same, row)
    assert len(rec.calls) == 2 and rec.calls[0][1][0] is None
    for out, add in ((row, torch.zeros(6, 1, 40)), (row, torch.zeros(6, 7, 40)[:, 2:3]), (bias, bias.transpose(0, 1).contiguous().transpose(0, 1)), (row, same.bfloat16()), (row, bias[:, 2:4])):
        with pytest.raises(pe.PEError, match="add"):
            call(out, add)
