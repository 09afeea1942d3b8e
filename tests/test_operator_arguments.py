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
