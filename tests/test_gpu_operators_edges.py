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
