"""The float64 definitions that the operators' GPU tests compare with, pinned by loops and central differences (CPU), and the
operators' refusals, which need no GPU."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import paper_2211_00235_amd as pe
from paper_2211_00235_amd import binding
from tests import op_reference as ref


def test_layernorm_backward_by_differences():
    rng = np.random.default_rng(0)
    x, g, b, dy = rng.normal(size=(3, 7)), rng.normal(size=7), rng.normal(size=7), rng.normal(size=(3, 7))
    y, mean, rstd = ref.layernorm(x, g, b)
    dx, dg, db = ref.layernorm_bwd(x, mean, rstd, g, dy)
    loss = lambda *a: float((ref.layernorm(*a)[0] * dy).sum())
    h = 1e-6
    for i in np.ndindex(*x.shape):
        e = np.zeros_like(x)
        e[i] = h
        assert abs((loss(x + e, g, b) - loss(x - e, g, b)) / (2 * h) - dx[i]) < 1e-6
    for i in range(7):
        e = np.zeros(7)
        e[i] = h
        assert abs((loss(x, g + e, b) - loss(x, g - e, b)) / (2 * h) - dg[i]) < 1e-6
        assert abs((loss(x, g, b + e) - loss(x, g, b - e)) / (2 * h) - db[i]) < 1e-6


def test_ckpt_by_loops():
    rng = np.random.default_rng(1)
    x = (rng.normal(size=(4, 70)) * np.exp2(rng.integers(-140, 100, size=(4, 1)))).astype(np.float32).astype(np.float64)
    x[1, 5] = 127.0 * 2.0 ** 40
    x[2, 40] = np.inf
    x[3, :32] = 0.0
    codes, scales, back = ref.ckpt(x)
    for r in range(4):
        for j in range(3):
            v = x[r, 32 * j:32 * (j + 1)]
            if not np.isfinite(v).all():
                assert scales[r, j] == 255 and np.isnan(back[r, 32 * j:32 * (j + 1)]).all()
                continue
            e = int(scales[r, j]) - 127
            top = max(abs(t) for t in v)
            assert e >= -126 and top <= 127 * 2.0 ** e and (e == -126 or top > 127 * 2.0 ** (e - 1))
            for k, t in enumerate(v):
                q = int(codes[r, 32 * j + k])
                assert abs(q) <= 127 and abs(t - q * 2.0 ** e) <= 2.0 ** (e - 1) and back[r, 32 * j + k] == q * 2.0 ** e
    again = ref.ckpt(np.nan_to_num(back))[2]
    assert np.array_equal(again[np.isfinite(back)], back[np.isfinite(back)])


def test_relpos_by_loops():
    rng = np.random.default_rng(2)
    pq, pk, sq, sk = rng.integers(-50, 50, 5), rng.integers(-50, 50, 6), rng.integers(0, 2, 5), rng.integers(0, 2, 6)
    edges, t, d = [-9, -3, 0, 1, 20], rng.normal(size=(7, 3)), rng.normal(size=(5, 6, 3))
    b = ref.buckets(pq, pk, edges, sq, sk)
    out, want = ref.relpos(b, t, d), np.zeros((7, 3))
    for i in range(5):
        for j in range(6):
            n = 6 if sq[i] != sk[j] else sum(int(pq[i]) - int(pk[j]) >= e for e in edges)
            assert b[i, j] == n and np.array_equal(out[i, j], d[i, j] + t[n])
            want[n] += d[i, j]
    assert np.allclose(ref.relpos_bwd(b, d, 7), want, rtol=0, atol=1e-12)
    assert np.allclose(ref.relpos_bwd(b, np.moveaxis(d, 2, 0), 7, "heads"), want, rtol=0, atol=1e-12)
    assert np.array_equal(ref.relpos(b, t, layout="heads")[1, 2], t[b[2], 1])


def test_sizes():
    assert pe.ckpt_bytes(0, 8) == 0 and pe.ckpt_bytes(3, 33) == 256 + 6 and pe.ckpt_bytes(256, 128) == 256 * 128 + 256 * 4
    for rows, c in ((-1, 8), (1, 0), (1, (1 << 20) + 1), (1 << 41, 1)):
        assert pe.ckpt_bytes(rows, c) == 0
    assert pe.layernorm_workspace_bytes(0, 8) > 0 and pe.layernorm_workspace_bytes(1, 16385) == 0
    for rows in (1, 5, 1000, 10 ** 6):
        for c in (1, 8, 33, 256, 16384):
            w = pe.layernorm_workspace_bytes(rows, c)
            assert w >= 8 * c and w % 256 == 0
    assert pe.relpos_workspace_bytes(5, 7, 3, 256) > 0 and pe.relpos_workspace_bytes(5, 7, 3, 257) == 0
    assert pe.relpos_workspace_bytes(5, 7, 1025, 4) == 0 and pe.relpos_workspace_bytes(-1, 7, 3, 4, "heads") == 0
    assert pe.relpos_workspace_bytes(0, 7, 3, 1) > 0


def test_without_a_handle():
    L = pe.lib()
    p = binding._Relpos(1, 1, 1, 0, 0, 0, 0, 0)
    assert L.pe_handle_device(None) == -1
    assert L.pe_layernorm_fwd(None, 1, 1, 0, None, 1, None, 1, None, None, 1e-5, None, 1, None, None, None) == -1
    assert L.pe_layernorm_bwd(None, 1, 1, 0, 0, None, 1, None, None, None, 1, None, 1, None, 1, None, None, 0, None, 0, None) == -1
    assert L.pe_ckpt_pack(None, 1, 1, 0, None, 1, None, None) == -1 and L.pe_ckpt_unpack(None, 1, 1, 0, None, None, 1, None) == -1
    assert L.pe_relpos_fwd(None, C.byref(p), *[None] * 9) == -1
    assert L.pe_relpos_bwd(None, C.byref(p), *[None] * 7, 0, None, 0, None) == -1


def test_refusals_under_sanitizers(tmp_path):
    """Every refusal of the operators' entry points comes before any HIP call: tests/host_checks/ops_host_check.cpp makes the calls
    on the CPU, with the host code instrumented."""
    from paper_2211_00235_amd import build
    exe = build.build_host_check(str(tmp_path / "ops_host_check"), program="ops_host_check.cpp", sources=["pe_ops.hip"])
    res = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stdout + res.stderr
    assert res.stdout.startswith("ok "), res.stdout + res.stderr
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr, res.stderr


def test_declared_in_the_header():
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pe.h")).read()
    for name in ("pe_layernorm_fwd", "pe_layernorm_bwd", "pe_layernorm_workspace_bytes", "pe_ckpt_bytes", "pe_ckpt_pack",
                 "pe_ckpt_unpack", "pe_relpos_fwd", "pe_relpos_bwd", "pe_relpos_workspace_bytes"):
        assert name + "(" in hdr and hasattr(pe.lib(), name)


@pytest.mark.parametrize("layout", ["pair", "heads"])
def test_workspace_grows_with_what_it_holds(layout):
    small, large = (pe.relpos_workspace_bytes(n, n, 16, 33, layout) for n in (8, 512))
    assert 0 < small <= large


@pytest.mark.parametrize("name", ["tiny", "af2_initial"])
def test_trunk_workspace_with_8_bit_checkpoints(name):
    """Saved inputs of the blocks between the first and the last take their 8-bit size; two of each kind are held as they are."""
    from pe_inputs import CONFIGS
    d = dict(CONFIGS[name][0])
    up = lambda n: (n + 255) // 256 * 256
    size = {0: 4, 1: 2}[d["dtype"]]
    z, m = up(d["r"] ** 2 * d["c_z"] * size), up(d["s"] * d["r"] * d["c_m"] * size)
    kz, km = up(pe.ckpt_bytes(d["r"] ** 2, d["c_z"])), up(pe.ckpt_bytes(d["s"] * d["r"], d["c_m"]))
    for n in (1, 2, 3, 8, 48):
        plain, ckpt = pe.stack_workspace_bytes(0, None, n, d), pe.stack_workspace_bytes(0, None, n, d, ckpt=True)
        assert plain - ckpt == (n - 1) * (z + m) - max(0, n - 2) * (kz + km) - 2 * (z + m)
    e = dict(CONFIGS["extra_msa"][0], r=d["r"], c_z=d["c_z"], dtype=d["dtype"])
    assert 0 < pe.stack_workspace_bytes(4, e, 48, d, ckpt=True) < pe.stack_workspace_bytes(4, e, 48, d)
    assert pe.stack_workspace_bytes(0, None, 0, None, ckpt=True) == 0
