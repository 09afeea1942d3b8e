"""The operators where the trunk uses them: block inputs saved in 8 bits by pe_stack_fwd_bwd, and one recycled step (layer norm of the
previous representations and relative positions into the trunk, the trunk with 8-bit checkpoints, the gradients back out)."""
import numpy as np
import pytest
import torch

import paper_2211_00235_amd as pe
from oracle.params import param_table
from pe_inputs import make_inputs, dims_for
from tests import op_reference as ref
from tests.gpu_util import to_dev, tdtype

pytestmark = pytest.mark.gpu
STACK_KEEP, STACK_CKPT = 5, 7          # pe_set_option numbers


def _bytes(n):
    return torch.empty(n, dtype=torch.uint8, device="cuda")


class Trunk:
    """A small trunk: dims, inputs on the device, and what a call writes."""

    def __init__(self, n_extra, n_main, dtype, variant=0, s=16, r=40):
        self.ne, self.nm = n_extra, n_main
        self.dm, mask, _ = dims_for("tiny")
        self.dm.update(dtype=dtype, s=s, r=r, variant=variant)
        self.de = dict(self.dm, s=24, c_m=16, col_global=1)
        (te, self.pe_n), (tm, self.pm_n) = param_table(self.de), param_table(self.dm)
        ie = make_inputs(self.de, te, self.pe_n, ("random_rows", 0.1), 61, n_blocks=max(n_extra, 1))
        im = make_inputs(self.dm, tm, self.pm_n, mask, 62, n_blocks=max(n_main, 1))
        dt, f32 = tdtype(self.dm), torch.float32
        self.ex, self.msa, self.pair = to_dev(ie["msa"], dt), to_dev(im["msa"], dt), to_dev(im["pair"], dt)
        self.exm, self.mm, self.pm = to_dev(ie["msa_mask"], f32), to_dev(im["msa_mask"], f32), to_dev(im["pair_mask"], f32)
        self.par = to_dev(np.concatenate([ie["params"]] * (n_extra > 0) + [im["params"]] * (n_main > 0)), f32)
        self.dmo, self.dzo = to_dev(im["d_msa_out"], dt), to_dev(im["d_pair_out"], dt)
        self.mo, self.zo, self.dmi, self.dzi = (torch.empty_like(t) for t in (self.msa, self.pair, self.msa, self.pair))
        self.dex, self.dpar = torch.empty_like(self.ex), torch.zeros_like(self.par)

    def workspace(self, **mode):
        ws = _bytes(pe.stack_workspace_bytes(self.ne, self.de if self.ne else None, self.nm, self.dm if self.nm else None, **mode))
        return ws.fill_(0x7F)     # large finite values wherever the call reads something it has not written

    def run(self, h, ws, sm, sp):
        pe.stack_fwd_bwd(h, self.ne, self.de if self.ne else None, self.nm, self.dm if self.nm else None,
                         self.ex if self.ne else None, self.msa if self.nm else None, self.pair, self.exm if self.ne else None,
                         self.mm if self.nm else None, self.pm, self.par, self.dmo if self.nm else None, self.dzo,
                         self.mo if self.nm else None, self.zo, self.dex if self.ne else None, self.dmi if self.nm else None,
                         self.dzi, self.dpar, ws, sm, sp)

    def outs(self):
        return [t for t, on in ((self.zo, 1), (self.mo, self.nm), (self.dzi, 1), (self.dex, self.ne), (self.dmi, self.nm), (self.dpar, 1)) if on]

    def chained(self, h, sm, sp):
        """The same by single-block calls, inputs of the blocks between the first and the last through an 8-bit checkpoint."""
        nb, ws = self.ne + self.nm, _bytes(max(pe.workspace_bytes(self.de, 1), pe.workspace_bytes(self.dm, 1)))
        off = lambda b: b * self.pe_n if b < self.ne else self.ne * self.pe_n + (b - self.ne) * self.pm_n
        of = lambda b: (self.de, self.exm, self.pe_n) if b < self.ne else (self.dm, self.mm, self.pm_n)
        xe, xm, zs = [self.ex], [self.msa], [self.pair]
        x_of = lambda b: xe[b] if b < self.ne else xm[b - self.ne]
        for b in range(nb):
            d, mask, n = of(b)
            xo, zo = torch.empty_like(x_of(b)), torch.empty_like(self.pair)
            pe.block_fwd(h, d, x_of(b), zs[b], mask, self.pm, self.par[off(b):off(b) + n], xo, zo, None, ws, sm, sp)
            (xe if b < self.ne else xm).append(xo)
            zs.append(zo)

        def kept(t):
            k, y = _bytes(pe.ckpt_bytes(t.numel() // t.shape[-1], t.shape[-1])), torch.empty_like(t)
            pe.ckpt_pack(h, t, k, sm)
            pe.ckpt_unpack(h, k, y, sm)
            return y
        dpar, gz, gm, ge = torch.zeros_like(self.par), self.dzo, self.dmo, torch.zeros_like(self.ex)
        for b in reversed(range(nb)):
            d, mask, n = of(b)
            x, z, is_e = x_of(b), zs[b], b < self.ne
            if 0 < b < nb - 1:
                z = kept(z)
                x = kept(x) if (b if is_e else b - self.ne) else x
            gx, gz2 = torch.empty_like(x), torch.empty_like(z)
            pe.block_bwd(h, d, x, z, mask, self.pm, self.par[off(b):off(b) + n], ge if is_e else gm, gz, gx, gz2, dpar[off(b):off(b) + n], None, ws, sm, sp)
            gz = gz2
            if is_e:
                ge = gx
            else:
                gm = gx
        return [t for t, on in ((zs[-1], 1), (xm[-1], self.nm), (gz, 1), (ge, self.ne), (gm, self.nm), (dpar, 1)) if on]


@pytest.mark.parametrize("two_streams", [True, False])
@pytest.mark.parametrize("dtype", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n_extra, n_main", [(0, 1), (0, 2), (0, 3), (0, 5), (1, 0), (3, 0), (1, 1), (2, 1), (1, 3), (3, 2)])
def test_stack_with_8_bit_checkpoints_equals_chained_blocks(n_extra, n_main, dtype, two_streams):
    t = Trunk(n_extra, n_main, dtype)
    h = pe.Handle()
    sm = torch.cuda.Stream() if two_streams else torch.cuda.current_stream()
    sp = torch.cuda.Stream() if two_streams else sm
    ws = t.workspace(ckpt=True)
    h.set_option(STACK_CKPT, 1)
    torch.cuda.synchronize()
    t.run(h, ws, sm, sp)
    torch.cuda.synchronize()
    want = t.chained(pe.Handle(), sm, sp)
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(t.outs(), want)):
        assert torch.equal(a, b), i


@pytest.mark.parametrize("variant", [1, 2])
def test_stack_with_8_bit_checkpoints_in_the_other_orderings(variant):
    t = Trunk(1, 4, 1, variant)
    h, sm, sp = pe.Handle(), torch.cuda.Stream(), torch.cuda.Stream()
    h.set_option(STACK_CKPT, 1)
    ws = t.workspace(ckpt=True)
    torch.cuda.synchronize()
    t.run(h, ws, sm, sp)
    torch.cuda.synchronize()
    want = t.chained(pe.Handle(), sm, sp)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(t.outs(), want))


def test_stack_checkpoint_option_leaves_outputs_and_refuses_kept_activations(capsys):
    """Outputs are the default's bits; gradients differ by what the restored inputs differ (reported); the options exclude each other."""
    t = Trunk(2, 4, 1, r=64)
    sm, sp = torch.cuda.Stream(), torch.cuda.Stream()
    h, h2 = pe.Handle(), pe.Handle()
    h2.set_option(STACK_CKPT, 1)
    ws, ws2 = t.workspace(), t.workspace(ckpt=True)
    torch.cuda.synchronize()
    t.run(h, ws, sm, sp)
    torch.cuda.synchronize()
    first = [o.clone() for o in t.outs()]
    t.dpar.zero_()
    torch.cuda.synchronize()
    t.run(h2, ws2, sm, sp)
    torch.cuda.synchronize()
    assert torch.equal(first[0], t.zo) and torch.equal(first[1], t.mo)
    far = [float((a.double() - b.double()).norm() / b.double().norm()) for a, b in zip(t.outs()[2:], first[2:])]
    with capsys.disabled():
        print("\n  gradients with 8-bit checkpoints against the default, 2 + 4 blocks, rel 2-norm: " + ", ".join("%.1e" % f for f in far))
    assert all(np.isfinite(far))
    h2.set_option(STACK_KEEP, 1)
    with pytest.raises(pe.PEError, match="set one of them"):
        t.run(h2, t.workspace(keep=True), sm, sp)
    h.set_option(STACK_CKPT, 1)
    with pytest.raises(pe.PEError, match="workspace too small"):
        t.run(h, _bytes(4096), sm, sp)


def test_recycled_step():
    _recycled_step(False)


def test_recycled_step_captured():
    _recycled_step(True)


def _recycled_step(capture):
    """z0 = pair + LN(prev pair) + relpos, m0[0] = msa[0] + LN(prev msa[0]); the trunk with 8-bit checkpoints; gradients of the
    relative positions' table and of both layer norms from the cotangents that come out of the trunk.  The trunk's own result is that of
    its call on z0, m0; the operators' results are compared with their float64 definitions at their inputs."""
    t = Trunk(1, 3, 1, r=48)
    s, r, cm, cz = t.dm["s"], t.dm["r"], t.dm["c_m"], t.dm["c_z"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    rnd = lambda *sh: torch.randn(*sh, generator=gen, device="cuda")
    prev_z, prev_m = (2 * rnd(r, r, cz)).bfloat16(), (2 * rnd(r, cm)).bfloat16()
    gz, bz, gm, bm = 1 + 0.1 * rnd(cz), 0.1 * rnd(cz), 1 + 0.1 * rnd(cm), 0.1 * rnd(cm)
    pos, seg = (torch.arange(r, device="cuda") % 29).int(), (torch.arange(r, device="cuda") // 29).int()
    edges, table = torch.arange(-31, 33, dtype=torch.int32), 0.3 * rnd(66, cz)
    base_z, base_m = t.pair.clone(), t.msa.clone()
    st_z, st_m = torch.empty(r * r, 2, device="cuda"), torch.empty(r, 2, device="cuda")
    k_z, k_m = _bytes(pe.ckpt_bytes(r * r, cz)), _bytes(pe.ckpt_bytes(r, cm))
    grads = [torch.empty(n, device="cuda") for n in (cz, cz, cm, cm)]
    dtab = torch.empty(66, cz, device="cuda")
    h, sm, sp = pe.Handle(), torch.cuda.Stream(), torch.cuda.Stream()
    h.set_option(STACK_CKPT, 1)
    ws = t.workspace(ckpt=True)
    w1, w2, w3 = _bytes(pe.layernorm_workspace_bytes(r * r, cz)), _bytes(pe.layernorm_workspace_bytes(r, cm)), _bytes(pe.relpos_workspace_bytes(r, r, cz, 66))

    def step():
        pe.layernorm_fwd(h, prev_z, gz, bz, t.pair, add=base_z, stats=st_z, ckpt=k_z, stream=sm)
        pe.relpos_fwd(h, pos, pos, edges, table, t.pair, seg, seg, add=t.pair, stream=sm)
        pe.layernorm_fwd(h, prev_m, gm, bm, t.msa[0], add=base_m[0], stats=st_m, ckpt=k_m, stream=sm)
        t.run(h, ws, sm, sp)
        pe.relpos_bwd(h, pos, pos, edges, t.dzi, dtab, w3, seg, seg, stream=sm)
        pe.layernorm_bwd(h, t.dzi, k_z, st_z, gz, None, grads[0], grads[1], w1, stream=sm)       # recycled inputs need no gradient
        pe.layernorm_bwd(h, t.dmi[0], k_m, st_m, gm, None, grads[2], grads[3], w2, stream=sm)
    torch.cuda.synchronize()
    step()
    torch.cuda.synchronize()
    outs = t.outs() + [t.pair, t.msa, dtab, *grads]
    if capture:
        want = [o.clone() for o in outs]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=sm):
            step()
        other = torch.randn(1 << 20, device="cuda")
        for rep in range(3):
            for o in outs:
                o.zero_()
            t.msa.copy_(base_m)
            ws.fill_(0x7F)
            other = other * 1.0001 + 1.0
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), rep
        return
    f64 = lambda x: x.detach().cpu().double().numpy()
    half, u = torch.finfo(torch.bfloat16).eps / 2, 2.0 ** -24
    # z0 is rounded twice, after the layer norm and after the relative positions; fp32 in between (48 additions in a row at most)
    y, mean, rstd = ref.layernorm(f64(prev_z).reshape(-1, cz), f64(gz), f64(bz), 1e-5, f64(base_z).reshape(-1, cz))
    b = ref.buckets(f64(pos), f64(pos), list(range(-31, 33)), f64(seg), f64(seg))
    rel = f64(table)[b].reshape(-1, cz)
    x = f64(prev_z).reshape(-1, cz)
    size = (np.abs(x) + np.abs(x).mean(1, keepdims=True)) * rstd[:, None] * np.abs(f64(gz)) + np.abs(f64(bz)) + np.abs(f64(base_z).reshape(-1, cz)) + np.abs(rel)
    assert (np.abs(f64(t.pair).reshape(-1, cz) - (y + rel)) <= 1.01 * half * (np.abs(y) + np.abs(y + rel)) + 64 * u * size).all()
    assert torch.equal(t.msa[1:], base_m[1:])
    y, _, rstd = ref.layernorm(f64(prev_m), f64(gm), f64(bm), 1e-5, f64(base_m[0]))
    x = f64(prev_m)
    size = (np.abs(x) + np.abs(x).mean(1, keepdims=True)) * rstd[:, None] * np.abs(f64(gm)) + np.abs(f64(bm)) + np.abs(f64(base_m[0]))
    assert (np.abs(f64(t.msa[0]) - y) <= 1.01 * half * np.abs(y) + 48 * u * size).all()
    # the trunk on these inputs
    want = t.chained(pe.Handle(), sm, sp)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(t.outs(), want))
    # gradients: sums over r r and r rows, additions in a row as in the operators' own tests
    d = f64(t.dzi)
    exact = ref.relpos_bwd(b, d, 66)
    assert (np.abs(f64(dtab) - exact) <= (64 + r * r / 4) * u * ref.relpos_bwd(b, np.abs(d), 66)).all()
    for prev, st, g, dy, (dg, db), rows, c in ((prev_z, st_z, gz, t.dzi, grads[:2], r * r, cz), (prev_m, st_m, gm, t.dmi[0], grads[2:], r, cm)):
        back = ref.ckpt(f64(prev).reshape(rows, c))[2]
        mean, rstd = f64(st)[:, 0], f64(st)[:, 1]
        dyy = f64(dy).reshape(rows, c)
        _, eg, eb = ref.layernorm_bwd(back, mean, rstd, f64(g), dyy)
        zz = (np.abs(back) + np.abs(mean)[:, None]) * rstd[:, None]
        assert (np.abs(f64(dg) - eg) <= (64 + rows / 64) * u * (np.abs(dyy) * zz).sum(0)).all()
        assert (np.abs(f64(db) - eb) <= (64 + rows / 64) * u * np.abs(dyy).sum(0)).all()
