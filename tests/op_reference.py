"""Plain float64 definitions of the operators around the trunk (numpy), which the GPU tests compare with, and the codes of an
8-bit checkpoint as integers.  tests/test_operator_reference.py pins them by loops and differences."""
import numpy as np

GROUP = 32


def layernorm(x, gain=None, offset=None, eps=1e-5, add=None):
    """y, mean, rstd of [rows][c]."""
    mean = x.mean(1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if gain is not None:
        y = y * gain
    if offset is not None:
        y = y + offset
    return (y if add is None else add + y), mean, rstd


def layernorm_bwd(x, mean, rstd, gain, dy, add=None):
    """dx, d_gain, d_offset; the statistics are taken as given."""
    z = (x - mean[:, None]) * rstd[:, None]
    u = dy if gain is None else dy * gain
    dx = rstd[:, None] * (u - u.mean(1, keepdims=True) - z * (u * z).mean(1, keepdims=True))
    return (dx if add is None else add + dx), (dy * z).sum(0), dy.sum(0)


def ckpt(x):
    """Codes [rows][c], scale bytes [rows][groups] and restored values of float64 x (values of fp32 or bf16)."""
    rows, c = x.shape
    g = -(-c // GROUP)
    codes, scales, back = np.zeros((rows, c), np.int64), np.zeros((rows, g), np.int64), np.zeros((rows, c))
    for j in range(g):
        v = x[:, j * GROUP:(j + 1) * GROUP]
        fine = np.isfinite(v).all(1)
        top = np.where(fine, np.abs(np.where(np.isfinite(v), v, 0.0)).max(1), 1.0)
        m, e = np.frexp(top)                                   # top = m 2^e, 0.5 <= m < 1 (e = 0 where top is 0)
        e = np.where(top == 0, -200, np.where(m * 128 <= 127, e - 7, e - 6))
        e = np.clip(e, -126, 121)
        q = np.where(fine[:, None], np.clip(np.rint(np.where(np.isfinite(v), v, 0.0) / np.exp2(e.astype(np.float64))[:, None]), -127, 127), 0.0)
        codes[:, j * GROUP:(j + 1) * GROUP] = q
        scales[:, j] = np.where(fine, e + 127, 255)
        back[:, j * GROUP:(j + 1) * GROUP] = np.where(fine[:, None], q * np.exp2(e.astype(np.float64))[:, None], np.nan)
    return codes, scales, back


def buckets(pos_q, pos_k, edges, seg_q=None, seg_k=None):
    d = pos_q.astype(np.int64)[:, None] - pos_k.astype(np.int64)[None, :]
    b = np.searchsorted(np.asarray(edges, np.int64), d, side="right")
    if seg_q is not None:
        b = np.where(seg_q[:, None] != seg_k[None, :], len(edges) + 1, b)
    return b


def relpos(b, table, add=None, layout="pair"):
    out = table[b] if layout == "pair" else np.moveaxis(table[b], 2, 0)
    return out if add is None else add + out


def relpos_bwd(b, d_out, n_buckets, layout="pair"):
    g = d_out if layout == "pair" else np.moveaxis(d_out, 0, 2)
    c = g.shape[2]
    d = np.zeros((n_buckets, c))
    for ch in range(c):
        d[:, ch] = np.bincount(b.reshape(-1), weights=g[:, :, ch].reshape(-1), minlength=n_buckets)
    return d
