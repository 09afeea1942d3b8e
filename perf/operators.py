"""The operators around the trunk and the calls they are measured with: layer norm (forward, backward, with the gradient
of its weights), the relative position embedding by buckets (with the gradient of its table) and activation checkpoints
in 8 bits (packed and restored; read by layer norm's backward pass).

A case names the operator (`op`), its sizes and its call:

  layernorm  call "fwd": y = add + LN(x), as a recycled representation joins the trunk's input;
             call "train": forward with saved statistics, then backward.  ckpt: the forward pass keeps x in 8 bits
             only, and the backward pass reads that
  relpos     call "fwd" or "train", layout "pair" (out[q][k][c] = add + table[bucket]) or "heads" (out[c][q][k], the bias of
             an attention with c heads).  edges "clip": buckets of one distance each up to +-32, all farther ones in the
             outermost two; "log": 32 buckets that widen with the distance.  chains > 1: several chains, and a bucket of its own
             for pairs of different chains
  ckpt       x packed into 8 bits and restored

Sizes come from pe_inputs.CONFIGS (c 16..256, s 8..5120, r 16..384) and, for wide rows and attention biases, are generic.
"""
import math

import torch

import paper_2211_00235_amd as pe

own = False

_EPS = 1e-5
_MOST = 130_000_000      # elements of a drawn case; ckpt_extra_msa_finetune has 126 million


def _ln(name, call, rows, c, dtype="bf16", ckpt=False):
    d = dict(op="layernorm", call=call, rows=rows, c=c, dtype=dtype, ckpt=ckpt)
    return dict(d, name=name) if name else d


def _rp(name, call, layout, n_q, n_k, c, edges, chains, dtype="bf16"):
    d = dict(op="relpos", call=call, layout=layout, n_q=n_q, n_k=n_k, c=c, edges=edges, chains=chains, dtype=dtype)
    return dict(d, name=name) if name else d


def _ck(name, rows, c, dtype="bf16"):
    d = dict(op="ckpt", call="both", rows=rows, c=c, dtype=dtype)
    return dict(d, name=name) if name else d


def listed():
    return [
        # first MSA row of a recycled step at the initial training size: the smallest call, latency
        _ln("ln_recycle_row", "fwd", 256, 256),
        # the pair representation of initial training, normalised in a training step
        _ln("ln_pair_train", "train", 256 * 256, 128),
        # a ragged MSA in full precision
        _ln("ln_msa_ragged_fp32", "train", 121 * 237, 256, "fp32"),
        # the MSA representation of fine-tuning, kept in 8 bits between the passes
        _ln("ln_msa_finetune_ckpt", "train", 512 * 384, 256, ckpt=True),
        # wide rows, as a sequence model's residual stream has them
        _ln("ln_wide_train", "train", 4096, 8192),
        # relative positions in the pair representation: initial training, and two chains at the fine-tuning crop
        _rp("relpos_pair_train", "train", "pair", 256, 256, 128, "clip", 1),
        _rp("relpos_pair_chains", "train", "pair", 384, 384, 128, "clip", 2),
        # one new position against a long sequence, eight heads
        _rp("relpos_heads_one", "fwd", "heads", 1, 8191, 8, "log", 1, "fp32"),
        # the bias of a self-attention over 2048 positions
        _rp("relpos_heads_train", "train", "heads", 2048, 2048, 16, "log", 1),
        # block inputs kept in 8 bits: the smallest configured pair representation, the pair representation of initial
        # training, and the extra MSA of fine-tuning
        _ck("ckpt_tiny_fp32", 48 * 48, 16, "fp32"),
        _ck("ckpt_pair", 256 * 256, 128),
        _ck("ckpt_extra_msa_finetune", 5120 * 384, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["layernorm", "layernorm", "relpos", "relpos", "ckpt"])
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        if op == "layernorm":
            call = rng.choice(["fwd", "train", "train"])
            c = rng.choice([64, 128, 256, _log_int(rng, 8, 8192), 8 * _log_int(rng, 1, 1024)])
            k = _ln(None, call, _log_int(rng, 1, 200_000), c, dtype, call == "train" and rng.random() < 0.4)
        elif op == "relpos":
            layout = rng.choice(["pair", "heads"])
            q = rng.choice([1, _log_int(rng, 2, 400 if layout == "pair" else 2048)])
            n = q if q > 1 and rng.random() < 0.6 else _log_int(rng, 1, 400 if layout == "pair" else 8192)
            c = rng.choice([16, 64, 128, 256, _log_int(rng, 4, 256)]) if layout == "pair" else rng.choice([1, 4, 8, 16, _log_int(rng, 1, 32)])
            k = _rp(None, rng.choice(["fwd", "train", "train"]), layout, q, n, c, rng.choice(["clip", "log"]),
                    rng.choice([1, 1, 2, 3]), dtype)
        else:
            c = rng.choice([16, 64, 128, 256, _log_int(rng, 8, 2048)])
            k = _ck(None, _log_int(rng, 1, 2_000_000), c, dtype)
        n = _elements(k)
        if n <= (_MOST if op == "ckpt" else 68_000_000) // (2 if dtype == "fp32" else 1):
            return k


def _elements(c):
    return c["n_q"] * c["n_k"] * c["c"] if c["op"] == "relpos" else c["rows"] * c["c"]


def _edges(kind):
    """Smallest distance of each bucket but the first, ascending."""
    if kind == "clip":
        return list(range(-31, 33))
    up = list(range(1, 9)) + [math.ceil(8 * 16 ** (i / 8)) for i in range(1, 9)]     # exact to 8, then widening to 128
    return sorted([1 - u for u in up] + up)[1:]


def _positions(n, chains, gen):
    """Residue numbers with gaps where residues are missing, and the chain of each; chains are numbered from 1 each."""
    step = 1 + (torch.rand(n, generator=gen, device="cuda") < 0.03) * torch.randint(1, 12, (n,), generator=gen, device="cuda")
    seg = (torch.arange(n, device="cuda") * chains) // n
    pos = torch.cumsum(step, 0)
    return (pos - pos[(seg * n + chains - 1) // chains] + 1).to(torch.int32), seg.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    st = {"case": dict(case), "h": pe.Handle()}
    if case["op"] == "relpos":
        n_q, n_k, c = case["n_q"], case["n_k"], case["c"]
        st["pos_k"], seg = _positions(n_k, case["chains"], gen)
        st["pos_q"], seg_q = (st["pos_k"], seg) if n_q == n_k else _positions(max(n_q, n_k), case["chains"], gen)
        st["pos_q"], seg_q = st["pos_q"][-n_q:].contiguous(), seg_q[-n_q:].contiguous()
        st["seg_q"], st["seg_k"] = (seg_q, seg) if case["chains"] > 1 else (None, None)
        st["edges"] = torch.tensor(_edges(case["edges"]), dtype=torch.int32)
        st["table"] = 0.3 * normal(len(st["edges"]) + (2 if case["chains"] > 1 else 1), c)
        shape = (n_q, n_k, c) if case["layout"] == "pair" else (c, n_q, n_k)
        st["add"] = normal(*shape).to(dt) if case["layout"] == "pair" else None     # the embedding is added to the pair input
        st["out"] = torch.empty(shape, dtype=dt, device="cuda")
        if case["call"] == "train":
            st["d_out"] = normal(*shape).to(dt)
            st["d_table"] = torch.empty_like(st["table"])
        return st
    rows, c = case["rows"], case["c"]
    # a residual stream: channels of different size, a few of them large, and a common offset of a row
    size = torch.exp(0.5 * normal(c)) * torch.where(torch.rand(c, generator=gen, device="cuda") < 0.02, 8.0, 1.0)
    st["x"] = (normal(rows, c) * size + 0.5 * normal(rows, 1)).to(dt)
    st["y"] = torch.empty_like(st["x"])
    if case["op"] == "layernorm":
        st["gain"], st["offset"] = 1.0 + 0.1 * normal(c), 0.1 * normal(c)
        if case["call"] == "fwd":
            st["add"] = normal(rows, c).to(dt)
        else:
            st["dy"] = normal(rows, c).to(dt)
            st["dx"] = torch.empty_like(st["x"])
            st["stats"] = torch.empty(rows, 2, device="cuda")
            st["d_gain"], st["d_offset"] = torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
    return st


def _groups(x):
    """[rows][groups of 32 channels][32], zeros behind the last channel."""
    rows, c = x.shape
    g = -(-c // 32)
    if c != 32 * g:
        x = torch.cat([x, x.new_zeros(rows, 32 * g - c)], 1)
    return x.reshape(rows, g, 32)


def _plain_pack(x):
    g = _groups(x.float())
    m, e = torch.frexp(g.abs().amax(2))                     # largest magnitude = m 2^e, 0.5 <= m < 1
    e = torch.where(m <= 127.0 / 128.0, e - 7, e - 6).clamp(min=-126)
    codes = torch.round(torch.ldexp(g, -e[:, :, None])).to(torch.int8)
    return codes, e.to(torch.int16)


def _plain_unpack(packed, c):
    codes, e = packed
    v = torch.ldexp(codes.float(), e[:, :, None].to(torch.int32))
    return v.reshape(v.shape[0], -1)[:, :c]


def _plain_layernorm(st):
    case, x = st["case"], st["x"].float()
    mean = x.mean(1, keepdim=True)
    xc = x - mean
    rstd = torch.rsqrt((xc * xc).mean(1, keepdim=True) + _EPS)
    y = xc * rstd * st["gain"] + st["offset"]
    if case["call"] == "fwd":
        return [(st["add"].float() + y).to(st["x"].dtype)]
    xs = _plain_unpack(_plain_pack(st["x"]), case["c"]) if case["ckpt"] else x
    xh, dy = (xs - mean) * rstd, st["dy"].float()
    gy = dy * st["gain"]
    dx = rstd * (gy - gy.mean(1, keepdim=True) - xh * (gy * xh).mean(1, keepdim=True))
    return [y.to(st["x"].dtype), torch.cat([mean, rstd], 1), dx.to(st["x"].dtype), (dy * xh).sum(0), dy.sum(0)]


def _plain_relpos(st):
    case = st["case"]
    d = st["pos_q"][:, None].long() - st["pos_k"][None, :].long()
    b = torch.bucketize(d, st["edges"].to(d.device).long(), right=True)
    if st["seg_q"] is not None:
        b = torch.where(st["seg_q"][:, None] == st["seg_k"][None, :], b, len(st["edges"]) + 1)
    if case["layout"] == "pair":
        out = st["table"][b] + st["add"].float()
    else:
        out = st["table"].t().contiguous()[:, b]
    out = out.to(st["out"].dtype)
    if case["call"] == "fwd":
        return [out]
    one = (torch.arange(len(st["table"]), device=d.device)[:, None] == b.reshape(1, -1)).float()
    if case["layout"] == "pair":
        return [out, torch.matmul(one, st["d_out"].float().reshape(-1, case["c"]))]
    return [out, torch.matmul(one, st["d_out"].float().reshape(case["c"], -1).t().contiguous())]


def _workspace(st, n):
    """Scratch that a program allocates once for the sizes it has."""
    if "ws" not in st:
        st["ws"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return st["ws"]


def _own_layernorm(st):
    h, case = st["h"], st["case"]
    if case["call"] == "fwd":
        pe.layernorm_fwd(h, st["x"], st["gain"], st["offset"], st["y"], eps=_EPS, add=st["add"])
        return [st["y"]]
    if case["ckpt"] and "ckpt" not in st:
        st["ckpt"] = torch.empty(pe.ckpt_bytes(case["rows"], case["c"]), dtype=torch.uint8, device="cuda")
    kept = st["ckpt"] if case["ckpt"] else None
    pe.layernorm_fwd(h, st["x"], st["gain"], st["offset"], st["y"], eps=_EPS, stats=st["stats"], ckpt=kept)
    ws = _workspace(st, 0 if "ws" in st else pe.layernorm_workspace_bytes(case["rows"], case["c"]))
    pe.layernorm_bwd(h, st["dy"], kept if case["ckpt"] else st["x"], st["stats"], st["gain"], st["dx"], st["d_gain"],
                     st["d_offset"], ws)
    return [st["y"], st["stats"], st["dx"], st["d_gain"], st["d_offset"]]


def _own_relpos(st):
    h, case = st["h"], st["case"]
    pe.relpos_fwd(h, st["pos_q"], st["pos_k"], st["edges"], st["table"], st["out"], seg_q=st["seg_q"], seg_k=st["seg_k"],
                  add=st["add"], layout=case["layout"])
    if case["call"] == "fwd":
        return [st["out"]]
    ws = _workspace(st, 0 if "ws" in st else pe.relpos_workspace_bytes(case["n_q"], case["n_k"], case["c"],
                                                                       st["table"].shape[0], case["layout"]))
    pe.relpos_bwd(h, st["pos_q"], st["pos_k"], st["edges"], st["d_out"], st["d_table"], ws, seg_q=st["seg_q"],
                  seg_k=st["seg_k"], layout=case["layout"])
    return [st["out"], st["d_table"]]


def _own_ckpt(st):
    case = st["case"]
    if "ckpt" not in st:
        st["ckpt"] = torch.empty(pe.ckpt_bytes(case["rows"], case["c"]), dtype=torch.uint8, device="cuda")
    pe.ckpt_pack(st["h"], st["x"], st["ckpt"])
    pe.ckpt_unpack(st["h"], st["ckpt"], st["y"])
    return [st["y"]]


def run(st):
    op = st["case"]["op"]
    if own:
        return {"layernorm": _own_layernorm, "relpos": _own_relpos, "ckpt": _own_ckpt}[op](st)
    if op == "ckpt":
        return [_plain_unpack(_plain_pack(st["x"]), st["case"]["c"]).to(st["x"].dtype)]
    return _plain_layernorm(st) if op == "layernorm" else _plain_relpos(st)


def work(case):
    """Each input read once, each output written once; what the passes hand on between them (statistics, 8-bit copies) counts on
    both sides, and a checkpoint's round trip counts its codes and scales written and read."""
    e, n = (4 if case["dtype"] == "fp32" else 2), _elements(case)
    if case["op"] == "relpos":
        buckets = len(_edges(case["edges"])) + (2 if case["chains"] > 1 else 1)
        small = 4 * buckets * case["c"] + 4 * (case["n_q"] + case["n_k"]) * (2 if case["chains"] > 1 else 1)
        b, f = n * e * (2 if case["layout"] == "pair" else 1) + small, n
        return {"bytes": b + n * e + 2 * small, "flops": 2 * f} if case["call"] == "train" else {"bytes": b, "flops": f}
    packed = n + case["rows"] * -(-case["c"] // 32)
    if case["op"] == "ckpt":
        return {"bytes": 2 * n * e + 2 * packed, "flops": 4 * n}
    if case["call"] == "fwd":
        return {"bytes": 3 * n * e + 8 * case["c"], "flops": 9 * n}
    kept = 2 * packed if case["ckpt"] else n * e
    return {"bytes": 4 * n * e + kept + 16 * case["rows"] + 20 * case["c"], "flops": 24 * n}


def _exact_kept(x):
    """The 8-bit form's values in 64 bits, group by group of 32 channels: rint(x / 2^e) 2^e with the smallest e >= -126 that keeps
    the codes within 127."""
    out = torch.empty_like(x)
    for a in range(0, x.shape[1], 32):
        g = x[:, a:a + 32]
        top = g.abs().max(1, keepdim=True).values
        e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / 127.0)).clamp(min=-126.0)
        e = torch.where(top > 127.0 * torch.exp2(e), e + 1, e)          # the logarithm's own rounding
        e = torch.where((top <= 127.0 * torch.exp2(e - 1)) & (e > -126), e - 1, e)
        out[:, a:a + 32] = torch.round(g / torch.exp2(e)) * torch.exp2(e)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "ckpt":
        return [_exact_kept(st["x"].double())]
    if case["op"] == "layernorm":
        x, g, b = st["x"].double().requires_grad_(), st["gain"].double().requires_grad_(), st["offset"].double().requires_grad_()
        n = x.shape[1]
        mu = x.sum(1, keepdim=True) / n
        sd = (((x - mu) ** 2).sum(1, keepdim=True) / n + _EPS).sqrt()
        y = (x - mu) / sd * g + b
        if case["call"] == "fwd":
            return [(y + st["add"].double()).detach()]
        dy, stats = st["dy"].double(), torch.cat([mu, 1 / sd], 1).detach()
        if not case["ckpt"]:
            return [y.detach(), stats, *torch.autograd.grad(y, (x, g, b), dy)]
        with torch.no_grad():       # the derivative's formula at the kept values, with the statistics of the exact ones
            z, u = (_exact_kept(x) - mu) / sd, dy * g
            dx = (u - u.sum(1, keepdim=True) / n - z * ((u * z).sum(1, keepdim=True) / n)) / sd
            return [y.detach(), stats, dx, torch.einsum("rc,rc->c", dy, z), dy.sum(0)]
    b = sum((st["pos_q"][:, None].long() - st["pos_k"][None, :].long() >= e).long() for e in _edges(case["edges"]))
    if case["chains"] > 1:
        b[st["seg_q"][:, None] != st["seg_k"][None, :]] = len(_edges(case["edges"])) + 1
    t = st["table"].double()
    pair = case["layout"] == "pair"
    out = torch.index_select(t, 0, b.reshape(-1)).reshape(*b.shape, -1)
    out = out + st["add"].double() if pair else out.permute(2, 0, 1)
    if case["call"] == "fwd":
        return [out]
    g = (st["d_out"] if pair else st["d_out"].permute(1, 2, 0)).double().reshape(-1, case["c"])
    d = torch.stack([g[(b == k).reshape(-1)].sum(0) for k in range(t.shape[0])])
    return [out, d]
