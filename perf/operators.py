"""What the layer operators are timed on: the passes that a training or serving step of n workers makes through them.

The framework holds one fp32 model row per worker.  Its layer operators run one layer of all n models at once: every
activation is [n][T][D] (worker, token, feature), a weight is a view of the model rows, a weight gradient an fp32 view
of rows beside them.  Activations that the backward pass needs are held in 8 bits: blocks of 32 features share a scale
that is a power of two, value = code * 2^(c - 133) with c the block's scale byte.

A case: kind, n workers, T tokens each, D features (of the gated activation: its width; of the weight gradient: the
layer's inputs), type of the activations ("bf16", "fp16", "fp32"), and
  norm       residual (x + r is normalised and returned), ckpt (the normalised rows in 8 bits too, recalled as bf16)
  norm_bwd   source of the normalised rows: "ckpt" (8 bits) or "full" (the sum itself); dtotal (the gradient that
             reaches the sum past the norm); lengths (each worker has its own number of tokens, the rest is padding)
  ckpt       8 bits and back
  gated      the gated activation alone
  gated_step the gated activation with its inputs kept in 8 bits, then its backward pass from them, which returns
             the activation again, in 8 bits (recalled as bf16), for the next layer's weight gradient
  wgrad      O outputs; scale (a factor per input feature, the norm's weight); lengths
offset is the first column of the views of the model rows: odd ones leave them unaligned.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS = 1e-5
BLOCK, PITCH = 32, 128


def _case(name, kind, n, T, D, type, offset=0, residual=False, ckpt=False, source="ckpt", dtotal=False, lengths=False,
          O=0, scale=False):
    c = dict(kind=kind, n=n, T=T, D=D, type=type)
    if kind == "norm":
        c.update(residual=residual, ckpt=ckpt, offset=offset)
    elif kind == "norm_bwd":
        c.update(source=source, dtotal=dtotal, lengths=lengths, offset=offset)
    elif kind == "wgrad":
        c.update(O=O, scale=scale, lengths=lengths, offset=offset)
    return dict(c, name=name) if name else c


def listed():
    return [
        # eight workers answer, one token each: latency is all there is
        _case("norm_token", "norm", 8, 1, 512, "bf16", residual=True),
        # the forward pass of a training step of four workers, its rows kept for the backward pass
        _case("norm_ckpt_large", "norm", 4, 4096, 4096, "bf16", residual=True, ckpt=True),
        # a width and a prompt length that nothing divides, in half precision, on unaligned rows
        _case("norm_ragged_fp16", "norm", 3, 1021, 1537, "fp16", residual=True, ckpt=True, offset=5),
        # the backward pass of the large step: the rows come from 8 bits, the residual's gradient joins
        _case("norm_bwd_ckpt_large", "norm_bwd", 4, 4096, 4096, "bf16", dtotal=True),
        # fp32 training of small models whose workers hold batches of unequal lengths
        _case("norm_bwd_full_fp32", "norm_bwd", 3, 777, 1000, "fp32", source="full", lengths=True, offset=5),
        # any activation put away and recalled: the large step's, and a small fp32 one of odd width
        _case("ckpt_large", "ckpt", 4, 4096, 8192, "bf16"),
        _case("ckpt_odd_fp32", "ckpt", 16, 33, 515, "fp32"),
        # one token of eight workers through the gated activation
        _case("gated_token", "gated", 8, 1, 2048, "bf16"),
        # forward and backward of the gated activation in the large training step
        _case("gated_step_large", "gated_step", 4, 4096, 8192, "bf16"),
        # the weight gradients of eight small models on short sequences
        _case("wgrad_small", "wgrad", 8, 64, 512, "bf16", O=512),
        # sizes that no tile divides, half precision, unequal lengths, the norm's weight folded in
        _case("wgrad_ragged_fp16", "wgrad", 3, 1000, 1537, "fp16", O=1111, lengths=True, scale=True, offset=5),
        # the largest: the projection out of the norm in a large step of two workers
        _case("wgrad_large", "wgrad", 2, 8192, 4096, "bf16", O=8192, scale=True),
    ]


def draw(rng):
    def logint(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))

    def width(lo, hi):
        d = logint(lo, hi)
        if rng.random() < 0.5:
            d = max(lo, d // 64 * 64)
        return d + 8 if d == 3 * 1024 else d

    kind = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "ckpt", "gated", "gated_step", "wgrad", "wgrad"])
    n = rng.choice([1, 2, 3, 4, 8, 16])
    type = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    offset = rng.choice([0, 0, 5])
    D = width(64, 8192)
    flag = [rng.random() < 0.5 for _ in range(4)]
    if kind == "wgrad":
        O = width(64, 8192)
        most = 2 * 8192 * 4096 * 8192 // (n * O * D)
        return _case(None, kind, n, logint(1, max(1, min(8192, most))), D, type, offset, O=O, scale=flag[0],
                     lengths=flag[1])
    most = 4 * 4096 * (8192 if kind in ("ckpt", "gated", "gated_step") else 4096) // (n * D)
    T = logint(1, max(1, min(16384, most)))
    return _case(None, kind, n, T, D, type, offset, residual=flag[0], ckpt=flag[1], dtotal=flag[2], lengths=flag[3],
                 source=rng.choice(["ckpt", "ckpt", "full"]))


# ------------------------------------------------------------------ inputs


def _lengths(case):
    """The workers' numbers of tokens: the first has all T, the others fewer and fewer, none where T < n."""
    n, T = case["n"], case["T"]
    return [T * (n - i) // n if i else T for i in range(n)]


def _activations(g, n, T, D, type):
    """A residual stream: normal values, with one feature in 64 that is 16 times as large in every row."""
    loud = torch.where(torch.rand(D, generator=g, device=DEV) < 1 / 64, 16.0, 1.0)
    return (torch.randn(n, T, D, generator=g, device=DEV) * loud).to(type)


def _gradients(g, n, T, D, type):
    """Gradients: small, of a size that varies from token to token; one token in 16 has none (not part of the loss)."""
    size = torch.exp(torch.randn(n, T, 1, generator=g, device=DEV)) * 1e-2
    size = size * (torch.rand(n, T, 1, generator=g, device=DEV) >= 1 / 16)
    return (torch.randn(n, T, D, generator=g, device=DEV) * size).to(type)


def _model_view(g, n, D, offset):
    """A norm's weight where it lies in the workers' fp32 model rows."""
    rows = 1 + 0.2 * torch.randn(n, (offset + D + 31) // 32 * 32, generator=g, device=DEV)
    return rows[:, offset:offset + D]


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    kind, n, T, D, type = case["kind"], case["n"], case["T"], case["D"], TYPES[case["type"]]
    s = {"case": dict(case)}
    if kind == "norm":
        s["x"] = _activations(g, n, T, D, type)
        s["residual"] = _activations(g, n, T, D, type) if case["residual"] else None
        s["weight"] = _model_view(g, n, D, case["offset"])
    elif kind == "norm_bwd":
        h = _activations(g, n, T, D, type)
        s["rstd"] = torch.rsqrt(h.float().square().mean(-1) + EPS)
        if case["source"] == "ckpt":
            s["codes"], s["scales"] = _pack(h.float() * s["rstd"][..., None])
        else:
            s["total"] = h
        del h
        s["dy"] = _gradients(g, n, T, D, type)
        s["dtotal"] = _gradients(g, n, T, D, type) if case["dtotal"] else None
        s["weight"] = _model_view(g, n, D, case["offset"])
    elif kind == "ckpt":
        s["x"] = _activations(g, n, T, D, type)
    elif kind in ("gated", "gated_step"):
        both = _activations(g, n, T, 2 * D, type)  # one projection gives both halves
        s["gate"], s["up"] = both[..., :D], both[..., D:]
        if kind == "gated_step":
            s["dout"] = _gradients(g, n, T, D, type)
    else:
        s["codes"], s["scales"] = _pack(_activations(g, n, T, D, type).float())
        s["dy"] = _gradients(g, n, T, case["O"], type)
        s["scale"] = _model_view(g, n, D, case["offset"]) if case["scale"] else None
    if kind in ("norm_bwd", "wgrad"):
        s["lengths"] = None
        if case["lengths"]:
            at = torch.randperm(n, generator=g, device=DEV)
            s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)[at].contiguous()
    return s


# ------------------------------------------------------------------ the plain form


def _blocks(x):
    """x (fp32) in blocks of 32 features, the last one filled up with zeros."""
    short = -x.shape[-1] % BLOCK
    if short:
        x = torch.nn.functional.pad(x, (0, short))
    return x.unflatten(-1, (-1, BLOCK))


def _scale_bytes(b):
    """The scale bytes of blocks b: the least power of two that leaves the largest code at 127 or less."""
    most = b.abs().amax(-1).view(torch.int32)
    return torch.clamp((most + 0x10000) >> 23, 7, 255)


def _codes_of(b, c):
    """Codes (whole fp32 numbers) of blocks b with scale bytes c."""
    return torch.round(b * ((260 - c) << 23).view(torch.float32)[..., None])


def _recalled(codes, c):
    """The values of codes (fp32) with scale bytes c (int32)."""
    unit = ((c - 6) << 23).view(torch.float32)
    return codes * torch.where(c == 255, float("nan"), unit)[..., None]


def _values(x):
    """What x (fp32) is in 8 bits, as fp32."""
    b = _blocks(x)
    c = _scale_bytes(b)
    return _recalled(_codes_of(b, c), c).flatten(-2)[..., :x.shape[-1]]


def _pack(x):
    """(codes int8, scales uint8) of x (fp32), in the rows' pitch."""
    b = _blocks(x)
    c = _scale_bytes(b)
    q = _codes_of(b, c).to(torch.int8).flatten(-2)
    pitch = -(-x.shape[-1] // PITCH) * PITCH
    codes = torch.zeros(*x.shape[:-1], pitch, dtype=torch.int8, device=DEV)
    codes[..., :q.shape[-1]] = q
    scales = torch.full((*x.shape[:-1], pitch // BLOCK), 7, dtype=torch.uint8, device=DEV)
    scales[..., :c.shape[-1]] = c.to(torch.uint8)
    return codes, scales


def _unpack(codes, scales, D):
    """The values of a checkpoint's rows, as fp32."""
    return _recalled(codes.float().unflatten(-1, (-1, BLOCK)), scales.int()).flatten(-2)[..., :D]


def _used(lengths, T):
    """[n][T][1]: whether a token is one of its worker's."""
    return (torch.arange(T, device=DEV)[None, :] < lengths[:, None])[..., None]


def _plain(s):
    case = s["case"]
    kind, T, D, type = case["kind"], case["T"], case["D"], TYPES[case["type"]]
    if kind == "norm":
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        rstd = 1 / torch.sqrt((h * h).mean(-1) + EPS)
        xhat = h * rstd[..., None]
        out = {"y": (xhat * s["weight"][:, None, :]).to(type), "rstd": rstd}
        if s["residual"] is not None:
            out["total"] = h.to(type)
        if case["ckpt"]:
            out["recalled"] = _values(xhat).to(torch.bfloat16)
        return out
    if kind == "norm_bwd":
        dy, rstd = s["dy"].float(), s["rstd"][..., None]
        xhat = _unpack(s["codes"], s["scales"], D) if case["source"] == "ckpt" else s["total"].float() * rstd
        u = dy * s["weight"][:, None, :]
        dx = rstd * (u - xhat * (u * xhat).mean(-1, keepdim=True))
        if s["dtotal"] is not None:
            dx = dx + s["dtotal"].float()
        dw = dy * xhat
        if s["lengths"] is not None:
            used = _used(s["lengths"], T)
            dx, dw = torch.where(used, dx, 0.0), torch.where(used, dw, 0.0)
        return {"dx": dx.to(type), "dweight": dw.sum(1)}
    if kind == "ckpt":
        return {"recalled": _values(s["x"].float()).to(type)}
    if kind in ("gated", "gated_step"):
        g, u = s["gate"].float(), s["up"].float()
        out = {"out": (g / (1 + torch.exp(-g)) * u).to(type)}
        if kind == "gated_step":
            g, u, d = _values(g), _values(u), s["dout"].float()
            p = 1 / (1 + torch.exp(-g))
            out["dup"] = (d * g * p).to(type)
            out["dgate"] = (d * u * p * (1 + g * (1 - p))).to(type)
            out["recalled"] = _values(g * p * u).to(torch.bfloat16)
        return out
    dy, xhat = s["dy"].float(), _unpack(s["codes"], s["scales"], D)
    if s["lengths"] is not None:
        used = _used(s["lengths"], T)
        dy, xhat = torch.where(used, dy, 0.0), torch.where(used, xhat, 0.0)
    dw = torch.matmul(dy.transpose(1, 2), xhat)
    if s["scale"] is not None:
        dw = dw * s["scale"][:, None, :]
    return {"dweight": dw}


# ------------------------------------------------------------------ the framework's operators


def _buffers(s):
    """The outputs and workspaces that a program keeps from step to step."""
    import paper_2110_04175_gb300 as rs

    case = s["case"]
    kind, n, T, D, type = case["kind"], case["n"], case["T"], case["D"], TYPES[case["type"]]

    def rows(width=D, t=type):
        return torch.empty(n, T, width, dtype=t, device=DEV)

    def model_rows(count):
        off = case["offset"]
        return torch.empty(n, (off + count + 31) // 32 * 32, device=DEV)[:, off:off + count]

    b = {"rs": rs}
    if kind == "norm":
        b.update(y=rows(), rstd=torch.empty(n, T, device=DEV), total=rows() if case["residual"] else None)
        if case["ckpt"]:
            b.update(kept=rs.ActivationCheckpoint(n, T, D, device=DEV), recalled=rows(t=torch.bfloat16))
    elif kind == "norm_bwd":
        b.update(dx=rows(), dweight=model_rows(D),
                 work=torch.empty(rs.relay_rms_norm_backward_workspace(n, T, D), dtype=torch.uint8, device=DEV))
    elif kind == "ckpt":
        b.update(kept=rs.ActivationCheckpoint(n, T, D, device=DEV), recalled=rows())
    elif kind in ("gated", "gated_step"):
        b.update(out=rows())
        if kind == "gated_step":
            both = rows(2 * D)
            b.update(dgate=both[..., :D], dup=both[..., D:], recalled=rows(t=torch.bfloat16))
            b.update({k: rs.ActivationCheckpoint(n, T, D, device=DEV) for k in ("gate", "up", "act")})
    else:
        O = case["O"]
        b.update(dweight=model_rows(O * D).unflatten(1, (O, D)),
                 work=torch.empty(rs.relay_weight_grad_workspace(n, T, O, D), dtype=torch.uint8, device=DEV))
    return b


def _kernels(s):
    if "buffers" not in s:
        s["buffers"] = _buffers(s)
    b, case = s["buffers"], s["case"]
    rs, kind = b["rs"], case["kind"]
    if kind == "norm":
        out = {"y": b["y"], "rstd": b["rstd"]}
        kept = b["kept"] if case["ckpt"] else None
        rs.relay_rms_norm(s["x"], s["weight"], b["y"], EPS, residual=s["residual"], total=b["total"], rstd=b["rstd"],
                          checkpoint=kept)
        if b["total"] is not None:
            out["total"] = b["total"]
        if kept is not None:
            rs.relay_checkpoint_unpack(kept, b["recalled"])
            out["recalled"] = b["recalled"]
        return out
    if kind == "norm_bwd":
        source = ({"checkpoint": (s["codes"], s["scales"])} if case["source"] == "ckpt" else {"total": s["total"]})
        rs.relay_rms_norm_backward(s["dy"], s["weight"], s["rstd"], b["dx"], b["dweight"], b["work"],
                                   dtotal=s["dtotal"], lengths=s["lengths"], **source)
        return {"dx": b["dx"], "dweight": b["dweight"]}
    if kind == "ckpt":
        rs.relay_checkpoint_pack(s["x"], b["kept"])
        rs.relay_checkpoint_unpack(b["kept"], b["recalled"])
        return {"recalled": b["recalled"]}
    if kind == "gated":
        rs.relay_gated(s["gate"], s["up"], b["out"])
        return {"out": b["out"]}
    if kind == "gated_step":
        rs.relay_gated(s["gate"], s["up"], b["out"], gate_checkpoint=b["gate"], up_checkpoint=b["up"])
        rs.relay_gated_backward(s["dout"], b["dgate"], b["dup"], gate_checkpoint=b["gate"], up_checkpoint=b["up"],
                                out_checkpoint=b["act"])
        rs.relay_checkpoint_unpack(b["act"], b["recalled"])
        return {k: b[k] for k in ("out", "dgate", "dup", "recalled")}
    rs.relay_weight_grad(s["dy"], (s["codes"], s["scales"]), b["dweight"], b["work"], column_scale=s["scale"],
                         lengths=s["lengths"])
    return {"dweight": b["dweight"]}


def run(state):
    return _kernels(state) if own else _plain(state)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    """Inputs read once and outputs written once; what is put away in 8 bits and recalled within a pass is neither."""
    kind, n, T, D, e = case["kind"], case["n"], case["T"], case["D"], SIZE[case["type"]]
    cells, eight = n * T * D, 1 + 1 / BLOCK
    used = sum(_lengths(case)) if case.get("lengths") else n * T
    if kind == "norm":
        b = cells * e * (4 if case["residual"] else 2) + cells * 2 * case["ckpt"] + 4 * n * (D + T)
        return {"bytes": b, "flops": 6 * cells}
    if kind == "norm_bwd":
        read = used * D * (e + (eight if case["source"] == "ckpt" else e) + e * case["dtotal"])
        return {"bytes": read + cells * e + 8 * n * D + 4 * used, "flops": 9 * used * D}
    if kind == "ckpt":
        return {"bytes": 2 * e * cells, "flops": 3 * cells}
    if kind == "gated":
        return {"bytes": 3 * e * cells, "flops": 6 * cells}
    if kind == "gated_step":
        return {"bytes": (6 * e + 2) * cells, "flops": 24 * cells}
    b = used * (case["O"] * e + D * eight) + 4 * n * D * (case["O"] + case["scale"])
    return {"bytes": b, "flops": 2 * used * case["O"] * D}


# ------------------------------------------------------------------ the definitions in 64 bits


def _two_to(e):
    """2^e for whole e, exactly (pow may be an ulp off, which would break ties)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _held(codes, scales, D):
    """A checkpoint's values: code * 2^(c - 133)."""
    c = scales.long().repeat_interleave(BLOCK, -1)[..., :D]
    v = codes[..., :D].double() * _two_to(c - 133)
    return torch.where(c == 255, math.nan, v)


def _nearest(x):
    """The values that x (64 bits) gets in 8 bits: whole multiples of the block's unit, the least power of two whose
    127 multiples reach the block's largest magnitude once that is rounded."""
    D = x.shape[-1]
    wide = -(-D // BLOCK) * BLOCK
    padded = torch.zeros(*x.shape[:-1], wide, dtype=torch.float64, device=x.device)
    padded[..., :D] = x
    most = padded.reshape(*x.shape[:-1], -1, BLOCK).abs().max(-1).values
    tiny = 2.0 ** -126
    m, e = torch.frexp(torch.clamp(most, min=tiny))  # most = m 2^e, 1/2 <= m < 1
    unit = _two_to(torch.clamp(e - 7 + (m * 128 >= 127.5).int(), min=-126))
    unit = unit.repeat_interleave(BLOCK, -1)[..., :D]
    return torch.round(x / unit) * unit


def exact(case, seed):
    s = prepare(case, seed)
    kind, n, T, D = case["kind"], case["n"], case["T"], case["D"]
    if kind == "norm":
        h = s["x"].double() + (0 if s["residual"] is None else s["residual"].double())
        root = torch.sqrt(torch.linalg.vector_norm(h, dim=-1) ** 2 / D + EPS)
        xhat = h / root[..., None]
        out = {"y": torch.einsum("ntd,nd->ntd", xhat, s["weight"].double()), "rstd": 1 / root}
        if s["residual"] is not None:
            out["total"] = h
        if case["ckpt"]:
            out["recalled"] = xhat  # the numbers that the 8 bits stand in for: both sides differ by the format's step
        return out
    if kind == "norm_bwd":
        r, w, dy = s["rstd"].double()[..., None], s["weight"].double()[:, None], s["dy"].double()
        xhat = _held(s["codes"], s["scales"], D) if case["source"] == "ckpt" else s["total"].double() * r
        along = torch.einsum("ntd,ntd->nt", dy * w, xhat)[..., None] / D
        dx = (dy * w - xhat * along) * r
        dx = dx if s["dtotal"] is None else dx + s["dtotal"].double()
        if s["lengths"] is not None:
            for i, m in enumerate(s["lengths"].tolist()):
                dx[i, m:], dy[i, m:] = 0, 0
        return {"dx": dx, "dweight": torch.einsum("ntd,ntd->nd", dy, xhat)}
    if kind == "ckpt":
        return {"recalled": _nearest(s["x"].double())}
    if kind in ("gated", "gated_step"):
        g, u = s["gate"].double(), s["up"].double()
        out = {"out": g * torch.sigmoid(g) * u}
        if kind == "gated_step":
            g, u, d = _nearest(g), _nearest(u), s["dout"].double()
            p, q = torch.sigmoid(g), torch.sigmoid(-g)
            out["dup"] = d * (g * p)
            out["dgate"] = d * u * (p + g * p * q)
            out["recalled"] = g * p * u  # as in the norm
        return out
    xhat = _held(s["codes"], s["scales"], D)
    dw = torch.empty(n, case["O"], D, dtype=torch.float64, device=DEV)
    for i in range(n):
        m = T if s["lengths"] is None else int(s["lengths"][i])
        dw[i] = s["dy"][i, :m].double().T @ xhat[i, :m]
        if s["scale"] is not None:
            dw[i] *= s["scale"][i].double()
    return {"dweight": dw}
