"""What the operators of a recurrent block and of its matrices' update are timed on.

Beside the layer operators of a feed-forward layer, the framework mixes tokens by a gated linear recurrence, joins a
block's output to the residual stream between two norms, and makes the update of a weight matrix orthogonal.  Activations
are [n][T][D] (worker or sequence, token, feature); weights, states and updates are fp32, views of the workers' model
rows or rows of their own.

A case: kind, n, T tokens each, D features, type of the activations ("bf16", "fp16", "fp32"), and
  rec        h_t = f_t h_{t-1} + (1 - f_t) v_t, f = sigma(gate); state (an fp32 state comes in and goes out), packed (several
             sequences behind one another: a token that begins one takes nothing from before it), lengths (each worker has
             its own number of tokens, the rest is padding)
  rec_bwd    its gradients, from the rows h as the forward pass left them; the same options (state: the gradient of the
             last state comes in, that of the first one goes out)
  block      h = scale r + sigma(gate) norm(x) w_post, y = norm(h) w_pre; gate, scale (without: 1); ckpt (the normalised h
             in 8 bits too, recalled as bf16)
  block_bwd  its gradients; gate, scale, dtotal (the gradient that reaches h past the second norm), lengths
  ortho      n fp32 matrices [rows][cols] made orthogonal by five Newton-Schulz steps
offset is the first column of the views of the model rows: odd ones leave them unaligned.
"""
import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
EPS, ORTHO_EPS = 1e-5, 1e-7
BLOCK = 32
STEPS, A, B, C = 5, 3.4445, -4.7750, 2.0315


def _case(name, kind, n, T=0, D=0, type="fp32", offset=0, state=False, packed=False, lengths=False, gate=False, scale=False,
          ckpt=False, dtotal=False, rows=0, cols=0):
    if kind == "ortho":
        c = dict(kind=kind, n=n, rows=rows, cols=cols, offset=offset)
    else:
        c = dict(kind=kind, n=n, T=T, D=D, type=type)
        if kind in ("rec", "rec_bwd"):
            c.update(state=state, packed=packed, lengths=lengths)
        elif kind == "block":
            c.update(offset=offset, gate=gate, scale=scale, ckpt=ckpt)
        else:
            c.update(offset=offset, gate=gate, scale=scale, dtotal=dtotal, lengths=lengths)
    return dict(c, name=name) if name else c


def listed():
    return [
        # 64 sequences answer, one token each, their states kept from call to call
        _case("rec_token", "rec", 64, 1, 2048, "bf16", state=True),
        # the forward pass of a training step of four workers
        _case("rec_large", "rec", 4, 4096, 4096, "bf16"),
        # one worker's few channels over a very long stretch of packed texts, carried on from the stretch before
        _case("rec_long_fp32", "rec", 1, 50021, 257, "fp32", state=True, packed=True),
        # the backward pass of the large step
        _case("rec_bwd_large", "rec_bwd", 4, 4096, 4096, "bf16"),
        # a width and a length that nothing divides, in half precision, workers with batches of unequal lengths
        _case("rec_bwd_ragged_fp16", "rec_bwd", 3, 1021, 1537, "fp16", state=True, packed=True, lengths=True),
        # one token of eight workers between two blocks
        _case("block_token", "block", 8, 1, 512, "bf16", gate=True, scale=True),
        # between two blocks of the large step, the next block's input kept in 8 bits for the weight gradient
        _case("block_large", "block", 4, 4096, 4096, "bf16", gate=True, scale=True, ckpt=True),
        # the same on the way back
        _case("block_bwd_large", "block_bwd", 4, 4096, 4096, "bf16", gate=True, scale=True, dtotal=True),
        # fp32 training of small models without a gate, unequal lengths, weights that lie unaligned
        _case("block_bwd_ragged_fp32", "block_bwd", 3, 777, 1000, "fp32", offset=5, lengths=True, scale=True),
        # the matrices of eight small models
        _case("ortho_small", "ortho", 8, rows=128, cols=256),
        # more rows than columns, neither of them a multiple of anything, in unaligned rows
        _case("ortho_tall_odd", "ortho", 3, rows=1537, cols=1001, offset=5),
        # the largest: one projection of each of four models
        _case("ortho_large", "ortho", 4, rows=2048, cols=8192),
    ]


def draw(rng):
    def logint(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))

    def width(lo, hi):
        d = logint(lo, hi)
        return max(lo, d // 64 * 64) if rng.random() < 0.5 else d

    kind = rng.choice(["rec", "rec", "rec_bwd", "rec_bwd", "block", "block_bwd", "ortho", "ortho"])
    offset = rng.choice([0, 0, 5])
    if kind == "ortho":
        n, rows, cols = rng.choice([1, 2, 3, 4, 8, 16]), width(16, 8192), width(16, 8192)
        short, long = min(rows, cols), max(rows, cols)
        most = 4 * 2048 * 2048 * (2048 + 3 * 8192)
        while n > 1 and n * short * short * (short + 3 * long) > most:
            n -= 1
        if short * short * (short + 3 * long) > most:
            rows = cols = 2048 - rng.randrange(64)
        return _case(None, kind, n, rows=rows, cols=cols, offset=offset)
    type = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    flag = [rng.random() < 0.5 for _ in range(4)]
    most = 4 * 4096 * 4096 * 2 // SIZE[type]
    if kind in ("rec", "rec_bwd"):
        n, D = logint(1, 128), width(16, 8192)
        T = logint(1, max(1, min(65536, most // (n * D))))
        return _case(None, kind, n, T, D, type, state=flag[0], packed=flag[1], lengths=flag[2])
    n, D = rng.choice([1, 2, 3, 4, 8, 16]), width(64, 8192)
    T = logint(1, max(1, min(16384, most // (n * D))))
    return _case(None, kind, n, T, D, type, offset, gate=flag[0], scale=flag[1], ckpt=flag[2], dtotal=flag[2], lengths=flag[3])


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


def _gates(g, n, T, D, type):
    """Forget gates before the sigmoid: each channel with a memory of its own, from one token to some hundreds."""
    base = torch.rand(D, generator=g, device=DEV) * 6 - 1
    return (torch.randn(n, T, D, generator=g, device=DEV) + base).to(type)


def _model_view(g, n, D, offset, size=0.2):
    """A weight around 1 where it lies in the workers' fp32 model rows."""
    rows = 1 + size * torch.randn(n, (offset + D + 31) // 32 * 32, generator=g, device=DEV)
    return rows[:, offset:offset + D]


def _updates(g, case):
    """Momentum of weight matrices: some strong directions, the rest weaker and weaker, as gradients of few tokens leave it."""
    n, r, c, off = case["n"], case["rows"], case["cols"], case["offset"]
    k = max(1, min(r, c) // 4)
    strong = torch.randn(n, r, k, generator=g, device=DEV) * torch.exp(-3 * torch.arange(k, device=DEV) / k)
    full = torch.bmm(strong, torch.randn(n, k, c, generator=g, device=DEV)) / math.sqrt(k)
    full += 0.3 * torch.randn(n, r, c, generator=g, device=DEV)
    rows = torch.zeros(n, (off + r * c + 31) // 32 * 32, device=DEV)
    rows[:, off:off + r * c] = full.flatten(1) * 1e-3
    return rows[:, off:off + r * c].unflatten(1, (r, c))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = {"case": dict(case)}
    if case["kind"] == "ortho":
        s["update"] = _updates(g, case)
        return s
    kind, n, T, D, type = case["kind"], case["n"], case["T"], case["D"], TYPES[case["type"]]
    s["lengths"] = None
    if case.get("lengths"):
        at = torch.randperm(n, generator=g, device=DEV)
        s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)[at].contiguous()
    if kind in ("rec", "rec_bwd"):
        s["gate"], s["value"] = _gates(g, n, T, D, type), _activations(g, n, T, D, type)
        s["initial"] = torch.randn(n, D, generator=g, device=DEV) if case["state"] else None
        s["begins"] = None
        if case["packed"]:
            s["begins"] = (torch.rand(n, T, generator=g, device=DEV) < 8 / (T + 8)).to(torch.uint8)
        if kind == "rec_bwd":
            s["out"] = _plain_rec(s)["out"]
            s["dout"] = _gradients(g, n, T, D, type)
            s["dlast"] = torch.randn(n, D, generator=g, device=DEV) * 1e-2 if case["state"] else None
        return s
    s["x"], s["residual"] = _activations(g, n, T, D, type) * 0.5, _activations(g, n, T, D, type)
    s["gate"] = torch.randn(n, T, D, generator=g, device=DEV).to(type) if case["gate"] else None
    s["scale"] = _model_view(g, n, D, case["offset"], 0.05) if case["scale"] else None
    s["post"], s["pre"] = _model_view(g, n, D, case["offset"]), _model_view(g, n, D, case["offset"])
    if kind == "block_bwd":
        s["rstd"] = _plain_block(s)["rstd"]
        s["dy"] = _gradients(g, n, T, D, type)
        s["dtotal"] = _gradients(g, n, T, D, type) if case["dtotal"] else None
    return s


# ------------------------------------------------------------------ the plain form


def _values(x):
    """What x (fp32) is in the framework's 8 bits, as fp32: blocks of 32 whole multiples of a power of two."""
    D = x.shape[-1]
    b = torch.nn.functional.pad(x, (0, -D % BLOCK)).unflatten(-1, (-1, BLOCK))
    c = torch.clamp((b.abs().amax(-1).view(torch.int32) + 0x10000) >> 23, 7, 255)
    q = torch.round(b * ((260 - c) << 23).view(torch.float32)[..., None])
    unit = ((c - 6) << 23).view(torch.float32)
    return (q * torch.where(c == 255, float("nan"), unit)[..., None]).flatten(-2)[..., :D]


def _used(lengths, T):
    """[n][T][1]: whether a token is one of its worker's."""
    return (torch.arange(T, device=DEV)[None, :] < lengths[:, None])[..., None]


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the tokens, both overwritten, in doubling steps."""
    step, T = 1, b.shape[1]
    while step < T:
        b[:, step:] += a[:, step:] * b[:, :-step]
        a[:, step:] = a[:, step:] * a[:, :-step]
        step *= 2
    return b


def _plain_rec(s):
    case = s["case"]
    T, type = case["T"], TYPES[case["type"]]
    g, v = s["gate"].float(), s["value"].float()
    keep, b = 1 / (1 + torch.exp(-g)), v / (1 + torch.exp(g))
    if s["begins"] is not None:
        keep = torch.where(s["begins"][..., None] != 0, 0.0, keep)
    if s["lengths"] is not None:  # padding leaves the state as it is
        used = _used(s["lengths"], T)
        keep, b = torch.where(used, keep, 1.0), torch.where(used, b, 0.0)
    if s["initial"] is not None:
        b[:, 0] += keep[:, 0] * s["initial"]
    h = _scan(keep, b)
    last = h[:, -1].clone()
    if s["lengths"] is not None:
        h = torch.where(used, h, 0.0)
    out = {"out": h.to(type)}
    if case["state"]:
        out["last"] = last
    return out


def _plain_rec_bwd(s):
    case = s["case"]
    T, type = case["T"], TYPES[case["type"]]
    g, v, h = s["gate"].float(), s["value"].float(), s["out"].float()
    f, rest, dh = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g)), s["dout"].float()
    keep, used = f, None
    if s["begins"] is not None:
        keep = torch.where(s["begins"][..., None] != 0, 0.0, f)
    if s["lengths"] is not None:
        used = _used(s["lengths"], T)
        keep, dh = torch.where(used, keep, 1.0), torch.where(used, dh, 0.0)
    if s["dlast"] is not None:
        dh = torch.cat([dh[:, :-1], (dh[:, -1] + s["dlast"])[:, None]], 1)
    # lambda_t = dh_t + keep_{t+1} lambda_{t+1}: the same scan from the other end
    after = torch.cat([keep[:, 1:], torch.zeros_like(keep[:, :1])], 1)
    l = _scan(after.flip(1), dh.flip(1)).flip(1)
    first = torch.zeros_like(h[:, :1]) if s["initial"] is None else s["initial"][:, None]
    before = torch.cat([first, h[:, :-1]], 1)
    if s["begins"] is not None:
        before = torch.where(s["begins"][..., None] != 0, 0.0, before)
    dvalue, dgate = l * rest, l * (before - v) * f * rest
    if used is not None:
        dvalue, dgate = torch.where(used, dvalue, 0.0), torch.where(used, dgate, 0.0)
    out = {"dgate": dgate.to(type), "dvalue": dvalue.to(type)}
    if case["state"]:
        out["dinitial"] = keep[:, 0] * l[:, 0]
    return out


def _plain_block(s):
    case = s["case"]
    type = TYPES[case["type"]]
    x, r = s["x"].float(), s["residual"].float()
    sx = 1 / torch.sqrt((x * x).mean(-1) + EPS)
    h = x * sx[..., None] * s["post"][:, None]
    if s["gate"] is not None:
        h = h / (1 + torch.exp(-s["gate"].float()))
    h = h + (r if s["scale"] is None else r * s["scale"][:, None])
    sh = 1 / torch.sqrt((h * h).mean(-1) + EPS)
    hhat = h * sh[..., None]
    out = {"total": h.to(type), "y": (hhat * s["pre"][:, None]).to(type), "rstd": torch.stack([sx, sh])}
    if case.get("ckpt"):
        out["recalled"] = _values(hhat).to(torch.bfloat16)
    return out


def _plain_block_bwd(s):
    case = s["case"]
    T, type = case["T"], TYPES[case["type"]]
    x, r, dy, (sx, sh) = s["x"].float(), s["residual"].float(), s["dy"].float(), s["rstd"][..., None]
    p = 1.0 if s["gate"] is None else 1 / (1 + torch.exp(-s["gate"].float()))
    rho = torch.ones_like(s["post"]) if s["scale"] is None else s["scale"]
    xhat = x * sx
    m = xhat * s["post"][:, None]
    hhat = (r * rho[:, None] + m * p) * sh
    used = None if s["lengths"] is None else _used(s["lengths"], T)
    if used is not None:
        dy = torch.where(used, dy, 0.0)
    u = dy * s["pre"][:, None]
    dh = sh * (u - hhat * (u * hhat).mean(-1, keepdim=True))
    if s["dtotal"] is not None:
        dtotal = s["dtotal"].float()
        dh = dh + (dtotal if used is None else torch.where(used, dtotal, 0.0))
    dm = dh * p
    v = dm * s["post"][:, None]
    dx = sx * (v - xhat * (v * xhat).mean(-1, keepdim=True))
    out = {"dx": dx.to(type), "dresidual": (dh * rho[:, None]).to(type), "dpost": (dm * xhat).sum(1), "dpre": (dy * hhat).sum(1)}
    if s["gate"] is not None:
        out["dgate"] = (dh * m * p * (1 - p)).to(type)
    if s["scale"] is not None:
        out["dscale"] = (dh * r).sum(1)
    return out


def _plain_ortho(s):
    u = s["update"]
    x = u / (torch.sqrt((u * u).sum((1, 2), keepdim=True)) + ORTHO_EPS)
    tall = x.shape[1] > x.shape[2]
    if tall:
        x = x.transpose(1, 2)
    for _ in range(STEPS):
        gram = torch.bmm(x, x.transpose(1, 2))
        x = A * x + torch.bmm(B * gram + C * torch.bmm(gram, gram), x)
    return {"out": (x.transpose(1, 2) if tall else x).contiguous()}


_PLAIN = {"rec": _plain_rec, "rec_bwd": _plain_rec_bwd, "block": _plain_block, "block_bwd": _plain_block_bwd, "ortho": _plain_ortho}


# ------------------------------------------------------------------ the framework's operators


def _buffers(s):
    """The outputs and workspaces that a program keeps from step to step."""
    import paper_2110_04175_gb300 as rs

    case = s["case"]
    kind, n = case["kind"], case["n"]

    def model_rows(count):
        off = case["offset"]
        return torch.empty(n, (off + count + 31) // 32 * 32, device=DEV)[:, off:off + count]

    def work(size):
        return torch.empty(size, dtype=torch.uint8, device=DEV)

    if kind == "ortho":
        r, c = case["rows"], case["cols"]
        return {"rs": rs, "out": model_rows(r * c).unflatten(1, (r, c)), "work": work(rs.relay_orthogonalise_workspace(n, r, c))}
    T, D, type = case["T"], case["D"], TYPES[case["type"]]

    def rows(t=type):
        return torch.empty(n, T, D, dtype=t, device=DEV)

    b = {"rs": rs}
    if kind in ("rec", "rec_bwd"):
        b["work"] = work(rs.relay_recurrence_workspace(n, T, D))
        state = torch.empty(n, D, device=DEV) if case["state"] else None
        b.update({"out": rows(), "last": state} if kind == "rec" else {"dgate": rows(), "dvalue": rows(), "dinitial": state})
    elif kind == "block":
        b.update(total=rows(), y=rows(), rstd=torch.empty(2, n, T, device=DEV))
        if case["ckpt"]:
            b.update(kept=rs.ActivationCheckpoint(n, T, D, device=DEV), recalled=rows(torch.bfloat16))
    else:
        b.update(dx=rows(), dresidual=rows(), dpost=model_rows(D), dpre=model_rows(D),
                 work=work(rs.relay_block_norm_backward_workspace(n, T, D)))
        if case["gate"]:
            b["dgate"] = rows()
        if case["scale"]:
            b["dscale"] = model_rows(D)
    return b


def _kernels(s):
    if "buffers" not in s:
        s["buffers"] = _buffers(s)
    b, case = s["buffers"], s["case"]
    rs, kind = b["rs"], case["kind"]
    if kind == "ortho":
        rs.relay_orthogonalise(s["update"], b["out"], b["work"], steps=STEPS, eps=ORTHO_EPS)
        return {"out": b["out"]}
    if kind == "rec":
        rs.relay_recurrence(s["gate"], s["value"], b["out"], b["work"], initial=s["initial"], last=b["last"], begins=s["begins"],
                            lengths=s["lengths"])
        return {"out": b["out"], "last": b["last"]} if case["state"] else {"out": b["out"]}
    if kind == "rec_bwd":
        rs.relay_recurrence_backward(s["dout"], s["gate"], s["value"], s["out"], b["dgate"], b["dvalue"], b["work"],
                                     initial=s["initial"], dlast=s["dlast"], dinitial=b["dinitial"], begins=s["begins"],
                                     lengths=s["lengths"])
        return {k: b[k] for k in (("dgate", "dvalue", "dinitial") if case["state"] else ("dgate", "dvalue"))}
    if kind == "block":
        kept = b["kept"] if case["ckpt"] else None
        rs.relay_block_norm(s["x"], s["residual"], s["post"], s["pre"], b["total"], b["y"], EPS, gate=s["gate"], scale=s["scale"],
                            rstd=b["rstd"], checkpoint=kept)
        if kept is None:
            return {k: b[k] for k in ("total", "y", "rstd")}
        rs.relay_checkpoint_unpack(kept, b["recalled"])
        return {k: b[k] for k in ("total", "y", "rstd", "recalled")}
    rs.relay_block_norm_backward(s["dy"], s["x"], s["residual"], s["post"], s["pre"], s["rstd"], b["dx"], b["dresidual"], b["dpost"],
                                 b["dpre"], b["work"], gate=s["gate"], scale=s["scale"], dtotal=s["dtotal"], dgate=b.get("dgate"),
                                 dscale=b.get("dscale"), lengths=s["lengths"])
    return {k: b[k] for k in ("dx", "dresidual", "dpost", "dpre", "dgate", "dscale") if k in b}


def run(state):
    return _kernels(state) if own else _PLAIN[state["case"]["kind"]](state)


# ------------------------------------------------------------------ what a pass cannot do without


def work(case):
    """Inputs read once and outputs written once; what is put away in 8 bits and recalled within a pass is neither."""
    n, kind = case["n"], case["kind"]
    if kind == "ortho":
        m, k = min(case["rows"], case["cols"]), max(case["rows"], case["cols"])
        # x x^T and its square are symmetric: half of each
        return {"bytes": 8 * n * m * k, "flops": STEPS * n * m * m * (m + 3 * k)}
    T, D, e = case["T"], case["D"], SIZE[case["type"]]
    cells = n * T * D
    used = D * (sum(_lengths(case)) if case.get("lengths") else n * T)
    if kind in ("rec", "rec_bwd"):
        read, written = (2, 1) if kind == "rec" else (4, 2)
        side = n * T * case["packed"] + 8 * n * D * case["state"] * (1 if kind == "rec" else 1.5)
        return {"bytes": int(used * e * read + cells * e * written + side), "flops": (8 if kind == "rec" else 14) * used}
    if kind == "block":
        b = cells * (e * (4 + case["gate"]) + 2 * case["ckpt"]) + 4 * n * (2 * T + D * (2 + case["scale"]))
        return {"bytes": b, "flops": 16 * cells}
    read, written = 3 + case["gate"] + case["dtotal"], 2 + case["gate"]
    return {"bytes": e * (used * read + cells * written) + 4 * n * (2 * T + 2 * D * (2 + case["scale"])), "flops": 32 * used}


# ------------------------------------------------------------------ the definitions in 64 bits


def _sequences(s):
    """Each worker's sequences as (worker, first token, one past the last, whether the state before it counts)."""
    case = s["case"]
    n, T = case["n"], case["T"]
    ends = [T] * n if s["lengths"] is None else s["lengths"].tolist()
    for i in range(n):
        cuts = [] if s["begins"] is None else [t for t in torch.nonzero(s["begins"][i, :ends[i]]).flatten().tolist()]
        bounds = sorted({0, ends[i], *cuts})
        for a, b in zip(bounds, bounds[1:]):
            yield i, a, b, a not in cuts


def _marks(s):
    """[n][T]: tokens that take nothing from before them; and which are used."""
    case = s["case"]
    used = torch.zeros(case["n"], case["T"], dtype=torch.bool, device=DEV)
    new = torch.zeros_like(used)
    for i, a, b, goes_on in _sequences(s):
        used[i, a:b] = True
        new[i, a] = not goes_on
    return new, used


def _exact_rec(s):
    case = s["case"]
    n, T, D = case["n"], case["T"], case["D"]
    new, used = _marks(s)
    h = torch.zeros(n, D, dtype=torch.float64, device=DEV) if s["initial"] is None else s["initial"].double()
    out = torch.zeros(n, T, D, dtype=torch.float64, device=DEV)
    f = torch.sigmoid(s["gate"].double())
    add = s["value"].double() * torch.sigmoid(-s["gate"].double())
    for t in range(T):
        h = torch.where(used[:, t, None], torch.where(new[:, t, None], 0.0, h * f[:, t]) + add[:, t], h)
        out[:, t] = h
    out[~used] = 0
    return {"out": out, "last": h} if case["state"] else {"out": out}


def _exact_rec_bwd(s):
    case = s["case"]
    n, T, D = case["n"], case["T"], case["D"]
    new, used = _marks(s)
    g, v, h, dh = (s[k].double() for k in ("gate", "value", "out", "dout"))
    f, rest = torch.sigmoid(g), torch.sigmoid(-g)
    carry = torch.zeros(n, D, dtype=torch.float64, device=DEV) if s["dlast"] is None else s["dlast"].double()
    l = torch.zeros(n, T, D, dtype=torch.float64, device=DEV)
    for t in range(T - 1, -1, -1):  # carry: what reaches the state behind token t
        here = torch.where(used[:, t, None], dh[:, t] + carry, 0.0)
        l[:, t] = here
        carry = torch.where(used[:, t, None], torch.where(new[:, t, None], 0.0, here * f[:, t]), carry)
    before = torch.zeros_like(h)
    before[:, 1:] = h[:, :-1]
    if s["initial"] is not None:
        before[:, 0] = s["initial"].double()
    before[new] = 0
    dgate = l * (before - v) * (f * rest)
    dgate[~used] = 0
    out = {"dgate": dgate, "dvalue": l * rest}
    if case["state"]:
        out["dinitial"] = carry
    return out


def _nearest(x):
    """The values that x (64 bits) gets in 8 bits: whole multiples of the block's unit, the least power of two whose
    127 multiples reach the block's largest magnitude once that is rounded."""
    D = x.shape[-1]
    padded = torch.zeros(*x.shape[:-1], -(-D // BLOCK) * BLOCK, dtype=torch.float64, device=x.device)
    padded[..., :D] = x
    most = padded.reshape(*x.shape[:-1], -1, BLOCK).abs().max(-1).values
    m, e = torch.frexp(torch.clamp(most, min=2.0 ** -126))  # most = m 2^e, 1/2 <= m < 1
    e = torch.clamp(e - 7 + (m * 128 >= 127.5).int(), min=-126)
    unit = ((e.long() + 1023) << 52).view(torch.float64).repeat_interleave(BLOCK, -1)[..., :D]
    return torch.round(x / unit) * unit


def _exact_block(s):
    D = s["case"]["D"]
    x, r = s["x"].double(), s["residual"].double()
    sx = (torch.linalg.vector_norm(x, dim=-1) ** 2 / D + EPS) ** -0.5
    m = torch.einsum("ntd,nt,nd->ntd", x, sx, s["post"].double())
    if s["gate"] is not None:
        m = m * torch.sigmoid(s["gate"].double())
    h = m + (r if s["scale"] is None else torch.einsum("ntd,nd->ntd", r, s["scale"].double()))
    sh = (torch.linalg.vector_norm(h, dim=-1) ** 2 / D + EPS) ** -0.5
    out = {"total": h, "y": torch.einsum("ntd,nt,nd->ntd", h, sh, s["pre"].double()), "rstd": torch.stack([sx, sh])}
    if s["case"].get("ckpt"):
        out["recalled"] = _nearest(h * sh[..., None])
    return out


def _exact_block_bwd(s):
    case = s["case"]
    n, T, D = case["n"], case["T"], case["D"]
    x, r, dy, post, pre = (s[k].double() for k in ("x", "residual", "dy", "post", "pre"))
    sx, sh = s["rstd"].double()
    over = torch.zeros_like(dy) if s["dtotal"] is None else s["dtotal"].double()
    if s["lengths"] is not None:
        for i, m in enumerate(s["lengths"].tolist()):
            dy[i, m:], over[i, m:] = 0, 0
    rho = torch.ones(n, D, dtype=torch.float64, device=DEV) if s["scale"] is None else s["scale"].double()
    z = torch.full_like(dy, math.inf) if s["gate"] is None else s["gate"].double()
    p = torch.sigmoid(z)
    xhat = torch.einsum("ntd,nt->ntd", x, sx)
    m = torch.einsum("ntd,nd->ntd", xhat, post)
    hhat = torch.einsum("ntd,nt->ntd", torch.einsum("ntd,nd->ntd", r, rho) + p * m, sh)
    along = torch.einsum("ntd,nd,ntd->nt", dy, pre, hhat) / D
    dh = (torch.einsum("ntd,nd->ntd", dy, pre) - hhat * along[..., None]) * sh[..., None] + over
    v = torch.einsum("ntd,ntd,nd->ntd", dh, p, post)
    dx = (v - xhat * (torch.einsum("ntd,ntd->nt", v, xhat) / D)[..., None]) * sx[..., None]
    out = {"dx": dx, "dresidual": torch.einsum("ntd,nd->ntd", dh, rho), "dpost": torch.einsum("ntd,ntd,ntd->nd", dh, p, xhat),
           "dpre": torch.einsum("ntd,ntd->nd", dy, hhat)}
    if s["gate"] is not None:
        out["dgate"] = dh * m * (p * torch.sigmoid(-z))
    if s["scale"] is not None:
        out["dscale"] = torch.einsum("ntd,ntd->nd", dh, r)
    return out


def _exact_ortho(s):
    """x <- a x + (x x^T) (b x + c (x x^T) x), or from the other side where rows outnumber columns."""
    out = torch.empty(s["update"].shape, dtype=torch.float64, device=DEV)
    for i, u in enumerate(s["update"]):
        x = u.double()
        x = x / (torch.linalg.matrix_norm(x) + ORTHO_EPS)
        for _ in range(STEPS):
            if x.shape[0] <= x.shape[1]:
                gram = x @ x.T
                x = A * x + gram @ (B * x + C * (gram @ x))
            else:
                gram = x.T @ x
                x = A * x + (B * x + C * (x @ gram)) @ gram
        out[i] = x
    return {"out": out}


_EXACT = {"rec": _exact_rec, "rec_bwd": _exact_rec_bwd, "block": _exact_block, "block_bwd": _exact_block_bwd, "ortho": _exact_ortho}


def exact(case, seed):
    return _EXACT[case["kind"]](prepare(case, seed))
