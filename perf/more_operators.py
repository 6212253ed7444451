"""The operators of a recurrent readout with a matrix for a state, as cases that can be timed and compared.

A case is a dict of plain values.  `kind` says what one pass is:

  heads        norm of every head of queries and keys and the rotation by position; with `train` its backward pass too
  delta        gated delta rule over whole sequences
  delta_train  the same forward and backward
  delta_step   one token of every sequence, the states in a pool

For every sequence and head, with a = sigmoid(gate), b = sigmoid(write) and a state S [Dk, Dv]:
S <- a S,  u = b (v - S^T k),  S <- S + k u^T,  out = S^T q; `hv / hk` heads of values share a head of queries and keys.
`own` chooses between the library's calls and their plain form: elementary tensor operations in 32 bits (64 for angles and sums of
logarithms), rounded once at the end.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-6
BASE = 10000.0
CHUNK = 64                      # steps that the plain form takes at once
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, kind, **values):
    c = dict(kind=kind, dtype="bf16", rows=0, hq=0, T=0, B=0, hk=0, hv=0, dk=0, dv=0, axes="", interleaved=False, far=0,
             train=False, ragged=False, slots=0)
    c.update(values)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # queries and keys of one token of 16 sequences in a serving loop: launch latency
        _case("heads_tokens", "heads", rows=16, hq=16, hk=8, dk=128, axes="64", far=200_000),
        # forward and backward of a training batch
        _case("heads_train", "heads", rows=16384, hq=16, hk=8, dk=128, axes="64", train=True),
        # 20 frames of 32 x 32 places with positions in time, height and width, fp32
        _case("heads_frames", "heads", dtype="f32", rows=20480, hq=4, hk=4, dk=64, axes="8,12,12", interleaved=True, train=True),
        # one long sequence far from its start, a quarter of the features rotated
        _case("heads_long", "heads", rows=65536, hq=16, hk=2, dk=128, axes="16", far=3_000_000),
        # one token of one sequence
        _case("step_one", "delta_step", B=1, hk=8, hv=16, dk=128, dv=128, slots=8),
        # one token of 128 running sequences out of a pool of states
        _case("step_tokens", "delta_step", B=128, hk=8, hv=16, dk=128, dv=128, slots=160),
        # one long sequence: few heads, a long chain
        _case("delta_long", "delta", T=32768, B=1, hk=8, hv=16, dk=128, dv=128),
        # prompts of unequal lengths, odd sizes
        _case("delta_prompt", "delta", T=777, B=5, hk=3, hv=6, dk=96, dv=80, ragged=True),
        # a training batch of sequences of unequal lengths
        _case("delta_train", "delta_train", T=2048, B=8, hk=8, hv=16, dk=128, dv=128, ragged=True),
        # the rate-coded network's readout: 25 frames of 128 images, 128 channels as 4 heads, fp32
        _case("delta_readout", "delta_train", dtype="f32", T=25, B=128, hk=4, hv=4, dk=32, dv=32),
        # fp32 training, shared heads, odd sizes
        _case("delta_train_f32", "delta_train", dtype="f32", T=500, B=3, hk=2, hv=4, dk=64, dv=100),
    ]


# ---- drawn cases -------------------------------------------------------------------------------

def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _width(rng, low, high):
    """A head's width: half of them multiples of 16, the others whatever comes, odd ones among them."""
    v = rng.randint(low, high)
    return max(16, v // 16 * 16) if rng.random() < 0.5 else v


def draw(rng):
    """Another case of the listed ranges, at most half of the largest listed case of its kind."""
    kind = rng.choice(["heads", "heads", "delta", "delta_train", "delta_step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    hk = rng.choice([1, 2, 3, 4, 8])
    if kind == "heads":
        d = 2 * max(8, _width(rng, 8, 128) // 2 * (1 if rng.random() < 0.5 else 2))
        d = min(d, 256)
        hq = hk * rng.choice([1, 2, 4])
        pairs = rng.randint(1, d // 2)
        if pairs >= 3 and rng.random() < 0.4:
            first = rng.randint(1, pairs - 2)
            second = rng.randint(1, pairs - first - 1)
            axes = "%d,%d,%d" % (first, second, pairs - first - second)
        else:
            axes = str(rng.choice([d // 2, pairs]))
        return _case(None, kind, dtype=dtype, rows=_log_int(rng, 1, min(65536, 40_000_000 // ((hq + hk) * d))), hq=hq, hk=hk, dk=d,
                     axes=axes, interleaved=rng.random() < 0.4, far=rng.choice([0, 0, 5000, 1_000_000]), train=rng.random() < 0.6)
    hv, dk, dv = hk * rng.choice([1, 1, 2, 3]), _width(rng, 16, 128), _width(rng, 16, 160)
    if kind == "delta_step":
        B = _log_int(rng, 1, min(256, 16_000_000 // (hv * dk * dv)))
        return _case(None, kind, dtype=dtype, B=B, hk=hk, hv=hv, dk=dk, dv=dv, slots=B + rng.randint(0, 30))
    most = {("delta", "bf16"): 250_000, ("delta", "f32"): 60_000, ("delta_train", "bf16"): 120_000, ("delta_train", "f32"): 30_000}[kind, dtype]
    T = _log_int(rng, 1, min(16384 if kind == "delta" else 4096, most // hv))
    B = _log_int(rng, 1, max(1, min(64, most // (T * hv))))
    return _case(None, kind, dtype=dtype, T=T, B=B, hk=hk, hv=hv, dk=dk, dv=dv, ragged=B > 1 and rng.random() < 0.5)


def work(c):
    """What a pass cannot do without: inputs read once, outputs written once, the recurrence's operations step by step."""
    s = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "heads":
        n = c["rows"] * (c["hq"] + c["hk"]) * c["dk"]
        return {"bytes": n * s * (5 if c["train"] else 2) + 4 * c["rows"] * len(c["axes"].split(",")), "flops": n * (25 if c["train"] else 8)}
    tokens = c["B"] * max(1, c["T"])
    qk, v, gates = 2 * tokens * c["hk"] * c["dk"] * s, tokens * c["hv"] * c["dv"] * s, 2 * tokens * c["hv"] * s
    one = tokens * c["hv"] * c["dk"] * c["dv"]
    states = 4 * c["B"] * c["hv"] * c["dk"] * c["dv"]
    if c["kind"] == "delta_train":
        return {"bytes": 2 * (qk + 2 * v + gates) + 4 * states, "flops": 18 * one}
    return {"bytes": qk + 2 * v + gates + 2 * states, "flops": 6 * one}


# ---- inputs ------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)


def _uniform(g, low, high, *shape):
    return torch.rand(shape, generator=g, device=DEVICE, dtype=torch.float32) * (high - low) + low


def _unit(x):
    return x * torch.rsqrt(x.square().sum(-1, keepdim=True) + 1e-6)


def prepare(c, seed):
    g, dt = _generator(seed), DTYPES[c["dtype"]]
    s = {"case": c}
    if c["kind"] == "heads":
        R, hq, hk, D = c["rows"], c["hq"], c["hk"], c["dk"]
        # queries and keys are slices of one product's rows
        rows = (_normal(g, R, (hq + hk) * D) * torch.exp(0.5 * _normal(g, (hq + hk) * D))).to(dt)
        s["q"], s["k"] = rows[:, :hq * D].view(R, hq, D), rows[:, hq * D:].view(R, hk, D)
        s["gain_q"], s["gain_k"] = 1 + 0.2 * _normal(g, D), 1 + 0.2 * _normal(g, D)
        at = torch.arange(R, device=DEVICE, dtype=torch.int32)
        s["sections"] = tuple(int(n) for n in c["axes"].split(","))
        if len(s["sections"]) == 3:
            s["positions"] = torch.stack([at // 1024, at // 32 % 32, at % 32], 1).contiguous()
        else:
            start = (_uniform(g, 0, 1, 1) * c["far"]).to(torch.int32)
            # tokens of a serving loop stand at positions of their own; others follow each other
            s["positions"] = at + start if R > 64 else (_uniform(g, 0, 1, R) * (c["far"] + 1)).to(torch.int32)
        if c["train"]:
            s["grad_q"], s["grad_k"] = (1e-3 * _normal(g, R, hq, D)).to(dt), (1e-3 * _normal(g, R, hk, D)).to(dt)
        return s
    T, B, hk, hv, dk, dv = (c[n] for n in ("T", "B", "hk", "hv", "dk", "dv"))
    lead = (B,) if c["kind"] == "delta_step" else (T, B)
    # keys of a head have a direction in common, as features do
    s["q"] = _unit(_normal(g, *lead, hk, dk)).to(dt)
    s["k"] = _unit(_normal(g, *lead, hk, dk) + _normal(g, hk, dk)).to(dt)
    # values and both gates are slices of one product's rows; leaks from 0.5 to nearly 1, one range per head
    rows = _normal(g, *lead, hv * dv + 2 * hv)
    rows[..., hv * dv:hv * dv + hv] += _uniform(g, 0, 7, hv)
    s["rows"] = rows.to(dt)
    if c["kind"] == "delta_step":
        s["pool"] = _normal(g, c["slots"], hv, dk, dv) / math.sqrt(dk)
        s["slots"] = torch.randperm(c["slots"], generator=g, device=DEVICE)[:B].to(torch.int32)
        return s
    s["h0"] = _normal(g, B, hv, dk, dv) / math.sqrt(dk)
    s["lengths"] = None
    if c["ragged"]:
        lengths = (_uniform(g, 0, 1, B) * (T + 1)).to(torch.int32).clamp(0, T)
        lengths[0] = T
        s["lengths"] = lengths
    if c["kind"] == "delta_train":
        s["grad_out"] = (1e-2 * _normal(g, T, B, hv, dv)).to(dt)
        s["grad_h_last"] = 1e-2 * _normal(g, B, hv, dk, dv)
    return s


def _parts(rows, hv, dv):
    """Values [.., hv, dv], gates and write strengths [.., hv] of a product's rows."""
    n = hv * dv
    return rows[..., :n].unflatten(-1, (hv, dv)), rows[..., n:n + hv], rows[..., n + hv:]


# ---- one pass ----------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2603_13810_amd import api
    c = s["case"]
    if c["kind"] == "heads":
        how = dict(eps=EPS, positions=s["positions"], sections=s["sections"], base=BASE, interleaved=c["interleaved"])
        out = api.tac_head_norm(s["q"], s["k"], s["gain_q"], s["gain_k"], **how)
        if c["train"]:
            out.update(api.tac_head_norm_backward(s["q"], s["k"], s["gain_q"], s["gain_k"], s["grad_q"], s["grad_k"], **how))
        return out
    value, gate, write = _parts(s["rows"], c["hv"], c["dv"])
    if c["kind"] == "delta_step":
        return {"out": api.tac_delta_step(s["q"], s["k"], value, gate, write, s["pool"], s["slots"]), "pool": s["pool"]}
    train = c["kind"] == "delta_train"
    r = api.tac_delta_scan(s["q"], s["k"], value, gate, write, lengths=s["lengths"], h0=s["h0"], want_kept=train)
    out = {"out": r["out"], "h_last": r["h_last"]}
    if train:
        rows = torch.empty_like(s["rows"])
        grad_value, grad_gate, grad_write = _parts(rows, c["hv"], c["dv"])
        g = api.tac_delta_scan_backward(s["q"], s["k"], value, gate, write, r["states"], r["updates"], s["grad_out"], lengths=s["lengths"],
                                        grad_h_last=s["grad_h_last"], grad_value=grad_value, grad_gate=grad_gate, grad_write=grad_write)
        out.update(grad_rows=rows, grad_q=g["grad_query"], grad_k=g["grad_key"], grad_h0=g["grad_h0"])
    return out


def _pair_index(D, n, interleaved):
    """Where the first and the second features of the `n` rotated pairs stand."""
    i = torch.arange(n, device=DEVICE)
    return (2 * i, 2 * i + 1) if interleaved else (i, n + i)


def _angles(positions, sections):
    """Angles [rows, pairs] in 64 bits."""
    p = positions.double()
    if len(sections) == 1:
        p = p.reshape(-1, 1)
    parts = [p[:, a:a + 1] * torch.exp(torch.arange(n, device=DEVICE, dtype=torch.float64) * (-math.log(BASE) / n)) for a, n in enumerate(sections)]
    return torch.cat(parts, 1)


def _rotated(x, cos, sin, first, second):
    y = x.clone()
    u, v = x[..., first], x[..., second]
    y[..., first] = u * cos - v * sin
    y[..., second] = v * cos + u * sin
    return y


def _plain_heads(s):
    c, dt, out = s["case"], DTYPES[s["case"]["dtype"]], {}
    first, second = _pair_index(c["dk"], sum(s["sections"]), c["interleaved"])
    angle = _angles(s["positions"], s["sections"])
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    for name in ("q", "k"):
        x, gain = s[name].float(), s["gain_" + name]
        rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        out[name] = _rotated(x * rstd * gain, cos, sin, first, second).to(dt)
        if c["train"]:
            n = x * rstd
            gy = _rotated(s["grad_" + name].float(), cos, -sin, first, second)
            w = gy * gain
            out["grad_" + name] = (rstd * (w - n * (w * n).mean(-1, keepdim=True))).to(dt)
            out["grad_gain_" + name] = (gy * n).sum((0, 1))
    return out


def _unit_lower_inverse(A):
    """(I + A)^-1 of strictly lower triangular matrices [.., C, C], C a power of two: blocks of doubled size."""
    C = A.shape[-1]
    T = torch.eye(C, device=A.device, dtype=A.dtype).expand(A.shape).clone()
    size = 1
    while size < C:
        blocks = T.unflatten(-2, (C // (2 * size), 2, size)).unflatten(-1, (C // (2 * size), 2, size))
        at = torch.arange(C // (2 * size), device=A.device)
        low = A.unflatten(-2, (C // (2 * size), 2, size)).unflatten(-1, (C // (2 * size), 2, size))[..., at, 1, :, at, 0, :]
        blocks[..., at, 1, :, at, 0, :] = -blocks[..., at, 1, :, at, 1, :] @ low @ blocks[..., at, 0, :, at, 0, :]
        size *= 2
    return T


def _chain(m, b):
    """s_c = m_c s_{c-1} + b_c from s = 0 along the first axis, in log2 steps of doubled reach."""
    reach = 1
    while reach < m.shape[0]:
        b = torch.cat([b[:reach], b[reach:] + m[reach:] @ b[:-reach]])
        m = torch.cat([m[:reach], m[reach:] @ m[:-reach]])
        reach *= 2
    return b


def _log_sigmoid(x):
    return torch.clamp(x, max=0) - torch.log1p(torch.exp(-x.abs()))


def _plain_delta(s):
    c, dt = s["case"], DTYPES[s["case"]["dtype"]]
    T, B, hk, hv, dk, dv = (c[n] for n in ("T", "B", "hk", "hv", "dk", "dv"))
    N, pad = -(-T // CHUNK), -T % CHUNK
    live = torch.ones((T, B), dtype=torch.bool, device=DEVICE)
    if s["lengths"] is not None:
        live = torch.arange(T, device=DEVICE)[:, None] < s["lengths"][None, :]

    def chunks(x):
        """[T, B, H, ..] -> [N, B, H, C, ..] in 32 bits, zero where no step is."""
        x = torch.where(live.view(T, B, *[1] * (x.dim() - 2)), x.float(), torch.zeros((), device=DEVICE))
        x = torch.cat([x, x.new_zeros(pad, *x.shape[1:])]).unflatten(0, (N, CHUNK))
        return x.movedim(1, 3)

    def steps(x):
        """Back to [T, B, H, ..]."""
        return x.movedim(3, 1).flatten(0, 1)[:T]

    spread = lambda x: x.repeat_interleave(hv // hk, 2)
    value, gate, write = _parts(s["rows"], hv, dv)
    q, k, v = spread(chunks(s["q"])), spread(chunks(s["k"])), chunks(value)
    on = chunks(torch.ones((T, B, hv), device=DEVICE))
    b = torch.sigmoid(chunks(write)) * on
    G = torch.cumsum(_log_sigmoid(chunks(gate).double()) * on, -1)            # [N, B, H, C]
    lower = torch.ones((CHUNK, CHUNK), device=DEVICE, dtype=torch.bool).tril()
    decay = torch.where(lower, torch.exp(torch.where(lower, G[..., :, None] - G[..., None, :], 0 * G[..., None])), 0 * G[..., None]).float()
    start, rest, whole = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None], torch.exp(G[..., -1:]).float()[..., None]
    strict = lower.tril(-1)
    A = torch.where(strict, b[..., None] * decay * (k @ k.transpose(-1, -2)), 0 * decay)
    inverse = _unit_lower_inverse(A)
    W, U0 = inverse @ (b[..., None] * start * k), inverse @ (b[..., None] * v)
    kr = (rest * k).transpose(-1, -2).contiguous()
    M, fed = whole * torch.eye(dk, device=DEVICE) - kr @ W, kr @ U0
    states = _chain(torch.cat([M[:1], M]), torch.cat([s["h0"][None], fed]))
    S = states[:-1]
    U = U0 - W @ S
    P = decay * (q @ k.transpose(-1, -2))
    out = {"out": steps(start * (q @ S) + P @ U).to(dt), "h_last": states[-1].clone()}
    if c["kind"] == "delta":
        return out
    do = chunks(s["grad_out"])
    fed = (start * q).transpose(-1, -2) @ do - W.transpose(-1, -2) @ (P.transpose(-1, -2) @ do)
    back = M.transpose(-1, -2).contiguous().flip(0)
    dS = _chain(torch.cat([back[:1], back]), torch.cat([s["grad_h_last"][None], fed.flip(0)])).flip(0)
    grad_h0, dS = dS[0].clone(), dS[1:]
    R = inverse.transpose(-1, -2) @ (P.transpose(-1, -2) @ do + rest * (k @ dS))
    Y = decay * (do @ U.transpose(-1, -2))
    X = torch.where(strict, -b[..., None] * decay * (R @ U.transpose(-1, -2)), 0 * decay)
    dq = Y @ k + start * (do @ S.transpose(-1, -2))
    dk_read = X @ k - b[..., None] * start * (R @ S.transpose(-1, -2))
    from_state = rest * (U @ dS.transpose(-1, -2))
    dk_write = X.transpose(-1, -2) @ k + Y.transpose(-1, -2) @ q + from_state
    dG = ((dq * q).sum(-1) + ((dk_read - dk_write) * k).sum(-1)).double()
    dG[..., -1] += (whole[..., 0, 0] * (S * dS).sum((-1, -2)) + (from_state * k).sum((-1, -2))).double()
    sums = dG.flip(-1).cumsum(-1).flip(-1).float()
    dgate = torch.sigmoid(-chunks(gate)) * sums * on
    dwrite = (1 - b) * (R * U).sum(-1)
    shared = lambda x: steps(x).unflatten(2, (hk, hv // hk)).sum(3).to(dt)
    rows = torch.cat([steps(b[..., None] * R).flatten(2), steps(dgate), steps(dwrite)], 2)
    out.update(grad_rows=rows.to(dt), grad_q=shared(dq), grad_k=shared(dk_read + dk_write), grad_h0=grad_h0)
    return out


def _run_plain(s):
    c = s["case"]
    if c["kind"] == "heads":
        return _plain_heads(s)
    if c["kind"] != "delta_step":
        return _plain_delta(s)
    value, gate, write = (x.float() for x in _parts(s["rows"], c["hv"], c["dv"]))
    at, spread = s["slots"].long(), lambda x: x.float().repeat_interleave(c["hv"] // c["hk"], 1)
    q, k = spread(s["q"]), spread(s["k"])
    S = torch.sigmoid(gate)[..., None, None] * s["pool"][at]
    u = torch.sigmoid(write)[..., None] * (value - (S * k[..., None]).sum(2))
    S = S + k[..., None] * u[..., None, :]
    s["pool"][at] = S
    return {"out": (S * q[..., None]).sum(2).to(DTYPES[c["dtype"]]), "pool": s["pool"]}


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _exact_heads(c, s):
    names, out = ["q", "k"], {}
    # a rotation of every pair as a product of complex numbers
    for name in names:
        x, gain = s[name].double().requires_grad_(), s["gain_" + name].double().requires_grad_()
        y = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["dk"] + EPS) * gain
        n, at, turns = sum(s["sections"]), 0, []
        for axis, count in enumerate(s["sections"]):
            p = s["positions"].double() if len(s["sections"]) == 1 else s["positions"][:, axis].double()
            for i in range(count):
                turns.append(p / BASE ** (i / count))
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), torch.stack(turns, 1))[:, None]
        head, tail = y[..., :2 * n], y[..., 2 * n:]
        pairs = torch.view_as_complex(head.unflatten(-1, (n, 2) if c["interleaved"] else (2, n)).movedim(-1 if c["interleaved"] else -2, -1).contiguous())
        turned = torch.view_as_real(pairs * turn)
        turned = turned.flatten(-2) if c["interleaved"] else turned.movedim(-1, -2).flatten(-2)
        y = torch.cat([turned, tail], -1)
        out[name] = y.detach()
        if c["train"]:
            out["grad_" + name], out["grad_gain_" + name] = torch.autograd.grad(y, (x, gain), s["grad_" + name].double())
    return out


def exact(c, seed):
    s = prepare(c, seed)
    if c["kind"] == "heads":
        return _exact_heads(c, s)
    hk, hv, dk, dv = (c[n] for n in ("hk", "hv", "dk", "dv"))
    step, train = c["kind"] == "delta_step", c["kind"] == "delta_train"
    value, gate, write = _parts(s["rows"].double(), hv, dv)
    one = [s["q"].double(), s["k"].double(), value, 1 / (1 + torch.exp(-gate)), 1 / (1 + torch.exp(-write))]
    if step:
        # run() goes on from the states as they are, pass after pass; the first pass has these values
        one = [x[None] for x in one]
        T, B, state, lengths = 1, c["B"], s["pool"].double()[s["slots"].long()], None
    else:
        T, B, state, lengths = c["T"], c["B"], s["h0"].double(), s["lengths"]
    q, k, v, a, b = one
    group = torch.arange(hv, device=DEVICE) // (hv // hk)
    on = torch.ones((T, B), dtype=torch.bool, device=DEVICE)
    if lengths is not None:
        on = torch.arange(T, device=DEVICE)[:, None] < lengths[None, :]

    def forward(S, t):
        """(state behind step t, faded state, what is written, how far the value was from what is read)"""
        K = k[t][:, group]
        faded = a[t][..., None, None] * S
        miss = v[t] - (K[..., None, :] @ faded)[..., 0, :]
        u = b[t][..., None] * miss
        return torch.where(on[t][:, None, None, None], faded + K[..., :, None] * u[..., None, :], S), faded, u, miss

    out, kept, S = torch.zeros((T, B, hv, dv), dtype=torch.float64, device=DEVICE), {}, state
    for t in range(T):
        if train and t % 64 == 0:
            kept[t] = S
        S = forward(S, t)[0]
        out[t] = torch.where(on[t][:, None, None], (q[t][:, group][..., None, :] @ S)[..., 0, :], 0.0)
    if step:
        pool = s["pool"].double()
        pool[s["slots"].long()] = S
        return {"out": out[0], "pool": pool}
    result = {"out": out, "h_last": S}
    if train:
        dS, go = s["grad_h_last"].double(), s["grad_out"].double()
        dq, dkey, dv_, da, db = (torch.zeros_like(x) for x in (q, k, v, a, b))
        for begin in sorted(kept, reverse=True):
            before = [kept[begin]]
            for t in range(begin, min(begin + 64, T) - 1):
                before.append(forward(before[-1], t)[0])
            for t in range(min(begin + 64, T) - 1, begin - 1, -1):
                now, faded, u, miss = forward(before[t - begin], t)
                K, Q, live = k[t][:, group], q[t][:, group], on[t][:, None, None]
                D = dS + Q[..., :, None] * go[t][..., None, :]
                du = (K[..., None, :] @ D)[..., 0, :]
                w = b[t][..., None] * du
                dQ = (now @ go[t][..., :, None])[..., 0]
                dK = (D @ u[..., :, None])[..., 0] - (faded @ w[..., :, None])[..., 0]
                D = D - K[..., :, None] * w[..., None, :]
                dq[t].index_add_(1, group, torch.where(live, dQ, 0.0))
                dkey[t].index_add_(1, group, torch.where(live, dK, 0.0))
                dv_[t] = torch.where(live, w, 0.0)
                db[t] = torch.where(on[t][:, None], (du * miss).sum(-1) * b[t] * (1 - b[t]), 0.0)
                da[t] = torch.where(on[t][:, None], (D * before[t - begin]).sum((-1, -2)) * a[t] * (1 - a[t]), 0.0)
                dS = torch.where(live[..., None], a[t][..., None, None] * D, dS)
        result.update(grad_rows=torch.cat([dv_.flatten(2), da, db], 2), grad_q=dq, grad_k=dkey, grad_h0=dS)
    return result
