"""The dense operators that read a spiking stack's features over time, as cases that can be timed and compared.

A case is a dict of plain values.  `kind` says what one pass is:

  norm         residual addition and root-mean-square norm; with `train` its backward pass too
  project      a block's entry: residual norm written in 8 bits, product with the 8-bit weights (gates and values)
  product      features to 8 bits along their rows, product with the 8-bit weights, bias
  input_grad   output gradient to 8 bits along its rows, product with the transposed 8-bit weights
  weight_grad  output gradient to 8 bits along the tokens, the kept 8-bit activations laid out along the tokens, their product
  scan         gated linear recurrence over whole sequences
  scan_train   the same forward and backward
  step         one token of every sequence, the states in a pool

8-bit matrices are OCP e4m3 codes [rows, 128 ceil(cols / 128)] with one power of two per row and 128 columns, kept as
the byte 127 + exponent in [rows, 4 ceil(cols / 512)].  `own` chooses between the library's calls and their plain form:
elementary tensor operations in 32 bits (64 where sums or factors need them), rounded once at the end.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, kind, **values):
    c = dict(kind=kind, dtype="bf16", rows=0, cols=0, n=0, residual=True, train=False, spikes=False, T=0, B=0, D=0,
             ragged=False, slots=0)
    c.update(values)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the norm of one token of 16 sequences in a serving loop: launch latency
        _case("norm_tokens", "norm", rows=16, cols=2048),
        # forward and backward of a training batch
        _case("norm_train", "norm", rows=16384, cols=4096, train=True),
        # one token of 16 sequences through a block's entry: the weights' bytes
        _case("project_tokens", "project", rows=16, cols=4096, n=8192),
        # a prompt or training batch through the same entry: the matrix cores
        _case("project_batch", "project", rows=16384, cols=4096, n=8192),
        # the dense readout of the rate-coded network: 25 frames x 128 images of 64 x 7 x 7 spikes, 500 outputs, fp32
        _case("product_readout", "product", dtype="f32", rows=3200, cols=3136, n=500, spikes=True),
        # gradient of a training batch towards the block's input
        _case("input_grad", "input_grad", rows=8192, cols=4096, n=8192),
        # gradient of the block's weights from the activations kept in 8 bits
        _case("weight_grad", "weight_grad", rows=8192, cols=4096, n=8192),
        # the same for the readout's weights: few tiles of output, a long sum over ragged sizes, fp32 gradients
        _case("weight_grad_readout", "weight_grad", dtype="f32", rows=3200, cols=3136, n=128),
        # one token of 256 running sequences out of a pool of states
        _case("step_tokens", "step", B=256, D=4096, slots=512),
        # one long sequence
        _case("scan_long", "scan", T=32768, B=1, D=2048),
        # a training batch of sequences of unequal lengths
        _case("scan_train", "scan_train", T=2048, B=16, D=2048, ragged=True),
        # the rate-coded network's readout: 25 frames of 128 images, 128 leaky integrators, fp32
        _case("scan_readout", "scan_train", dtype="f32", T=25, B=128, D=128),
    ]


# ---- drawn cases -------------------------------------------------------------------------------

def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _columns(rng, low, high):
    """A width: half of them multiples of 64, the others whatever comes, odd ones among them."""
    v = _log_int(rng, low, high)
    return max(64, v // 64 * 64) if rng.random() < 0.5 else v


def draw(rng):
    """Another case of the listed ranges, at most half of the largest listed case of its kind."""
    kind = rng.choice(["norm", "norm", "project", "product", "input_grad", "weight_grad", "scan", "scan_train", "step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "norm":
        cols = _columns(rng, 64, 12000)
        return _case(None, kind, dtype=dtype, rows=_log_int(rng, 1, min(16384, 30_000_000 // cols)), cols=cols,
                     residual=rng.random() < 0.7, train=rng.random() < 0.6)
    if kind in ("project", "product", "input_grad", "weight_grad"):
        cols, n = _columns(rng, 100, 8192), _columns(rng, 64, 8192)
        low = 1 if kind in ("project", "product") else 32
        rows = _log_int(rng, low, min(16384, 250_000_000_000 // (cols * n)))
        return _case(None, kind, dtype="bf16" if kind == "project" else dtype, rows=rows, cols=cols, n=n,
                     residual=rng.random() < 0.7, spikes=kind == "product" and rng.random() < 0.3)
    if kind == "step":
        B = _log_int(rng, 1, 512)
        return _case(None, kind, dtype=dtype, B=B, D=_columns(rng, 64, 6000), slots=B + rng.randint(0, 200))
    T, D = _log_int(rng, 1, 32768), _columns(rng, 32, 4096)
    B = _log_int(rng, 1, max(1, min(256, 30_000_000 // (T * D))))
    while T * B * D > 30_000_000:
        T = max(1, T // 2)
    return _case(None, kind, dtype=dtype, T=T, B=B, D=D, ragged=B > 1 and rng.random() < 0.5)


def work(c):
    """What a pass cannot do without: inputs read once, outputs written once, the products' operations."""
    s = 2 if c["dtype"] == "bf16" else 4
    R, C, N, k = c["rows"], c["cols"], c["n"], c["kind"]
    if k == "norm":
        tensors = (4 if c["residual"] else 2) + ((4 if c["residual"] else 3) if c["train"] else 0)
        return {"bytes": R * C * s * tensors + 4 * C * (3 if c["train"] else 1), "flops": R * C * (15 if c["train"] else 5)}
    if k == "project":
        return {"bytes": R * C * s * (3 if c["residual"] else 1) + N * C + R * N * s, "flops": 2 * R * C * N}
    if k == "product":
        return {"bytes": R * C * s + N * C + R * N * s, "flops": 2 * R * C * N}
    if k == "input_grad":
        return {"bytes": R * N * s + N * C + R * C * s, "flops": 2 * R * C * N}
    if k == "weight_grad":
        return {"bytes": R * N * s + R * C + 4 * N * C, "flops": 2 * R * C * N}
    n = c["B"] * c["D"] * max(1, c["T"])
    if k == "step":
        return {"bytes": n * (3 * s + 8), "flops": 8 * n}
    return {"bytes": n * s * (3 if k == "scan" else 8), "flops": n * (8 if k == "scan" else 30)}


# ---- inputs ------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(int(seed))


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)


def _uniform(g, low, high, *shape):
    return torch.rand(shape, generator=g, device=DEVICE, dtype=torch.float32) * (high - low) + low


def _exponents(amax):
    """The smallest e with amax <= 448 * 2^e, from -127 on."""
    m, x = torch.frexp(amax)
    return torch.clamp(x - 9 + (m > 0.875).to(x.dtype), -127, 127)


def _power(e):
    """2^e as float32, e from -127 to 127: the exponent field itself, since pow() may be off in its last bit."""
    e = e.to(torch.int32)
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(torch.float32)


def _to_8bit(v, tiles=False):
    """Codes and scale bytes of a float32 matrix, blocks of 128 along its rows (or one scale for 128 x 128)."""
    R, C = v.shape
    kb = -(-C // 128)
    v = torch.nn.functional.pad(v, (0, kb * 128 - C))
    amax = v.abs().reshape(R, kb, 128).amax(2)
    if tiles:
        rb = -(-R // 128)
        top = torch.nn.functional.pad(amax, (0, 0, 0, rb * 128 - R)).reshape(rb, 128, kb).amax(1)
        amax = top.repeat_interleave(128, 0)[:R]
    e = _exponents(amax)
    q = (v.reshape(R, kb, 128) * _power(-e)[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).reshape(R, kb * 128)
    scales = torch.zeros((R, 4 * (-(-C // 512))), dtype=torch.uint8, device=v.device)
    scales[:, :kb] = (e + 127).to(torch.uint8)
    return q, scales


def _from_8bit(q, scales, cols):
    """The float32 values that codes and scale bytes stand for."""
    R, kb = q.shape[0], q.shape[1] // 128
    e = scales[:, :kb].to(torch.int32) - 127
    v = q.view(torch.float8_e4m3fn).to(torch.float32).reshape(R, kb, 128) * _power(e)[:, :, None]
    return v.reshape(R, kb * 128)[:, :cols]


def prepare(c, seed):
    g, dt, k = _generator(seed), DTYPES[c["dtype"]], c["kind"]
    R, C, N, T, B, D = (c[n] for n in ("rows", "cols", "n", "T", "B", "D"))
    s = {"case": c}
    if k in ("norm", "project"):
        # activations with a few wide channels, as residual streams have them
        spread = torch.exp(0.7 * _normal(g, C))
        s["x"] = (_normal(g, R, C) * spread).to(dt)
        s["residual"] = (2 * _normal(g, R, C) * spread).to(dt) if c["residual"] else None
        s["gain"] = 1 + 0.2 * _normal(g, C)
        if c["train"]:
            s["grad_y"] = (1e-3 * _normal(g, R, C)).to(dt)
            s["grad_h"] = (1e-3 * _normal(g, R, C)).to(dt) if c["residual"] else None
    if k == "product":
        s["x"] = ((_uniform(g, 0, 1, R, C) < 0.1).to(dt) if c["spikes"] else _normal(g, R, C).to(dt))
        s["bias"] = _normal(g, N)
    if k in ("project", "product", "input_grad"):
        w = _normal(g, N, C) / math.sqrt(C)
        s["w"] = _to_8bit(w.t().contiguous() if k == "input_grad" else w, tiles=True)
    if k in ("input_grad", "weight_grad"):
        # gradients whose size differs from token to token
        s["grad"] = (1e-3 * _normal(g, R, N) * torch.exp(_normal(g, R, 1))).to(dt)
    if k == "weight_grad":
        s["x8"] = _to_8bit(_normal(g, R, C) * torch.exp(0.7 * _normal(g, C)))
    if k in ("scan", "scan_train"):
        # gates and values come from one product; leaks from 0.5 to nearly 1, one range per channel
        both = _normal(g, T, B, 2 * D)
        both[:, :, :D] += _uniform(g, 0, 7, D)
        s["both"] = both.to(dt)
        s["h0"] = _normal(g, B, D)
        s["lengths"] = None
        if c["ragged"]:
            lengths = (_uniform(g, 0, 1, B) * (T + 1)).to(torch.int32).clamp(0, T)
            lengths[0] = T
            s["lengths"] = lengths
        if k == "scan_train":
            s["grad_out"] = (1e-2 * _normal(g, T, B, D)).to(dt)
            s["grad_h_last"] = 1e-2 * _normal(g, B, D)
    if k == "step":
        both = _normal(g, B, 2 * D)
        both[:, :D] += _uniform(g, 0, 7, D)
        s["both"] = both.to(dt)
        s["pool"] = _normal(g, c["slots"], D)
        s["slots"] = torch.randperm(c["slots"], generator=g, device=DEVICE)[:B].to(torch.int32)
    return s


# ---- one pass ----------------------------------------------------------------------------------

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_2603_13810_amd import api
    c = s["case"]
    k, dt = c["kind"], DTYPES[c["dtype"]]
    if k == "norm":
        r = api.tac_residual_norm(s["x"], s["residual"], s["gain"], eps=EPS, want_rstd=c["train"])
        out = {"y": r["y"], "h": r["h"]}
        if c["train"]:
            h = r["h"] if c["residual"] else s["x"]
            out.update(api.tac_residual_norm_backward(h, s["gain"], r["rstd"], s["grad_y"], s["grad_h"]))
        return out
    if k == "project":
        r = api.tac_residual_norm(s["x"], s["residual"], s["gain"], eps=EPS, want_y=False, want_scaled=True)
        return {"out": api.tac_scaled_product(*r["scaled"], *s["w"], c["cols"], dtype=dt), "h": r["h"]}
    if k == "product":
        a = api.tac_quantize(s["x"])["rows"]
        return api.tac_scaled_product(*a, *s["w"], c["cols"], bias=s["bias"], dtype=dt)
    if k == "input_grad":
        a = api.tac_quantize(s["grad"])["rows"]
        return api.tac_scaled_product(*a, *s["w"], c["n"], dtype=dt)
    if k == "weight_grad":
        a = api.tac_quantize(s["grad"], rows=False, columns=True)["columns"]
        b = api.tac_quantize(s["x8"], cols=c["cols"], rows=False, columns=True)["columns"]
        return api.tac_scaled_product(*a, *b, c["rows"], dtype=torch.float32)
    D = c["D"]
    gate, value = s["both"][..., :D], s["both"][..., D:]
    if k == "step":
        return {"out": api.tac_gated_step(gate, value, s["pool"], s["slots"]), "pool": s["pool"]}
    train = k == "scan_train"
    r = api.tac_gated_scan(gate, value, lengths=s["lengths"], h0=s["h0"], want_states=train)
    if train:
        both = torch.empty_like(s["both"])
        g = api.tac_gated_scan_backward(gate, value, r["states"], s["grad_out"], lengths=s["lengths"],
                                        grad_h_last=s["grad_h_last"], grad_gate=both[..., :D], grad_value=both[..., D:])
        return {"out": r["out"], "h_last": r["h_last"], "grad_both": both, "grad_h0": g["grad_h0"]}
    return {"out": r["out"], "h_last": r["h_last"]}


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t from h = 0 along the first axis, in log2(T) steps of doubled reach."""
    reach, T = 1, a.shape[0]
    while reach < T:
        b = torch.cat([b[:reach], b[reach:] + a[reach:] * b[:-reach]])
        a = torch.cat([a[:reach], a[reach:] * a[:-reach]])
        reach *= 2
    return b


def _run_plain(s):
    c = s["case"]
    k, dt = c["kind"], DTYPES[c["dtype"]]
    if k in ("norm", "project"):
        total = s["x"].float()
        if s["residual"] is not None:
            total = total + s["residual"].float()
        rstd = torch.rsqrt(total.square().mean(1, keepdim=True) + EPS)
        y = total * rstd * s["gain"]
        h = total.to(dt) if s["residual"] is not None else None
        if k == "project":
            q = _from_8bit(*_to_8bit(y), c["cols"])
            return {"out": (q @ _from_8bit(*s["w"], c["cols"]).t()).to(dt), "h": h}
        out = {"y": y.to(dt), "h": h}
        if c["train"]:
            n = (h if h is not None else s["x"]).float() * rstd
            gy = s["grad_y"].float()
            w = gy * s["gain"]
            gx = rstd * (w - n * (w * n).mean(1, keepdim=True))
            if s["grad_h"] is not None:
                gx = gx + s["grad_h"].float()
            out.update(grad_x=gx.to(dt), grad_gain=(gy * n).sum(0))
        return out
    if k == "product":
        return (_from_8bit(*_to_8bit(s["x"].float()), c["cols"]) @ _from_8bit(*s["w"], c["cols"]).t() + s["bias"]).to(dt)
    if k == "input_grad":
        return (_from_8bit(*_to_8bit(s["grad"].float()), c["n"]) @ _from_8bit(*s["w"], c["n"]).t()).to(dt)
    if k == "weight_grad":
        gt = _from_8bit(*_to_8bit(s["grad"].float().t().contiguous()), c["rows"])
        x = _from_8bit(*s["x8"], c["cols"])
        xt = _from_8bit(*_to_8bit(x.t().contiguous()), c["rows"])
        return gt @ xt.t()
    D = c["D"]
    a, keep, u = torch.sigmoid(s["both"][..., :D].float()), torch.sigmoid(-s["both"][..., :D].float()), s["both"][..., D:].float()
    if k == "step":
        at = s["slots"].long()
        h = a * s["pool"][at] + keep * u
        s["pool"][at] = h
        return {"out": h.to(dt), "pool": s["pool"]}
    T, one = c["T"], torch.ones((), device=DEVICE)
    live = None
    if s["lengths"] is not None:
        live = (torch.arange(T, device=DEVICE)[:, None] < s["lengths"][None, :])[:, :, None]
    a_live = a if live is None else torch.where(live, a, one)
    b = keep * u if live is None else torch.where(live, keep * u, 0 * one)
    b = torch.cat([s["h0"][None], b])
    h = _scan(torch.cat([one.expand(1, *a.shape[1:]), a_live]), b)
    out = {"out": (h[1:] if live is None else torch.where(live, h[1:], 0 * one)).to(dt), "h_last": h[-1].clone()}
    if k == "scan_train":
        gy = s["grad_out"].float() if live is None else torch.where(live, s["grad_out"].float(), 0 * one)
        # c_t = gy_t + a_{t+1} c_{t+1} with c_{T+1} = the last state's gradient and a_{T+1} = 1
        b = torch.cat([s["grad_h_last"][None], gy.flip(0)])
        m = torch.cat([one.expand(2, *a.shape[1:]), a_live[1:].flip(0)])
        cot = _scan(m, b)[1:].flip(0)
        gv = keep * cot
        gg = cot * (h[:-1] - u) * a * keep
        if live is not None:
            gv, gg = torch.where(live, gv, 0 * one), torch.where(live, gg, 0 * one)
        out.update(grad_both=torch.cat([gg, gv], 2).to(dt), grad_h0=a_live[0] * cot[0])
    return out


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _rounded_8bit(v, axis):
    """What a float64 matrix becomes in 8 bits with blocks of 128 along `axis`: the nearest multiples of the e4m3 spacing
    at each value, in units of the block's power of two."""
    if axis == 0:
        return _rounded_8bit(v.t(), 1).t()
    R, C = v.shape
    room = torch.zeros((R, -(-C // 128) * 128), dtype=torch.float64, device=v.device)
    room[:, :C] = v
    room = room.reshape(R, -1, 128)
    top = room.abs().amax(2, keepdim=True)
    unit = torch.exp2(torch.ceil(torch.log2((top / 448).clamp_min(2.0 ** -127))))
    unit = torch.where(top > 448 * unit, 2 * unit, torch.where(top <= 224 * unit, (unit / 2).clamp_min(2.0 ** -127), unit))
    r = room / unit
    spacing = torch.exp2((torch.frexp(r)[1] - 1).clamp_min(-6).double() - 3)
    return (torch.round(r / spacing) * spacing * unit).reshape(R, -1)[:, :C]


def _values_64(m, cols):
    """An 8-bit matrix decoded bit by bit: sign, four exponent bits (bias 7), three mantissa bits; times the scale."""
    q, scales = m
    q = q.to(torch.int64)
    e, f = (q >> 3) & 15, (q & 7).double()
    v = torch.where(e == 0, f * 2.0 ** -9, (8 + f) * torch.exp2(e.double() - 10))
    v = torch.where(q >= 128, -v, v)
    return (v * torch.exp2(scales.double() - 127).repeat_interleave(128, 1)[:, :v.shape[1]])[:, :cols]


def exact(c, seed):
    s, k, dt = prepare(c, seed), c["kind"], DTYPES[c["dtype"]]
    if k in ("norm", "project"):
        x = s["x"].double()
        if c["residual"]:
            x += s["residual"].double()
        inv = 1 / torch.sqrt((x * x).sum(1, keepdim=True) / c["cols"] + EPS)
        y = x * inv * s["gain"].double()
        h = x if c["residual"] else None
        if k == "project":
            return {"out": _rounded_8bit(y, 1) @ _values_64(s["w"], c["cols"]).t(), "h": h}
        out = {"y": y, "h": h}
        if c["train"]:
            kept = x.to(dt).double()           # the backward pass reads the stream as it was stored
            gy = s["grad_y"].double()
            inner = (gy * s["gain"].double() * kept).sum(1, keepdim=True) / c["cols"]
            gx = inv * gy * s["gain"].double() - inv ** 3 * kept * inner
            out["grad_x"] = gx + s["grad_h"].double() if c["residual"] else gx
            out["grad_gain"] = (gy * kept * inv).sum(0)
        return out
    if k == "product":
        return _rounded_8bit(s["x"].double(), 1) @ _values_64(s["w"], c["cols"]).t() + s["bias"].double()
    if k == "input_grad":
        return _rounded_8bit(s["grad"].double(), 1) @ _values_64(s["w"], c["n"]).t()
    if k == "weight_grad":
        return _rounded_8bit(s["grad"].double(), 0).t() @ _rounded_8bit(_values_64(s["x8"], c["cols"]), 0)
    D = c["D"]
    g, u = s["both"][..., :D].double(), s["both"][..., D:].double()
    a, rest = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    if k == "step":
        # run() goes on from the states as they are, pass after pass; the first pass has these values
        at = s["slots"].long()
        h = a * s["pool"].double()[at] + rest * u
        pool = s["pool"].double()
        pool[at] = h
        return {"out": h, "pool": pool}
    T = c["T"]
    lengths = s["lengths"].long() if c["ragged"] else torch.full((c["B"],), T, dtype=torch.int64, device=DEVICE)
    before, out, h = torch.empty_like(u), torch.zeros_like(u), s["h0"].double()
    for t in range(T):
        before[t] = h
        new = a[t] * h + rest[t] * u[t]
        if c["ragged"]:
            on = (lengths > t)[:, None]
            h = torch.where(on, new, h)
            out[t] = torch.where(on, new, 0.0)
        else:
            h = out[t] = new
    result = {"out": out, "h_last": h.clone()}
    if k == "scan_train":
        both, back = torch.zeros(s["both"].shape, dtype=torch.float64, device=DEVICE), s["grad_h_last"].double()
        for t in range(T - 1, -1, -1):
            here = back + s["grad_out"][t].double()
            on = (lengths > t)[:, None]
            both[t, :, :D] = torch.where(on, here * (before[t] - u[t]) * a[t] * rest[t], 0.0)
            both[t, :, D:] = torch.where(on, here * rest[t], 0.0)
            back = torch.where(on, here * a[t], back)
        result.update(grad_both=both, grad_h0=back)
    return result
