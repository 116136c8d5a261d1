"""Operators of a transformer's feed-forward block in the library's number format, as timed cases.

Every operator has a plain form, in elementary torch operations, and the call that a user makes of the library
(``own`` selects).  A number in the format is an int8 payload with a power-of-two exponent, value = payload * 2^s; what is
held in 8 bits is returned as those values, which bfloat16 represents exactly.

``norm_fwd``    h = x + residual, root-mean-square norm of h, payload with one exponent per row or one for the tensor.
``norm_bwd``    its gradients: of the rows (both summands) and of the gain.
``linear_fwd``  act(a w^T + bias) + residual from int8 operands, and the pre-activation z where a backward pass follows.
``linear_bwd``  gradients of the input, of the weights and of the bias; the error is rounded to int8 with one exponent.
``adamw``       one AdamW step over many tensors, states in 32 or in 8 bits, with the refreshed int8 weights.

``listed()`` holds the cases, ``draw()`` more of the same ranges, ``exact()`` the results from the definitions in 64 bits."""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_LR, _BETA1, _BETA2, _EPS, _STEP = 1e-3, 0.9, 0.999, 1e-8, 10
_NORM_EPS = 1e-6
_BLOCK = 256

# The weight tensors of the 784-256-256-10 network and of the VGG-16 stack (thirteen 3 x 3 convolutions, three fully
# connected layers on 224 x 224 images), each followed by a bias or gain of its output width.
_MLP = [784 * 256, 256, 256 * 256, 256, 256 * 10, 10]
_VGG_CHANNELS = [3, 64, 64, 128, 128, 256, 256, 256, 512, 512, 512, 512, 512, 512]
_VGG = [n for i in range(13) for n in (9 * _VGG_CHANNELS[i] * _VGG_CHANNELS[i + 1], _VGG_CHANNELS[i + 1])] + \
    [25088 * 4096, 4096, 4096 * 4096, 4096, 4096 * 1000, 1000]


def listed():
    return [
        # One token of a decoding loop: the norm in front of a projection, a launch and its latency.
        {"name": "norm_token_4096", "kind": "norm_fwd", "m": 1, "c": 4096, "type": "bf16", "residual": True, "rows": True,
         "round_mode": 0},
        # A long prompt or a training batch: the largest norm.
        {"name": "norm_8192x4096", "kind": "norm_fwd", "m": 8192, "c": 4096, "type": "bf16", "residual": True, "rows": True,
         "round_mode": 0},
        # Training with one exponent for the whole tensor, as the integer backward multiplies need it; odd sizes, float32.
        {"name": "norm_shared_2047x1000_f32", "kind": "norm_fwd", "m": 2047, "c": 1000, "type": "f32", "residual": False,
         "rows": False, "round_mode": 1},
        # The gradients of the large norm, the residual's own gradient added.
        {"name": "norm_bwd_8192x4096", "kind": "norm_bwd", "m": 8192, "c": 4096, "type": "bf16", "residual": True},
        # One token through an up projection with its activation: the weights are read once, nothing else counts.
        {"name": "linear_token_8192x4096", "kind": "linear_fwd", "m": 1, "n": 8192, "k": 4096, "type": "bf16", "act": "silu",
         "bias": True, "residual": False, "rows": True, "z": False},
        # A batch of sixteen decoding sequences through a down projection onto the residual stream.
        {"name": "linear_16x4096x4096", "kind": "linear_fwd", "m": 16, "n": 4096, "k": 4096, "type": "bf16", "act": "none",
         "bias": False, "residual": True, "rows": True, "z": False},
        # A classification layer of odd sizes with float32 results: 1000 rows, 1000 classes, rows of 777 bytes.
        {"name": "linear_1000x1000x777_f32", "kind": "linear_fwd", "m": 1000, "n": 1000, "k": 777, "type": "f32", "act": "gelu",
         "bias": True, "residual": True, "rows": True, "z": True},
        # The largest multiply of the benchmark's sweep, with everything its epilogue can do.
        {"name": "linear_8192x8192x8192", "kind": "linear_fwd", "m": 8192, "n": 8192, "k": 8192, "type": "bf16", "act": "gelu",
         "bias": True, "residual": True, "rows": False, "z": True},
        # Backward of an ordinary layer in training.
        {"name": "linear_bwd_4096x4096x1024", "kind": "linear_bwd", "m": 4096, "n": 4096, "k": 1024, "type": "bf16",
         "act": "gelu", "round_mode": 0},
        # Backward of a ragged layer in half precision: few output tiles, a contraction over the batch.
        {"name": "linear_bwd_2000x520x777_f16", "kind": "linear_bwd", "m": 2000, "n": 520, "k": 777, "type": "f16",
         "act": "relu", "round_mode": 1},
        # The optimizer on a network of six tensors with 32-bit states: one launch and its latency.
        {"name": "adamw_mlp_32", "kind": "adamw", "net": "mlp", "bits": 32, "gtype": "f32", "w8": True},
        # The optimizer on the 138 million weights of the VGG-16 stack with 8-bit states.
        {"name": "adamw_vgg16_8", "kind": "adamw", "net": "vgg16", "bits": 8, "gtype": "bf16", "w8": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over the logarithm of their range; a case above the bound is drawn again."""
    kind = rng.choice(["norm_fwd", "norm_bwd", "linear_fwd", "linear_fwd", "linear_bwd", "adamw"])
    opt = {"kind": kind} if kind == "adamw" else {"kind": kind, "round_mode": rng.choice([0, 0, 1])}
    if kind.startswith("norm"):
        while True:
            m, c = _log_int(rng, 1, 16384), _log_int(rng, 16, 16384)
            if rng.random() < 0.5:
                c = max(16, c // 16 * 16)
            if m * c <= 8192 * 4096:
                break
        case = dict(opt, m=m, c=c, type=rng.choice(["bf16", "bf16", "f16", "f32"]), residual=rng.random() < 0.6)
        if kind == "norm_fwd":
            case["rows"] = rng.random() < 0.6
        return case
    if kind == "adamw":
        count = _log_int(rng, 1, 400)
        return dict(opt, net="drawn", count=count, most=_log_int(rng, 64, min(1 << 24, (1 << 26) // count)),
                    sizes=rng.randrange(1 << 30), bits=rng.choice([8, 8, 32]), gtype=rng.choice(["bf16", "f32", "f16"]),
                    w8=rng.random() < 0.6)
    while True:
        m, n, k = _log_int(rng, 1, 8192), _log_int(rng, 16, 8192), _log_int(rng, 16, 8192)
        if rng.random() < 0.6:
            n, k = max(16, n // 16 * 16), max(16, k // 16 * 16)
        if m * n * k <= 2 ** 37 and n * k >= 4096:
            break
    case = dict(opt, m=m, n=n, k=k, type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                act=rng.choice(["none", "relu", "gelu", "silu"]))
    if kind == "linear_bwd" and case["act"] in ("gelu", "silu") and case["type"] == "f32":
        case["type"] = "bf16"             # (float32 gradients where the error that is rounded to 8 bits is exact in float32)
    if case["type"] != "f32" and case["act"] in ("none", "relu"):
        case["round_mode"] = 1            # (the error has the few bits of its type: nothing to draw a rounding from)
    if kind == "linear_fwd":
        del case["round_mode"]
        case.update(bias=rng.random() < 0.6, residual=rng.random() < 0.5, rows=rng.random() < 0.6, z=rng.random() < 0.4)
    return case


# ---- inputs ----------------------------------------------------------------------------------

_handle = None


def _niti():
    """The library's context, which a program creates once."""
    global _handle
    if _handle is None:
        from paper_2009_13108_b200 import Niti
        _handle = Niti(0)
    return _handle


def _sizes(case):
    if case["net"] == "mlp":
        return list(_MLP)
    if case["net"] == "vgg16":
        return list(_VGG)
    g = torch.Generator().manual_seed(case["sizes"])
    return [max(1, int(case["most"] * f)) for f in torch.rand(case["count"], generator=g).tolist()]


def prepare(case, seed):
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev).manual_seed(seed)
    st = {"case": case, "niti": _niti() if own else None}
    kind = case["kind"]

    def normal(*shape):
        return torch.randn(shape, device=dev, generator=g)

    def payload(rows, cols, spread):
        # int8 payloads as a norm or a weight tensor has them: bell-shaped, the widest about 127
        return (normal(rows, cols) * spread).round_().clamp_(-127, 127).to(torch.int8)

    if kind.startswith("norm"):
        m, c, t = case["m"], case["c"], _TYPES[case["type"]]
        # a residual stream: rows of different magnitude, a few channels that are larger than the others
        rows = torch.exp(0.5 * normal(m, 1))
        chan = torch.exp(0.2 * normal(1, c)).clamp(0.6, 1.4) * (1 + 1.5 * (torch.rand((1, c), device=dev, generator=g) < 0.005))
        st["gain"] = 1 + 0.1 * normal(c)
        st["x"] = (normal(m, c) * rows * chan).to(t)
        if case["residual"]:
            st["res"] = (normal(m, c) * rows * chan).to(t)
        if kind == "norm_bwd":
            h = st["x"].float()
            st["rstd"] = torch.rsqrt(h.square().mean(1) + _NORM_EPS)
            st["dy"] = (1e-3 * normal(m, c)).to(t)
            if case["residual"]:
                st["res"] = (1e-3 * normal(m, c)).to(t)
    elif kind.startswith("linear"):
        m, n, k, t = case["m"], case["n"], case["k"], _TYPES[case["type"]]
        st["a"] = payload(m, k, 30.0)
        st["w"] = payload(n, k, 40.0)
        # exponents that leave outputs of order one: a has standard deviation 30 * 2^s_a, w about 1 / sqrt(k)
        rows = case.get("rows", False)
        st["s_a"] = torch.randint(-6, -3, (m,) if rows else (1,), device=dev, generator=g, dtype=torch.int32)
        st["s_w"] = torch.full((1,), -round(math.log2(40.0 * math.sqrt(k))), dtype=torch.int32, device=dev)
        if kind == "linear_fwd":
            st["bias"] = 0.1 * normal(n) if case["bias"] else None
            st["res"] = normal(m, n).to(t) if case["residual"] else None
        else:
            st["z"] = normal(m, n).to(t) if case["act"] != "none" else None
            st["dout"] = (1e-2 * normal(m, n) * torch.exp(0.5 * normal(m, 1))).to(t)
    else:
        sizes = _sizes(case)
        offs, total = [], 0
        for s in sizes:
            offs.append(total)
            total += (s + _BLOCK - 1) // _BLOCK * _BLOCK        # tensors of one allocation, each on a block boundary
        blocks = torch.tensor([(s + _BLOCK - 1) // _BLOCK for s in sizes], device=dev)
        last = torch.tensor([o + s for o, s in zip(offs, sizes)], device=dev)
        # which elements of the allocation belong to a tensor, and where in it they are
        live = torch.arange(total, device=dev) < torch.repeat_interleave(last, blocks * _BLOCK)
        if case["bits"] == 8:
            st["index"] = torch.arange(total, device=dev) - torch.repeat_interleave(torch.tensor(offs, device=dev), blocks * _BLOCK)
        st["p"] = 0.02 * normal(total) * live
        st["g"] = (1e-3 * normal(total) * live).to(_TYPES[case["gtype"]])
        m = 3e-4 * normal(total) * live
        r = (1e-3 * (0.05 + normal(total).abs())) * live
        if case["bits"] == 8:
            (st["m"], st["s_m"]), (st["v"], st["s_v"]) = _encode_states(m.view(-1, _BLOCK), r.view(-1, _BLOCK), 32768, 32768)
        else:
            st["m"], st["v"] = m, r * r
        st["step"] = torch.full((1,), _STEP, dtype=torch.int32, device=dev)
        # weight matrices decay, biases and gains do not
        decay = [0.1 if s >= 4096 else 0.0 for s in sizes]
        st["decay"] = torch.repeat_interleave(torch.tensor(decay, device=dev), blocks)[:, None]
        if case["w8"]:
            st["w8"] = torch.zeros(total, dtype=torch.int8, device=dev)
            st["s_w"] = torch.randint(-11, -9, (len(sizes),), device=dev, generator=g, dtype=torch.int32)
            st["s_w_blocks"] = torch.repeat_interleave(st["s_w"], blocks)[:, None]
        if own:
            view = lambda x: [x[o:o + s] for o, s in zip(offs, sizes)]                                     # noqa: E731
            eight = case["bits"] == 8
            scales = lambda x: [x[o // _BLOCK:(o + s + _BLOCK - 1) // _BLOCK] for o, s in zip(offs, sizes)]  # noqa: E731
            st["plan"] = st["niti"].adamw_tensors(
                view(st["p"]), view(st["g"]), view(st["m"]), view(st["v"]),
                s_m=scales(st["s_m"]) if eight else None, s_v=scales(st["s_v"]) if eight else None,
                w8=view(st["w8"]) if case["w8"] else None,
                s_w=[st["s_w"][i:i + 1] for i in range(len(sizes))] if case["w8"] else None, weight_decay=decay)
    return st


# ---- plain forms -----------------------------------------------------------------------------

def _pow2(s):
    """2^s as float32 for a tensor of exponents in [-126, 127]."""
    return ((s.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent_of(amax, bits):
    """The exponent that leaves ``bits`` integer bits to magnitudes up to amax (0 for a zero maximum)."""
    s = (torch.frexp(amax)[1] - bits).clamp(min=-100)
    return torch.where(amax == 0, torch.zeros_like(s), s).to(torch.int32)


def _round_units(u, round_mode):
    """Magnitudes in units of the result, rounded to whole ones: half up, or pseudo-stochastically from 16 fraction bits."""
    if round_mode == 1:
        return torch.floor(u + 0.5)
    v = torch.floor(u * 65536.0).to(torch.int32)
    return ((v >> 16) + (((v >> 8) & 255) > (v & 255)).to(torch.int32)).to(torch.float32)


def _payload(x, s, round_mode):
    """Payload of float32 values with exponents s, as float32 whole numbers in [-127, 127]."""
    q = _round_units(x.abs() * _pow2(-s), round_mode).clamp(max=127.0)
    return torch.where(x < 0, -q, q)


def _e4m3_units(x):
    """Of float32 blocks: block exponents, exponent fields (at least -6) and magnitudes in units of the last place."""
    s = _exponent_of(x.abs().amax(1, keepdim=True), 8)
    t = x.abs() * _pow2(-s)
    e = (torch.frexp(t)[1] - 1).clamp(min=-6)
    e = torch.where(t == 0, torch.full_like(e, -6), e)
    return s, e, t * _pow2(3 - e)


def _encode_states(m, r, t_m, t_r):
    """Codes (uint8) and block exponents (int8) of the 8-bit states, the first moment and the root of the second: rounded up
    where 16 fraction bits and 16 random ones carry.  The root does not round to zero."""
    (s_m, e_m, u_m), (s_r, e_r, u_r) = _e4m3_units(m), _e4m3_units(r)
    q_m = (torch.floor(u_m * 65536.0).to(torch.int32) + t_m) >> 16
    q_r = torch.maximum((torch.floor(u_r * 65536.0).to(torch.int32) + t_r) >> 16, (r > 0).to(torch.int32))
    code_m = ((e_m + 6) << 3) + q_m + torch.where(m < 0, 128, 0)
    code_r = ((e_r + 6) << 3) + q_r
    return [(c.to(torch.uint8).view(-1), s.to(torch.int8).view(-1)) for c, s in ((code_m, s_m), (code_r, s_r))]


def _random_bits(index, step):
    """32 bits for an element of a tensor in a step: a mixing function of both (multiplications and shifts mod 2^32)."""
    x = index ^ ((step.long() * 0x9E3779B9) & 0xFFFFFFFF)
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _decode_e4m3(code, s):
    """float32 values [blocks][256] of an 8-bit state."""
    c = code.view(-1, _BLOCK).to(torch.int32)
    field, frac = (c >> 3) & 15, c & 7
    mag = torch.where(field > 0, frac + 8, frac).to(torch.float32) * _pow2(field.clamp(min=1) - 10)
    return torch.where(c >= 128, -mag, mag) * _pow2(s.to(torch.int32))[:, None]


def _act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    s = 1 / (1 + torch.exp(-z))
    return s * (1 + z * (1 - s))


def _plain(st):
    case, kind = st["case"], st["case"]["kind"]
    if kind == "norm_fwd":
        t = _TYPES[case["type"]]
        h = st["x"].float()
        if case["residual"]:
            h = (h + st["res"].float()).to(t).float()
        rstd = torch.rsqrt(h.square().mean(1) + _NORM_EPS)
        y = h * rstd[:, None] * st["gain"]
        s = _exponent_of(y.abs().amax(1, keepdim=True) if case["rows"] else y.abs().amax().view(1, 1), 7)
        values = (_payload(y, s, case["round_mode"]) * _pow2(s)).to(torch.bfloat16)
        return {"values": values, "rstd": rstd, **({"h": h.to(t)} if case["residual"] else {})}
    if kind == "norm_bwd":
        h, dy, r = st["x"].float(), st["dy"].float(), st["rstd"][:, None]
        gdy = dy * st["gain"]
        dx = r * gdy - h * (r * r * r) * (gdy * h).mean(1, keepdim=True)
        if case["residual"]:
            dx = dx + st["res"].float()
        return {"dx": dx.to(st["dy"].dtype), "dgain": (dy * (h * r)).sum(0)}
    if kind == "linear_fwd":
        t = _TYPES[case["type"]]
        z = (st["a"].float() @ st["w"].float().t()) * _pow2(st["s_a"] + st["s_w"])[:, None]
        if st["bias"] is not None:
            z = z + st["bias"]
        out = _act(z, case["act"])
        if st["res"] is not None:
            out = out + st["res"].float()
        return {"out": out.to(t), **({"z": z.to(t)} if case["z"] else {})}
    if kind == "linear_bwd":
        e = st["dout"].float()
        if case["act"] != "none":
            e = e * _act_slope(st["z"].float(), case["act"])
        s_e = _exponent_of(e.abs().amax().view(1), 7)
        q = _payload(e, s_e, case["round_mode"])
        dx = (q @ st["w"].float()) * _pow2(s_e + st["s_w"])
        dw = (q.t() @ st["a"].float()) * _pow2(s_e + st["s_a"])
        t16 = torch.bfloat16
        return {"dx": dx.to(st["dout"].dtype), "dw": dw.to(t16), "dbias": e.sum(0)}
    eight = case["bits"] == 8
    p, g = st["p"].view(-1, _BLOCK), st["g"].view(-1, _BLOCK).float()
    t = st["step"].double()
    c1, c2 = 1 - _BETA1 ** t, 1 - _BETA2 ** t
    m = _decode_e4m3(st["m"], st["s_m"]) if eight else st["m"].view(-1, _BLOCK)
    v = _decode_e4m3(st["v"], st["s_v"]).square() if eight else st["v"].view(-1, _BLOCK)
    m = _BETA1 * m + (1 - _BETA1) * g
    v = _BETA2 * v + (1 - _BETA2) * g * g
    p.copy_(p * (1 - _LR * st["decay"]) - (_LR / c1).float() * (m / (v.sqrt() * (1 / c2.sqrt()).float() + _EPS)))
    out = {"p": st["p"]}
    if eight:
        bits = _random_bits(st["index"], st["step"]).view(-1, _BLOCK)
        for name, (code, s) in zip("mv", _encode_states(m, v.sqrt(), (bits >> 16).to(torch.int32), (bits & 65535).to(torch.int32))):
            st[name].copy_(code)
            st["s_" + name].copy_(s)
            out[name] = _decode_e4m3(code, s).to(torch.bfloat16).view(-1)
    else:
        st["m"].copy_(m.view(-1))
        st["v"].copy_(v.view(-1))
        out["m"], out["v"] = st["m"], st["v"]
    if case["w8"]:
        q = _payload(p, st["s_w_blocks"], 1)
        st["w8"].copy_(q.view(-1))
        out["w8"] = (q * _pow2(st["s_w_blocks"])).to(torch.bfloat16).view(-1)
    return out


# ---- the library's calls ---------------------------------------------------------------------

def _calls(st):
    n, case, kind = st["niti"], st["case"], st["case"]["kind"]
    if kind == "norm_fwd":
        y, s_y, h, rstd = n.rmsnorm_fwd(st["x"], st["gain"], residual=st.get("res"), rows=case["rows"], eps=_NORM_EPS,
                                        round_mode=case["round_mode"])
        values = n.dequantize(y, s_y, dtype=torch.bfloat16)
        return {"values": values, "rstd": rstd, **({"h": h} if case["residual"] else {})}
    if kind == "norm_bwd":
        dx, dgain = n.rmsnorm_bwd(st["dy"], st["x"], st["gain"], st["rstd"], dh=st.get("res"))
        return {"dx": dx, "dgain": dgain}
    if kind == "linear_fwd":
        out, z = n.linear_act_fwd(st["a"], st["s_a"], st["w"], st["s_w"], bias=st["bias"], residual=st["res"],
                                  act=case["act"], keep_z=case["z"], dtype=_TYPES[case["type"]])
        return {"out": out, **({"z": z} if case["z"] else {})}
    if kind == "linear_bwd":
        dx, dw, dbias = n.linear_act_bwd(st["a"], st["s_a"], st["w"], st["s_w"], st["dout"], z=st["z"], act=case["act"],
                                         dw_dtype=torch.bfloat16, round_mode=case["round_mode"])
        return {"dx": dx, "dw": dw, "dbias": dbias}
    n.adamw(st["plan"], st["step"], lr=_LR, betas=(_BETA1, _BETA2), eps=_EPS)
    out = {"p": st["p"], "m": st["m"], "v": st["v"]}
    if case["bits"] == 8:
        out["m"] = n.dequantize(st["m"], st["s_m"], dtype=torch.bfloat16, block=_BLOCK)
        out["v"] = n.dequantize(st["v"], st["s_v"], dtype=torch.bfloat16, block=_BLOCK)
    if case["w8"]:
        out["w8"] = n.dequantize(st["w8"].view(-1, _BLOCK), st["s_w_blocks"].view(-1), dtype=torch.bfloat16).view(-1)
    return out


def run(state):
    return _calls(state) if own else _plain(state)


def work(case):
    kind = case["kind"]
    if kind.startswith("norm"):
        n, b = case["m"] * case["c"], _TYPES[case["type"]].itemsize
        if kind == "norm_fwd":
            # x, residual, h, the values; per row the reciprocal root
            return {"bytes": n * (b * (3 if case["residual"] else 1) + 2) + 4 * (case["m"] + case["c"]), "flops": 8 * n}
        return {"bytes": n * b * (4 if case["residual"] else 3) + 4 * (case["m"] + 2 * case["c"]), "flops": 12 * n}
    if kind.startswith("linear"):
        m, n, k, b = case["m"], case["n"], case["k"], _TYPES[case["type"]].itemsize
        if kind == "linear_fwd":
            outs = 1 + case["residual"] + case["z"]
            return {"bytes": m * k + n * k + outs * m * n * b + 4 * n * case["bias"], "flops": 2 * m * n * k}
        return {"bytes": m * k + n * k + m * n * b * (2 if case["act"] != "none" else 1) + m * k * b + 2 * n * k + 4 * n,
                "flops": 4 * m * n * k}
    n = sum(_sizes(case))
    state = (2 + 4) if case["bits"] == 8 else 16          # both read; written as the values they stand for
    return {"bytes": n * (8 + _TYPES[case["gtype"]].itemsize + state + 2 * case["w8"]), "flops": 20 * n}


# ---- 64 bits ---------------------------------------------------------------------------------

def _exact_round(mag, round_mode):
    """Non-negative float64 magnitudes to whole numbers, by the definition of the two roundings."""
    whole = mag.floor()
    frac = mag - whole
    if round_mode == 1:
        return whole + (frac >= 0.5).double()
    high = (frac * 256).floor()
    low = ((frac * 256 - high) * 256).floor()
    return whole + (high > low).double()


def _exact_scale(top, integer_bits):
    """2^s with top / 2^s in [2^(integer_bits - 1), 2^integer_bits), s >= -100; 1 for a zero maximum."""
    s = top.clamp(min=1e-300).log2().floor()
    s = torch.where(torch.exp2(s) > top, s - 1, s)
    s = torch.where(torch.exp2(s + 1) <= top, s + 1, s) - (integer_bits - 1)
    return torch.where(top > 0, torch.exp2(s.clamp(min=-100.0)), torch.ones_like(top))


def _exact_states(m, r, index, step):
    """What the 8-bit states stand for: four significant bits of a value over its block's scale, steps of 2^-9 below 2^-6,
    rounded up with the probability of the remainder (by 16 random bits)."""
    x = index ^ (step * 0x9E3779B9 % 2 ** 32)
    for shift, factor in ((16, 0x7FEB352D), (15, 0x846CA68B)):
        x = x ^ torch.div(x, 2 ** shift, rounding_mode="floor")
        # (times the factor's halves, to stay within 64 bits)
        x = (x * (factor % 65536) + ((x * (factor // 65536)) % 65536) * 65536) % 2 ** 32
    x = x ^ torch.div(x, 65536, rounding_mode="floor")
    found = []
    for v, draw in ((m, torch.div(x, 65536, rounding_mode="floor")), (r, x % 65536)):
        v = v.view(-1, _BLOCK)
        scale = _exact_scale(v.abs().amax(1, keepdim=True), 8)
        t = v.abs() / scale
        unit = torch.where(t > 0, _exact_scale(t, 4).clamp(min=2.0 ** -9), torch.full_like(t, 2.0 ** -9))
        q = ((t / unit * 65536).floor() + draw.view(-1, _BLOCK).double()).div(65536).floor()
        found.append((q, unit * scale))
    (q_m, unit_m), (q_r, unit_r) = found
    q_r = torch.maximum(q_r, (r.view(-1, _BLOCK) > 0).double())
    return (torch.sign(m).view(-1, _BLOCK) * q_m * unit_m).view(-1), (q_r * unit_r).view(-1)


def _exact_state_values(code, s):
    table = torch.arange(256, device=code.device).to(torch.uint8).view(torch.float8_e4m3fn).double()
    return table[code.long()] * torch.exp2(s.double()).repeat_interleave(_BLOCK)


def exact(case, seed):
    st, kind, d = prepare(case, seed), case["kind"], torch.float64
    if kind == "norm_fwd":
        h = st["x"].to(d)
        if case["residual"]:
            h = (h + st["res"].to(d)).to(_TYPES[case["type"]]).to(d)
        rstd = (h.pow(2).sum(1) / case["c"] + _NORM_EPS).pow(-0.5)
        y = h * st["gain"].to(d)[None] * rstd[:, None]
        top = y.abs().max(1, keepdim=True).values if case["rows"] else y.abs().max().reshape(1, 1)
        scale = _exact_scale(top, 7)
        q = _exact_round(y.abs() / scale, case["round_mode"]).clamp(max=127)
        return {"values": torch.sign(y) * q * scale, "rstd": rstd, **({"h": h} if case["residual"] else {})}
    if kind == "norm_bwd":
        # with n = h r the normalised row: dx = dh + r (g dy - n mean(g dy n))
        n = st["x"].to(d) * st["rstd"].to(d)[:, None]
        dn = st["dy"].to(d) * st["gain"].to(d)
        dx = (dn - n * ((dn * n).sum(1, keepdim=True) / case["c"])) * st["rstd"].to(d)[:, None]
        if case["residual"]:
            dx += st["res"].to(d)
        return {"dx": dx, "dgain": torch.einsum("mc,mc->c", st["dy"].to(d), n)}
    if kind == "linear_fwd":
        z = torch.einsum("mk,nk->mn", st["a"].to(d), st["w"].to(d))
        z *= torch.exp2(st["s_a"].to(d) + st["s_w"].to(d))[:, None]
        if st["bias"] is not None:
            z += st["bias"].to(d)
        act = case["act"]
        out = {"none": lambda v: v, "relu": lambda v: v * (v > 0), "silu": lambda v: v * torch.sigmoid(v),
               "gelu": lambda v: v * torch.special.ndtr(v)}[act](z)
        if st["res"] is not None:
            out = out + st["res"].to(d)
        return {"out": out, **({"z": z} if case["z"] else {})}
    if kind == "linear_bwd":
        e = st["dout"].to(d)
        if case["act"] != "none":
            z = st["z"].to(d)
            if case["act"] == "relu":
                e = e * (z > 0)
            elif case["act"] == "gelu":
                e = e * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi))
            else:
                sg = torch.sigmoid(z)
                e = e * (sg + z * sg * (1 - sg))
        scale = _exact_scale(e.abs().max(), 7)
        q = torch.sign(e) * _exact_round(e.abs() / scale, case["round_mode"]).clamp(max=127)
        return {"dx": torch.einsum("mn,nk->mk", q, st["w"].to(d)) * (scale * torch.exp2(st["s_w"].to(d))),
                "dw": torch.einsum("mn,mk->nk", q, st["a"].to(d)) * (scale * torch.exp2(st["s_a"].to(d))),
                "dbias": e.sum(0)}
    eight = case["bits"] == 8
    g = st["g"].to(d)
    m = _exact_state_values(st["m"], st["s_m"]) if eight else st["m"].to(d)
    v = _exact_state_values(st["v"], st["s_v"]) ** 2 if eight else st["v"].to(d)
    m = m + (1 - _BETA1) * (g - m)
    v = v + (1 - _BETA2) * (g * g - v)
    decay = st["decay"].to(d).expand(-1, _BLOCK).reshape(-1)
    decay = torch.where(decay > 0, 0.1, 0.0).to(d)
    p = st["p"].to(d)
    p = p - _LR * decay * p - _LR * (m / (1 - _BETA1 ** _STEP)) / ((v / (1 - _BETA2 ** _STEP)).sqrt() + _EPS)
    out = {"p": p, "m": m, "v": v}
    if eight:
        out["m"], out["v"] = _exact_states(m, v.sqrt(), st["index"], _STEP)
    if case["w8"]:
        scale = torch.exp2(st["s_w_blocks"].to(d)).expand(-1, _BLOCK).reshape(-1)
        out["w8"] = torch.sign(p) * _exact_round(p.abs() / scale, 1).clamp(max=127) * scale
    return out
