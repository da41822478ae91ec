"""Products of 8-bit integers and activations kept in 8 bits, as timed cases.

  linear   z = s[t] sw[j] (q . w8[j]) + bias, y = act(z) * mul + residual: q, s the tokens x in 8 bits with a scale each
           (s = max|x| / 127), w8 [d_out, d_in] and sw a frozen weight in 8 bits with a scale for each output channel
  back     dx of that: dy sw in 8 bits with a scale for each token, times w8 (+ a gradient that is there already)
  down     SwiGLU of gu = [gate | up], its hidden activations (bf16) in 8 bits for the linear that follows
  swiglu   a training step's SwiGLU: h = silu(gate) up, gate and up kept in 8 bits (32 columns share an exponent), and
           the gradients [dgate | dup] from what was kept
  epilogue the backward of y = act(z) * mul (+ a bias in z) from a z and a mul that were kept in 8 bits

`own` chooses between the plain forms below (32-bit torch operations, 64-bit where codes are rounded) and the framework's calls.
"""
import math

import torch

own = False
DEV = "cuda"
_ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def _linear(name, tokens, d_in, d_out, act="none", bias=False, mul=False, residual=False, keep_z=False, bf16=True):
    return dict(name=name, kind="linear", tokens=tokens, d_in=d_in, d_out=d_out, act=act, bias=bias, mul=mul, residual=residual,
                keep_z=keep_z, bf16=bf16)


def _back(name, tokens, d_in, d_out, residual, bf16):
    return dict(name=name, kind="back", tokens=tokens, d_in=d_in, d_out=d_out, residual=residual, bf16=bf16)


def _down(name, tokens, cols, d_out, residual):
    return dict(name=name, kind="down", tokens=tokens, cols=cols, d_out=d_out, residual=residual)


def _swiglu(name, tokens, cols):
    return dict(name=name, kind="swiglu", tokens=tokens, cols=cols)


def _epilogue(name, tokens, cols, act, mul, bias):
    return dict(name=name, kind="epilogue", tokens=tokens, cols=cols, act=act, mul=mul, bias=bias)


def listed():
    return [
        # One decoded token through the gate of a 65B MLP: the weight is read once, the up half is at hand.
        _linear("decode_gate", 1, 8192, 22016, act="silu", mul=True),
        # A small biased layer, sixteen sequences at once, fp32 out: the smallest call, where launches count.
        _linear("decode_small", 16, 1024, 1024, act="gelu", bias=True, residual=True, bf16=False),
        # An odd count of tokens in serving: between decode and prompt.
        _linear("serve_ragged", 61, 5120, 13824, act="gelu_tanh", bias=True),
        # The gate of a 7B MLP block in fine-tuning, 4096 tokens: z is kept for the backward.
        _linear("train_gate", 4096, 4096, 11008, act="silu", mul=True, keep_z=True),
        # The gradient through a small layer on a short sequence.
        _back("back_small", 64, 1024, 1024, False, False),
        # The gradient through the gate of train_gate, added to the up projection's.
        _back("back_gate", 4096, 4096, 11008, True, True),
        # Four decoded sequences through SwiGLU and the down projection of a 65B MLP onto the residual stream.
        _down("down_decode", 4, 22016, 8192, True),
        # A prompt of odd length through those of a 13B MLP.
        _down("down_prompt", 1531, 13824, 5120, True),
        # A training step's SwiGLU of a small block: launches count.
        _swiglu("swiglu_small", 64, 1024),
        # ... of a 7B MLP block at a 4096-token batch.
        _swiglu("swiglu_block", 4096, 11008),
        # The backward of a small biased layer's epilogue.
        _epilogue("epilogue_small", 64, 1024, "gelu", False, True),
        # The backward of a gated layer's epilogue on an odd batch, with the gradient of its bias.
        _epilogue("epilogue_ragged", 1531, 13824, "silu", True, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mult(rng, lo, hi, unit):
    return max(lo, _log(rng, lo, hi) // unit * unit)


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "linear", "back", "back", "down", "swiglu", "epilogue"])
    if kind in ("swiglu", "epilogue"):
        while True:
            tokens, cols = _log(rng, 1, 4096), _mult(rng, 256, 22016, 8)
            if 16384 <= tokens * cols <= 4096 * 11008:
                break
        if kind == "swiglu":
            c = _swiglu("", tokens, cols)
        else:
            c = _epilogue("", tokens, cols, rng.choice(_ACTS[1:]), rng.random() < 0.5, rng.random() < 0.6)
    else:
        while True:
            tokens, d_in = _log(rng, 1, 4096), _mult(rng, 512, 22016, rng.choice([16, 64, 128]))
            d_out = _mult(rng, 512, 22016, rng.choice([8, 64, 128]))
            if tokens * d_in * d_out <= 4096 * 4096 * 11008 and d_in * d_out <= 8192 * 22016:
                break
        if kind == "back":
            c = _back("", tokens, d_in, d_out, rng.random() < 0.4, rng.random() < 0.7)
        elif kind == "down":
            c = _down("", tokens, d_in, d_out, rng.random() < 0.7)
        else:
            c = _linear("", tokens, d_in, d_out, rng.choice(_ACTS), rng.random() < 0.5, rng.random() < 0.4, rng.random() < 0.5,
                        rng.random() < 0.3, rng.random() < 0.7)
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(gen, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * std).to(dtype)


def _activations(gen, tokens, width, std=1.0):
    x = _normal(gen, (tokens, width), std)
    if width >= 1000:  # a few channels are much larger than the rest
        x[:, torch.randint(0, width, (width // 1000,), generator=gen, device=DEV)] *= 20.0
    return x.to(torch.bfloat16)


def _weight(gen, d_in, d_out):
    """Codes [d_out, d_in] of weights ~ N(0, 0.02) and the channels' scales, as a model in 8 bits holds them."""
    codes = torch.randn((d_out, d_in), generator=gen, device=DEV)
    top = codes.abs().amax(1, keepdim=True)
    codes = codes.mul_(127.0 / top).round_().to(torch.int8)
    return codes, (top[:, 0] * (0.02 / 127.0)).contiguous()


def prepare(case, seed):
    gen, kind, T = _gen(seed), case["kind"], case["tokens"]
    st = {"case": case}
    if kind in ("swiglu", "epilogue"):
        C = case["cols"]
        if kind == "swiglu":
            st["gu"] = _activations(gen, T, 2 * C)
            st["dh"] = _normal(gen, (T, C), 1.0, torch.bfloat16)
        else:
            st["z"] = _activations(gen, T, C, 1.5)
            st["mul"] = _normal(gen, (T, C), 1.0, torch.bfloat16) if case["mul"] else None
            st["dy"] = _normal(gen, (T, C), 1.0, torch.bfloat16)
        return st
    d_in, d_out = case["cols"] if kind == "down" else case["d_in"], case["d_out"]
    st["w8"], st["sw"] = _weight(gen, d_in, d_out)
    if kind == "down":
        st["gu"] = _activations(gen, T, 2 * d_in)
        st["residual"] = _normal(gen, (T, d_out), 1.0, torch.bfloat16) if case["residual"] else None
        return st
    narrow = torch.bfloat16 if case["bf16"] else torch.float32
    if kind == "back":
        st["dy"] = _activations(gen, T, d_out)
        st["residual"] = _normal(gen, (T, d_in), 1.0, narrow) if case["residual"] else None
        return st
    st["x"] = _activations(gen, T, d_in)
    st["bias"] = _normal(gen, (d_out,), 0.5) if case["bias"] else None
    st["mul"] = _normal(gen, (T, d_out), 1.0, torch.bfloat16) if case["mul"] else None
    st["residual"] = _normal(gen, (T, d_out), 1.0, narrow) if case["residual"] else None
    return st


# ---- one pass: the plain forms ------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z * math.sqrt(0.5))
    if act == "gelu_tanh":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * torch.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = 2 * math.sqrt(2 / math.pi)
        s = 1 / (1 + torch.exp(-k * (z + 0.044715 * z * z * z)))
        return s + z * s * (1 - s) * k * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _tokens8(v):
    """Whole numbers (as fp32) and a scale for each row of v (fp32).  The quotients in 64 bits: in 32 some would land on the
    border between two codes that are not there."""
    s = v.abs().amax(1, keepdim=True) / 127
    q = torch.round(v.double() / s.double()).clamp_(-127, 127)
    return torch.where(s > 0, q, torch.zeros_like(q)).float(), s


def _kept8(x):
    """What comes back of x from 8 bits: 32 neighbouring columns share the exponent of their largest magnitude."""
    T, C = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -C % 32)).view(T, -1, 32)
    k = torch.frexp(v.abs().amax(2, keepdim=True))[1].clamp(min=-125) - 7
    return torch.ldexp(torch.round(torch.ldexp(v, -k)).clamp(-127, 127), k).view(T, -1)[:, :C]


def _product(q, s, w8, sw):
    return (q @ w8.float().T) * s * sw


def _plain_linear(st):
    case = st["case"]
    z = _product(*_tokens8(st["x"].float()), st["w8"], st["sw"])
    if case["bias"]:
        z = z + st["bias"]
    y = _act(z, case["act"])
    if case["mul"]:
        y = y * st["mul"].float()
    if case["residual"]:
        y = y + st["residual"].float()
    out = {"y": y.to(torch.bfloat16 if case["bf16"] else torch.float32)}
    if case["keep_z"]:
        out["z"] = z.to(torch.bfloat16)
    return out


def _plain_back(st):
    case = st["case"]
    q, s = _tokens8(st["dy"].float() * st["sw"])
    dx = (q @ st["w8"].float()) * s
    if case["residual"]:
        dx = dx + st["residual"].float()
    return {"dx": dx.to(torch.bfloat16 if case["bf16"] else torch.float32)}


def _plain_down(st):
    C = st["case"]["cols"]
    h = (_act(st["gu"][:, :C].float(), "silu") * st["gu"][:, C:].float()).to(torch.bfloat16)
    y = _product(*_tokens8(h.float()), st["w8"], st["sw"])
    if st["case"]["residual"]:
        y = y + st["residual"].float()
    return {"y": y.to(torch.bfloat16)}


def _plain_swiglu(st):
    C = st["case"]["cols"]
    h = _act(st["gu"][:, :C].float(), "silu") * st["gu"][:, C:].float()
    g, u, dh = _kept8(st["gu"][:, :C]), _kept8(st["gu"][:, C:]), st["dh"].float()
    dgu = torch.cat([dh * u * _act_slope(g, "silu"), dh * _act(g, "silu")], 1)
    return {"h": h.to(torch.bfloat16), "dgu": dgu.to(torch.bfloat16)}


def _plain_epilogue(st):
    case = st["case"]
    z, dy = _kept8(st["z"]), st["dy"].float()
    dz = dy * _act_slope(z, case["act"])
    out = {}
    if case["mul"]:
        dz = dz * _kept8(st["mul"])
        out["dmul"] = (dy * _act(z, case["act"])).to(torch.bfloat16)
    if case["bias"]:
        out["dbias"] = dz.sum(0)
    out["dz"] = dz.to(torch.bfloat16)
    return out


# ---- one pass: the framework's calls ------------------------------------------------------------

def _own_linear(st):
    from paper_2309_14717_amd import api
    case = st["case"]
    got = api.forward_int8(st["x"], st["w8"], st["sw"], bias=st["bias"], act=case["act"], mul=st["mul"], residual=st["residual"],
                           keep_z=case["keep_z"], out_dtype=torch.bfloat16 if case["bf16"] else torch.float32)
    return {"y": got[0], "z": got[1]} if case["keep_z"] else {"y": got}


def _own_back(st):
    from paper_2309_14717_amd import api
    return {"dx": api.backward_int8(st["dy"], st["w8"], st["sw"], residual=st["residual"],
                                    dx_dtype=torch.bfloat16 if st["case"]["bf16"] else torch.float32)}


def _own_down(st):
    from paper_2309_14717_amd import api
    tokens8 = api.swiglu_forward_int8(st["gu"], st["case"]["cols"])
    return {"y": api.forward_int8(tokens8, st["w8"], st["sw"], residual=st["residual"], out_dtype=torch.bfloat16)}


def _own_swiglu(st):
    from paper_2309_14717_amd import api
    C = st["case"]["cols"]
    h, kept = api.swiglu_forward_keep8(st["gu"], C)
    return {"h": h, "dgu": api.swiglu_backward_kept8(st["dh"], kept, C)}


def _own_epilogue(st):
    from paper_2309_14717_amd import api
    case = st["case"]
    z8 = api.keep8(st["z"])
    mul8 = api.keep8(st["mul"]) if case["mul"] else None
    dz, dmul, dbias = api.epilogue_backward_kept8(st["dy"], z8, case["act"], mul8=mul8, want_dbias=case["bias"])
    out = {"dz": dz}
    if case["mul"]:
        out["dmul"] = dmul
    if case["bias"]:
        out["dbias"] = dbias
    return out


def run(st):
    kind = st["case"]["kind"]
    if own:
        calls = {"linear": _own_linear, "back": _own_back, "down": _own_down, "swiglu": _own_swiglu, "epilogue": _own_epilogue}
    else:
        calls = {"linear": _plain_linear, "back": _plain_back, "down": _plain_down, "swiglu": _plain_swiglu,
                 "epilogue": _plain_epilogue}
    return calls[kind](st)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    kind, T = case["kind"], case["tokens"]
    if kind == "swiglu":  # gate, up and dh read; h, dgate and dup written
        n = T * case["cols"]
        return {"bytes": 12 * n, "flops": 24 * n}
    if kind == "epilogue":  # z and dy read, dz written; mul read and dmul written; dbias
        n = T * case["cols"]
        return {"bytes": n * (6 + (4 if case["mul"] else 0)) + (4 * case["cols"] if case["bias"] else 0), "flops": 20 * n}
    i, o = case["cols"] if kind == "down" else case["d_in"], case["d_out"]
    nbytes, flops = i * o + 4 * o, 2 * T * i * o
    if kind == "down":
        nbytes += 4 * T * i + 2 * T * o * (2 if case["residual"] else 1)
    else:
        es = 2 if case["bf16"] else 4
        if kind == "back":
            nbytes += 2 * T * o + T * i * es * (2 if case["residual"] else 1)
        else:
            nbytes += 2 * T * i + T * o * (es + (2 if case["mul"] else 0) + (es if case["residual"] else 0) + (2 if case["keep_z"] else 0))
            nbytes += 4 * o if case["bias"] else 0
    return {"bytes": nbytes, "flops": flops}


# ---- the same in 64 bits ------------------------------------------------------------------------

def _phi(z):
    """The standard normal distribution function."""
    return 0.5 * (1 + torch.erf(z / math.sqrt(2.0)))


def _exact_act(z, act):
    """act(z) and its slope."""
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    if act == "gelu":
        return z * _phi(z), _phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 0.134145 * z ** 2)
    return z, torch.ones_like(z)


def _exact_rows(v):
    """The codes of the rows of v and their scales (stored as fp32)."""
    scale = (torch.linalg.vector_norm(v, ord=math.inf, dim=1) / 127).to(torch.float32).to(torch.float64)[:, None]
    return (v / scale.clamp(min=1e-300)).round().clamp(-127, 127), scale


def _exact_kept(x):
    """Groups of 32 columns: the largest magnitude lies in [2^e, 2^(e+1)), the step is 2^(e-6)."""
    out = x.double().clone()
    for c in range(0, x.shape[1], 32):
        part = out[:, c:c + 32]
        top = part.abs().max(1, keepdim=True).values.clamp(min=2.0 ** -126)
        step = torch.exp2(torch.floor(torch.log2(top)) - 6)
        part.copy_((part / step).round().clamp(-127, 127) * step)
    return out


def exact(case, seed):
    D, kind = torch.float64, case["kind"]
    st = prepare(case, seed)
    if kind == "swiglu":
        C, dh = case["cols"], st["dh"].to(D)
        h = _exact_act(st["gu"][:, :C].to(D), "silu")[0] * st["gu"][:, C:].to(D)
        value, slope = _exact_act(_exact_kept(st["gu"][:, :C]), "silu")
        return {"h": h, "dgu": torch.cat([dh * _exact_kept(st["gu"][:, C:]) * slope, dh * value], 1)}
    if kind == "epilogue":
        value, slope = _exact_act(_exact_kept(st["z"]), case["act"])
        dz = st["dy"].to(D) * slope * (_exact_kept(st["mul"]) if case["mul"] else 1.0)
        out = {"dz": dz}
        if case["mul"]:
            out["dmul"] = st["dy"].to(D) * value
        if case["bias"]:
            out["dbias"] = dz.sum(0)
        return out
    w, sw = st["w8"].to(D), st["sw"].to(D)
    if kind == "back":
        q, s = _exact_rows((st["dy"].to(D) * sw).to(torch.float32).to(D))
        dx = (q * s) @ w
        return {"dx": dx + st["residual"].to(D) if case["residual"] else dx}
    if kind == "down":
        C = case["cols"]
        x = (_exact_act(st["gu"][:, :C].to(D), "silu")[0] * st["gu"][:, C:].to(D)).to(torch.bfloat16)
    else:
        x = st["x"]
    q, s = _exact_rows(x.to(D))
    z = (q * s) @ w.T * sw
    if kind == "down":
        return {"y": z + st["residual"].to(D) if case["residual"] else z}
    if case["bias"]:
        z = z + st["bias"].to(D)
    y = _exact_act(z, case["act"])[0]
    if case["mul"]:
        y = y * st["mul"].to(D)
    if case["residual"]:
        y = y + st["residual"].to(D)
    return {"y": y, "z": z} if case["keep_z"] else {"y": y}
