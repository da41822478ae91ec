"""The linear with an epilogue, the epilogue's backward and the orthogonalised update, as timed cases.

  linear  z = x W~ + s (pool_g(x) A) B + bias,  y = act(z) * mul + residual  (each part optional; z kept in
          bf16 where a backward follows), W~ = alpha code + beta per group of input rows
  back    dz = dy * mul * act'(z),  dmul = dy * act(z),  dbias = sum over the tokens of dz
  muon    momentum, Newton-Schulz orthogonalisation and update of a set of matrices

`own` chooses between the plain forms below (32-bit torch operations) and the framework's calls.
"""
import math

import torch

own = False
DEV = "cuda"
_ACTS = ("none", "relu", "silu", "gelu", "gelu_tanh")


def _linear(name, tokens, d_in, d_out, bits=4, group=32, rank=0, act="none", bias=False, mul=False, residual=False,
            keep_z=False, bf16=True):
    return dict(name=name, kind="linear", tokens=tokens, d_in=d_in, d_out=d_out, bits=bits, group=group, rank=rank, act=act,
                bias=bias, mul=mul, residual=residual, keep_z=keep_z, bf16=bf16)


def _back(name, tokens, cols, act, mul, bias):
    return dict(name=name, kind="back", tokens=tokens, cols=cols, act=act, mul=mul, bias=bias)


def _muon(name, d, ff, group, rank, linears, steps=5, nesterov=True):
    return dict(name=name, kind="muon", d=d, ff=ff, group=group, rank=rank, linears=linears, steps=steps, nesterov=nesterov)


def listed():
    return [
        # One decoded token through the gate of a merged 65B MLP: the weight is read once, the up half is at hand.
        _linear("decode_gate", 1, 8192, 22016, act="silu", mul=True),
        # Three tokens (one each of three sequences) through its down projection onto a residual stream kept in fp32.
        _linear("decode_down", 3, 22016, 8192, residual=True, bf16=False),
        # A small biased layer, sixteen tokens: the smallest call, where the launch counts.
        _linear("decode_small", 16, 1024, 1024, act="gelu", bias=True, residual=True),
        # An odd count of tokens in serving, 3-bit codes: between decode and prompt.
        _linear("serve_int3", 61, 5120, 13824, bits=3, group=64, act="gelu_tanh", bias=True),
        # A small adapted layer on a short sequence.
        _linear("train_small", 64, 1024, 1024, rank=16, act="silu", mul=True, keep_z=True),
        # An odd batch through an adapted 2-bit layer with bias and residual.
        _linear("train_ragged", 1531, 5120, 13824, bits=2, group=128, rank=64, act="relu", bias=True, residual=True, keep_z=True),
        # The gate of a 7B MLP block in fine-tuning, 4096 tokens: z is kept for the backward.
        _linear("train_gate", 4096, 4096, 11008, rank=64, act="silu", mul=True, keep_z=True),
        # The backward of a small layer's epilogue: launches count.
        _back("back_small", 64, 1024, "gelu_tanh", False, True),
        # The backward of train_gate's, with the gradient of a bias too.
        _back("back_gate", 4096, 11008, "silu", True, True),
        # The two matrices of one small adapter.
        _muon("muon_one", 1024, 1024, 32, 16, 1),
        # The fourteen adapter matrices of a 7B decoder layer at the paper's rank.
        _muon("muon_layer", 4096, 11008, 32, 64, 7),
        # Those of a 65B layer at the largest rank a layer can have.
        _muon("muon_wide", 8192, 22016, 32, 128, 7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _mult(rng, lo, hi, unit):
    return max(lo, _log(rng, lo, hi) // unit * unit)


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear", "linear", "back", "muon", "muon"])
    group = rng.choice([32, 32, 64, 128])
    if kind == "back":
        while True:
            tokens, cols = _log(rng, 1, 4096), _mult(rng, 256, 22016, 8)
            if 16384 <= tokens * cols <= 4096 * 11008:
                break
        c = _back("", tokens, cols, rng.choice(_ACTS[1:]), rng.random() < 0.5, rng.random() < 0.5)
    elif kind == "muon":
        c = _muon("", _mult(rng, 512, 8192, 128), _mult(rng, 1024, 22016, 128), group, rng.choice([4, 8, 16, 32, 48, 64, 64, 96, 128]),
                  rng.choice([1, 3, 7, 7]), rng.choice([3, 5, 5, 6]), rng.random() < 0.7)
    else:
        bits = rng.choice([4, 4, 4, 3, 2])
        rank = rng.choice([0, 0, 8, 16, 64, 128])
        while True:
            tokens, d_in = _log(rng, 1, 4096), _mult(rng, 512, 22016, 128)
            d_out = _mult(rng, 512, 22016, rng.choice([8, 64, 128]))
            if tokens * d_in * d_out <= 4096 * 4096 * 11008 and d_in * d_out <= 8192 * 22016:
                break
        # fp32 outputs where the weights' factors are exact (few tokens of a merged layer); longer batches rebuild the
        # weights with eleven bits
        exact_factors = rank == 0 and tokens <= (32 if bits == 4 else 16)
        c = _linear("", tokens, d_in, d_out, bits, group, rank, rng.choice(_ACTS), rng.random() < 0.5, rng.random() < 0.4,
                    rng.random() < 0.5, rank > 0 and rng.random() < 0.7, not (exact_factors and rng.random() < 0.5))
    del c["name"]
    return c


# ---- inputs -------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(gen, shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32) * std).to(dtype)


def _words(codes, width, rows):
    """Codes of `width` bits, `rows` consecutive input rows of a column to a 32-bit word: even rows in the low half, odd
    rows in the high one."""
    p = torch.arange(rows, device=DEV)
    at = (width * (p // 2) + 16 * (p % 2)).view(1, rows, 1)
    w = (codes.view(-1, rows, codes.shape[1]).long() << at).sum(1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _packed(codes, bits):
    """The library's packed codes (3 bits: the low two bits of all codes, then the high ones)."""
    if bits == 3:
        return torch.cat([_words(codes & 3, 2, 16).view(-1), _words(codes >> 2, 1, 32).view(-1)])
    return _words(codes, bits, 32 // bits).view(-1)


def _linear_inputs(case, seed):
    gen, T, i, o, g = _gen(seed), case["tokens"], case["d_in"], case["d_out"], case["group"]
    x = _normal(gen, (T, i))
    if i >= 1000:  # a few channels are much larger than the rest
        x[:, torch.randint(0, i, (i // 1000,), generator=gen, device=DEV)] *= 20.0
    top = 2 ** case["bits"] - 1
    st = {"case": case, "x": x.to(torch.bfloat16),
          "codes": torch.randint(0, top + 1, (i, o), generator=gen, device=DEV, dtype=torch.uint8)}
    # steps and minima of groups of weights ~ N(0, 0.02)
    st["alpha"] = (0.067 + 0.034 * torch.rand((i // g, o), generator=gen, device=DEV)) / top
    st["beta"] = -0.5 * top * st["alpha"] + _normal(gen, (i // g, o), 0.003)
    r, narrow = case["rank"], torch.bfloat16 if case["bf16"] else torch.float32
    st["A"] = _normal(gen, (i // g, r), 0.02) if r else None
    st["B"] = _normal(gen, (r, o), 0.02) if r else None
    st["bias"] = _normal(gen, (o,), 0.5) if case["bias"] else None
    st["mul"] = _normal(gen, (T, o), 1.0, torch.bfloat16) if case["mul"] else None
    st["residual"] = _normal(gen, (T, o), 1.0, narrow) if case["residual"] else None
    return st


def _back_inputs(case, seed):
    gen, shape = _gen(seed), (case["tokens"], case["cols"])
    st = {"case": case, "dy": _normal(gen, shape, 1.0, torch.bfloat16), "z": _normal(gen, shape, 1.5, torch.bfloat16)}
    st["mul"] = _normal(gen, shape, 1.0, torch.bfloat16) if case["mul"] else None
    return st


def _shapes(case):
    """A [d_in / g, r] and B [r, d_out] of a layer's linears: q, k, v, o, gate, up, down, as many as asked for."""
    d, f, r = case["d"], case["ff"], case["rank"]
    of = [(d, f), (f, d), (d, f), (d, d), (d, d), (d, d), (d, d)][: case["linears"]]
    return [s for i, o in of for s in ((i // case["group"], r), (r, o))]


def _muon_inputs(case, seed):
    """Gradients of adapters: a few strong directions over noise; momentum of the same kind."""
    gen = _gen(seed)

    def gradient(shape):
        k = max(1, min(shape) // 4)
        strong = (_normal(gen, (shape[0], k)) * 0.7 ** torch.arange(k, device=DEV)) @ _normal(gen, (k, shape[1]))
        return 1e-3 * strong + _normal(gen, shape, 2e-4)

    shapes = _shapes(case)
    return {"case": case, "p": [_normal(gen, s, 0.02) for s in shapes], "g": [gradient(s) for s in shapes],
            "m": [5.0 * gradient(s) for s in shapes]}


_S = 0.25  # the adapters' coefficient
_HP = dict(lr=0.01, momentum=0.95, weight_decay=0.01, eps=1e-7, a=3.4445, b=-4.7750, c=2.0315)


def _scale(shape):
    """0.2 sqrt(longer side): the step's mean square is then like AdamW's."""
    return 0.2 * math.sqrt(max(shape))


def prepare(case, seed):
    if case["kind"] == "back":
        return _back_inputs(case, seed)
    if case["kind"] == "muon":
        return _muon_inputs(case, seed)
    st = _linear_inputs(case, seed)
    st["packed"] = _packed(st["codes"], case["bits"])
    return st


# ---- one pass -----------------------------------------------------------------------------------

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


def _plain_linear(st):
    case = st["case"]
    T, i, o, g = case["tokens"], case["d_in"], case["d_out"], case["group"]
    x = st["x"].float()
    W = (st["codes"].view(i // g, g, o).float() * st["alpha"][:, None] + st["beta"][:, None]).view(i, o)
    z = x @ W
    if case["rank"]:
        z = z + _S * ((x.view(T, i // g, g).mean(2) @ st["A"]) @ st["B"])
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
    dy, z = st["dy"].float(), st["z"].float()
    dz = dy * _act_slope(z, case["act"])
    out = {}
    if case["mul"]:
        dz = dz * st["mul"].float()
        out["dmul"] = (dy * _act(z, case["act"])).to(torch.bfloat16)
    if case["bias"]:
        out["dbias"] = dz.sum(0)
    out["dz"] = dz.to(torch.bfloat16)
    return out


def _plain_orthogonal(u, steps):
    wide = u if u.shape[0] <= u.shape[1] else u.T
    X = wide / (torch.sqrt((wide * wide).sum()) + _HP["eps"])
    for _ in range(steps):
        G = X @ X.T
        X = _HP["a"] * X + (_HP["b"] * G + _HP["c"] * (G @ G)) @ X
    return X if u.shape[0] <= u.shape[1] else X.T


def _plain_muon(st):
    case = st["case"]
    for p, g, m in zip(st["p"], st["g"], st["m"]):
        m.mul_(_HP["momentum"]).add_(g)
        u = g + _HP["momentum"] * m if case["nesterov"] else m
        O = _plain_orthogonal(u, case["steps"])
        p.mul_(1 - _HP["lr"] * _HP["weight_decay"]).sub_(_HP["lr"] * _scale(p.shape) * O)
    return {"p": st["p"], "m": st["m"]}


def _own_linear(st):
    from paper_2309_14717_amd import api
    case = st["case"]
    desc = api.make_desc(case["d_in"], case["d_out"], case["bits"], case["group"], case["rank"], _S)
    got = api.forward_epilogue(desc, st["x"], st["packed"], st["alpha"], st["beta"], st["A"], st["B"], bias=st["bias"],
                               act=case["act"], mul=st["mul"], residual=st["residual"], keep_z=case["keep_z"],
                               out_dtype=torch.bfloat16 if case["bf16"] else torch.float32)
    return {"y": got[0], "z": got[1]} if case["keep_z"] else {"y": got}


def _own_back(st):
    from paper_2309_14717_amd import api
    case = st["case"]
    dz, dmul, dbias = api.epilogue_backward(st["dy"], st["z"], case["act"], mul=st["mul"], want_dbias=case["bias"])
    out = {"dz": dz}
    if case["mul"]:
        out["dmul"] = dmul
    if case["bias"]:
        out["dbias"] = dbias
    return out


def _own_muon(st):
    from paper_2309_14717_amd import api
    case = st["case"]
    hp = api.Muon(scale_mode=api.MUON_SCALE_RMS, steps=case["steps"], nesterov=case["nesterov"], **_HP)
    api.muon_step(hp, st["p"], st["g"], st["m"])
    return {"p": st["p"], "m": st["m"]}


def run(st):
    kind = st["case"]["kind"]
    if own:
        return _own_linear(st) if kind == "linear" else _own_back(st) if kind == "back" else _own_muon(st)
    return _plain_linear(st) if kind == "linear" else _plain_back(st) if kind == "back" else _plain_muon(st)


# ---- what a pass cannot do without --------------------------------------------------------------

def work(case):
    if case["kind"] == "back":
        n = case["tokens"] * case["cols"]
        # dy and z read, dz written; mul read and dmul written; dbias
        return {"bytes": n * (6 + (4 if case["mul"] else 0)) + (4 * case["cols"] if case["bias"] else 0), "flops": 16 * n}
    if case["kind"] == "muon":
        nbytes = flops = 0
        for rows, cols in _shapes(case):
            r, n = min(rows, cols), max(rows, cols)
            nbytes += 20 * r * n  # p, g, m read; p, m written
            # of a step: half of a symmetric X X^T, half of its square, and the product with X
            flops += case["steps"] * (r * r * n + r * r * r + 2 * r * r * n) + 6 * r * n
        return {"bytes": nbytes, "flops": flops}
    T, i, o, g, r = (case[k] for k in ("tokens", "d_in", "d_out", "group", "rank"))
    es = 2 if case["bf16"] else 4
    nbytes = i * o * case["bits"] / 8 + 8 * (i // g) * o + 4 * r * (i // g + o) + 2 * T * i
    nbytes += T * o * (es + (2 if case["mul"] else 0) + (es if case["residual"] else 0) + (2 if case["keep_z"] else 0))
    nbytes += 4 * o if case["bias"] else 0
    return {"bytes": nbytes, "flops": 2 * T * i * o + 2 * T * r * (i // g + o)}


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


def _exact_muon(case, seed):
    """The first pass on a new state.  The iteration acts on the singular values alone: with G = Q diag(l) Q^T its result is
    Q diag(f(sqrt l) / sqrt l) Q^T X0, f the polynomial a t + b t^3 + c t^5 applied `steps` times."""
    hp = {k: float(torch.tensor(v, dtype=torch.float32)) for k, v in _HP.items()}
    st = _muon_inputs(case, seed)
    out = {"p": [], "m": []}
    for p, g, m in zip(st["p"], st["g"], st["m"]):
        p, g, m = p.double(), g.double(), m.double()
        m = hp["momentum"] * m + g
        u = g + hp["momentum"] * m if case["nesterov"] else m
        X = (u.T if u.shape[0] > u.shape[1] else u) / (torch.linalg.norm(u) + hp["eps"])
        lam, Q = torch.linalg.eigh((X @ X.T).cpu())
        # t -> a t + b t^3 + c t^5 on t = sqrt(lam), as the factor q with t_k = q sqrt(lam)
        lam, q = lam.clamp(min=0), torch.ones_like(lam)
        for _ in range(case["steps"]):
            t2 = q * q * lam
            q = q * (hp["a"] + hp["b"] * t2 + hp["c"] * t2 * t2)
        O = ((Q * q) @ Q.T).to(DEV) @ X
        O = O.T if u.shape[0] > u.shape[1] else O
        out["p"].append(p * (1 - hp["lr"] * hp["weight_decay"]) - hp["lr"] * _scale(p.shape) * O)
        out["m"].append(m)
    return out


def exact(case, seed):
    D = torch.float64
    if case["kind"] == "muon":
        return _exact_muon(case, seed)
    if case["kind"] == "back":
        st = _back_inputs(case, seed)
        value, slope = _exact_act(st["z"].to(D), case["act"])
        dz = st["dy"].to(D) * slope * (st["mul"].to(D) if case["mul"] else 1.0)
        out = {"dz": dz}
        if case["mul"]:
            out["dmul"] = st["dy"].to(D) * value
        if case["bias"]:
            out["dbias"] = dz.sum(0)
        return out
    st = _linear_inputs(case, seed)
    x, g = st["x"].to(D), case["group"]
    beta = st["beta"].to(D)
    if case["rank"]:  # the merge identity: the adapter moves the groups' minima
        beta = beta + (_S / g) * (st["A"].to(D) @ st["B"].to(D))
    W = st["codes"].to(D) * st["alpha"].to(D).repeat_interleave(g, 0)
    W += beta.repeat_interleave(g, 0)
    z = x @ W
    if case["bias"]:
        z = z + st["bias"].to(D)
    y = _exact_act(z, case["act"])[0]
    if case["mul"]:
        y = y * st["mul"].to(D)
    if case["residual"]:
        y = y + st["residual"].to(D)
    return {"y": y, "z": z} if case["keep_z"] else {"y": y}
