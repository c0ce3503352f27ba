"""What stands between and inside the blocks of a residual network, as cases that can be timed and compared.

Four operators next to the feed-forward products:

  ``norm``      s = r + scale * gate * N_after(b),  h = N_before(s): a block's output b goes through its norm and its gate onto
                the residual stream r, and the new stream through the norm of the block that follows; and the backward pass;
  ``quantize``  a matrix in microscaled 4-bit floating point, and the values that this stands for;
  ``mx``        y = act(x w^T + bias) + residual of a 4-bit weight, x quantised on the way;
  ``moe``       a whole layer of experts for a few tokens: router, gated products of the chosen experts, their weighted sum.

With ``own`` false a pass is elementary torch operations in 32 bits, rounded once at the end (the router's sums in 64 bits, so
that the choice of experts does not hang on the order of a sum); with ``own`` true it is what a program calls in
``paper_1504_04343_amd.binding``.

Matrices have one type (fp32, bf16, fp16); their rows lie ``pad`` elements further apart than they are long, as in slices
of wider tensors.  Microscaled: 32 consecutive values of a row share a power of two, a byte that holds its exponent + 127; each
is one of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times that, 4 bits (sign, number in this list), two of them to a byte, the first in the
lower half.  A row of codes is whole blocks of 16 bytes, its scales a multiple of four bytes.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _norm(name, M, D, type, before, after, gate, backward=False, affine=False, pad=0):
    """gate: rows of the stream that share a row of the gate, 0 for no gate; affine: the norms have biases too."""
    return dict(name=name, kind="norm", M=M, D=D, type=type, before=before, after=after, gate=gate, backward=backward,
                affine=affine, pad=pad)


def _quantize(name, M, D, type, pad=0):
    return dict(name=name, kind="quantize", M=M, D=D, type=type, pad=pad)


def _mx(name, M, N, K, type, act, bias=True, residual=False, pad=0):
    return dict(name=name, kind="mx", M=M, N=N, K=K, type=type, act=act, bias=bias, residual=residual, pad=pad)


def _moe(name, T, E, k, D, F, type, act, normalize=True, residual=False, pad=0):
    return dict(name=name, kind="moe", T=T, E=E, k=k, D=D, F=F, type=type, act=act, normalize=normalize, residual=residual,
                pad=pad)


def listed():
    return [
        # serving: a single token between two blocks, norms on both sides
        _norm("norm_one_row", 1, 4096, "bf16", "rms", "rms", 1),
        # training and prompts: what most blocks have, the addition and the norm of the block that follows
        _norm("norm_forward", 8192, 4096, "bf16", "rms", "none", 0),
        # training: the backward pass of norms on both sides of a block and a gate that all tokens share
        _norm("norm_backward", 8192, 4096, "bf16", "rms", "rms", 8192, backward=True),
        # odd sizes in slices of wider tensors, layer norms with biases, a gate for each sequence of 37 tokens, in fp16
        _norm("norm_backward_odd", 1531, 2049, "f16", "layer", "layer", 37, backward=True, affine=True, pad=3),
        # weights or a large batch's activations to 4 bits
        _quantize("quantize_large", 8192, 8192, "bf16"),
        # fp32 weights of odd sizes in a wider tensor
        _quantize("quantize_odd", 1531, 2049, "f32", pad=3),
        # serving: one token through a layer whose weights are held in 4 bits
        _mx("mx_one_row", 1, 4096, 4096, "bf16", "none"),
        # serving: a batch of sequences, one token each
        _mx("mx_few_rows", 48, 16384, 4096, "f16", "silu", residual=True),
        # prompts: a large batch through the same kind of layer
        _mx("mx_large", 8192, 8192, 8192, "bf16", "gelu"),
        # serving: one token, two of sixteen wide experts
        _moe("moe_one_token", 1, 16, 2, 4096, 8192, "bf16", "silu"),
        # serving: a batch of sequences, one token each, many small experts
        _moe("moe_few_tokens", 16, 64, 4, 2048, 2048, "bf16", "silu", residual=True),
        # odd sizes, the weights of all experts' softmax
        _moe("moe_odd", 37, 24, 3, 1000, 1531, "f16", "gelu", normalize=False, pad=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A number of features: mostly round, but not always."""
    n = _log_int(rng, lo, hi)
    u = rng.random()
    return max(lo, n // 64 * 64) if u < 0.5 else max(lo, n // 8 * 8) if u < 0.7 else n


def draw(rng):
    while True:
        u = rng.random()
        type = rng.choice(["bf16", "bf16", "f16", "f32"])
        pad = rng.choice([0, 0, 0, 8, 64, 1, 5])
        if u < 0.4:
            M = _log_int(rng, 1, 16384)
            after = rng.choice(["none", "rms", "layer"])
            case = _norm("", M, _size(rng, 16, 16384), type, rng.choice(["rms", "rms", "layer"]), after,
                         rng.choice([0, M, M, 1, min(M, _log_int(rng, 2, 2048))]), rng.random() < 0.5, rng.random() < 0.4, pad)
        elif u < 0.55:
            case = _quantize("", _log_int(rng, 1, 16384), _size(rng, 16, 16384), type, pad)
        elif u < 0.8:
            case = _mx("", _log_int(rng, 1, 8192), _size(rng, 16, 16384), _size(rng, 16, 16384), type,
                       rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), rng.random() < 0.6, rng.random() < 0.4, pad)
        else:
            E = _log_int(rng, 2, 256)
            case = _moe("", _log_int(rng, 1, 64), E, min(E, rng.randrange(1, 9)), _size(rng, 32, 4096), _size(rng, 32, 8192), type,
                        rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), rng.random() < 0.7, rng.random() < 0.5, pad)
            if 3 * E * case["D"] * case["F"] * _SIZE[type] > 3.3e9:  # what all experts take
                continue
        del case["name"]
        w = work(case)
        if w["flops"] <= 1.1e12 and w["bytes"] <= 5.0e8:
            return case


# ---- what a program has in hand before the call -------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _matrix(g, rows, cols, type, std=1.0, pad=0, mean=0.0):
    """rows x cols values, rows cols + pad elements apart."""
    t = torch.empty(rows, cols + pad, dtype=_TYPES[type], device="cuda")
    t.copy_(torch.randn(t.shape, generator=g, device="cuda").mul_(std).add_(mean))
    return t[:, :cols]


def _vector(g, n, type, std=1.0, mean=0.0):
    return _matrix(g, 1, n, type, std, 0, mean).view(n)


def _empty(rows, cols, type, pad=0):
    return torch.empty(rows, cols + pad, dtype=_TYPES[type], device="cuda")[:, :cols]


_EPS, _SCALE = 1e-6, 0.5


def _norm_state(case, seed):
    g = _gen(seed)
    M, D, ty, pad = case["M"], case["D"], case["type"], case["pad"]
    groups = -(-M // case["gate"]) if case["gate"] else 0
    after, affine = case["after"] != "none", case["affine"]
    s = dict(r=_matrix(g, M, D, ty, 2.0, pad, 0.3), b=_matrix(g, M, D, ty, 1.0, pad, 0.1),
             gate=_matrix(g, groups, D, ty, 0.3, pad, 0.5) if groups else None,
             w_after=_vector(g, D, ty, 0.2, 1.0) if after else None,
             c_after=_vector(g, D, ty, 0.1) if after and affine else None,
             w_before=_vector(g, D, ty, 0.2, 1.0), c_before=_vector(g, D, ty, 0.1) if affine else None)
    if not case["backward"]:
        return dict(s, s=_empty(M, D, ty, pad), h=_empty(M, D, ty, pad))
    s["s"] = s.pop("r")  # the stream that the forward pass left
    s["ds"], s["dh"] = _matrix(g, M, D, ty, 0.1, pad), _matrix(g, M, D, ty, 0.1, pad)
    s["dr"], s["db"] = _empty(M, D, ty, pad), _empty(M, D, ty, pad)
    s["dgate"] = _empty(groups, D, ty, pad) if groups else None
    for n in ("w_after", "c_after", "w_before", "c_before"):
        s["d" + n] = None if s[n] is None else torch.empty_like(s[n])
    return s


def _quantize_state(case, seed):
    M, D = case["M"], case["D"]
    x = _matrix(_gen(seed), M, D, case["type"], 1.0, case["pad"])
    blocks = -(-D // 32)
    return dict(x=x, values=_empty(M, D, case["type"], case["pad"]),
                codes=torch.empty(M, blocks * 16, dtype=torch.uint8, device="cuda"),
                scales=torch.empty(M, -(-blocks // 4) * 4, dtype=torch.uint8, device="cuda"))


def _mx_state(case, seed):
    g = _gen(seed)
    M, N, K, ty, pad = (case[k] for k in ("M", "N", "K", "type", "pad"))
    codes, scales = _plain_quantize(_matrix(g, N, K, "f32", K ** -0.5))
    return dict(x=_matrix(g, M, K, ty, 1.0, pad), codes=codes, scales=scales,
                bias=_vector(g, N, ty, 0.1) if case["bias"] else None,
                residual=_matrix(g, M, N, ty, 1.0, pad) if case["residual"] else None, y=_empty(M, N, ty, pad))


def _moe_state(case, seed):
    g = _gen(seed)
    T, E, k, D, F, ty, pad = (case[n] for n in ("T", "E", "k", "D", "F", "type", "pad"))

    def experts(rows, cols):
        t = torch.empty(E, rows, cols + pad, dtype=_TYPES[ty], device="cuda")
        for e in range(E):
            t[e].copy_(torch.randn(t[e].shape, generator=g, device="cuda").mul_(cols ** -0.5))
        return t[:, :, :cols]

    return dict(x=_matrix(g, T, D, ty, 1.0, pad), router=_matrix(g, E, D, ty, D ** -0.5, pad), wg=experts(F, D),
                wu=experts(F, D), wd=experts(D, F), residual=_matrix(g, T, D, ty, 1.0, pad) if case["residual"] else None,
                y=_empty(T, D, ty, pad), chosen=torch.empty(T, k, dtype=torch.int32, device="cuda"),
                weights=torch.empty(T, k, device="cuda"))


def prepare(case, seed):
    make = {"norm": _norm_state, "quantize": _quantize_state, "mx": _mx_state, "moe": _moe_state}
    s = dict(case=case, **make[case["kind"]](case, seed))
    if own:  # the descriptors and workspaces that a program keeps between its calls
        from paper_1504_04343_amd import binding as B
        s["B"], k = B, case["kind"]
        ty = {"f32": B.TYPE_F32, "bf16": B.TYPE_BF16, "f16": B.TYPE_F16}[case["type"]]
        acts = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU,
                "gelu_tanh": B.ACT_GELU_TANH}
        if k == "norm":
            norms = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}
            s["desc"] = B.make_residual_norm_desc(case["M"], case["D"], ty, norms[case["before"]], norms[case["after"]],
                                                  max(1, case["gate"]), _EPS, _SCALE)
            if case["backward"]:
                s["ws"] = B.alloc_residual_norm_workspace(s["desc"])
        elif k == "quantize":
            s["mx"] = B.MxMatrix(case["M"], case["D"], s["codes"], s["scales"])
        elif k == "mx":
            s["w"] = B.MxMatrix(case["N"], case["K"], s["codes"], s["scales"])
            s["desc"] = B.make_linear_desc(case["M"], case["N"], case["K"], ty, acts[case["act"]])
            s["ws"] = B.alloc_mx_linear_workspace(s["desc"], True)
        else:
            s["desc"] = B.make_moe_desc(case["T"], case["E"], case["k"], case["D"], case["F"], ty, acts[case["act"]],
                                        case["normalize"])
            s["ws"] = B.alloc_moe_workspace(s["desc"])
    return s


# ---- one pass, in plain form --------------------------------------------------------------------

def _plain_stats(kind, v):
    """What a norm multiplies its weight by, and the factor in it."""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((v * v).mean(1, keepdim=True) + _EPS)
    return v * rstd, rstd


def _plain_affine(n, w, c):
    n = n * w.float()
    return n if c is None else n + c.float()


def _gate_rows(s, gate):
    return gate.float().repeat_interleave(s["case"]["gate"], 0)[: s["case"]["M"]]


def _plain_norm(s):
    case, ty = s["case"], s["b"].dtype
    b = s["b"].float()
    p = b if case["after"] == "none" else _plain_affine(_plain_stats(case["after"], b)[0], s["w_after"], s["c_after"])
    if s["gate"] is not None:
        p = p * _gate_rows(s, s["gate"])
    new = s["r"].float() + _SCALE * p
    h = _plain_affine(_plain_stats(case["before"], new)[0], s["w_before"], s["c_before"])
    return dict(s=new.to(ty), h=h.to(ty))


def _plain_back(kind, d, n, rstd):
    """The gradient of a norm's input from that of what its weight is multiplied by."""
    v = d - n * (d * n).mean(1, keepdim=True)
    return rstd * (v - d.mean(1, keepdim=True) if kind == "layer" else v)


def _plain_norm_backward(s):
    case, ty = s["case"], s["b"].dtype
    M, D, after = case["M"], case["D"], case["after"]
    dh, b = s["dh"].float(), s["b"].float()
    n, rstd = _plain_stats(case["before"], s["s"].float())
    ds = s["ds"].float() + _plain_back(case["before"], dh * s["w_before"].float(), n, rstd)
    out = dict(dr=ds, dw_before=(dh * n).sum(0))
    if s["c_before"] is not None:
        out["dc_before"] = dh.sum(0)
    dp = _SCALE * ds
    if after != "none":
        n, rstd = _plain_stats(after, b)
        b = _plain_affine(n, s["w_after"], s["c_after"])
    if s["gate"] is not None:
        rows, groups = case["gate"], s["gate"].shape[0]
        each = torch.zeros(groups * rows, D, device=b.device)
        each[:M] = dp * b
        out["dgate"] = each.view(groups, rows, D).sum(1)
        dp = dp * _gate_rows(s, s["gate"])
    if after != "none":
        out["dw_after"] = (dp * n).sum(0)
        if s["c_after"] is not None:
            out["dc_after"] = dp.sum(0)
        dp = _plain_back(after, dp * s["w_after"].float(), n, rstd)
    out["db"] = dp
    return {k: v.to(ty) for k, v in out.items()}


_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _power(e):
    """2^e for whole numbers e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64).float()


def _plain_quantize(x):
    """The codes and scales of a matrix."""
    rows, cols = x.shape
    blocks = -(-cols // 32)
    v = torch.zeros(rows, blocks * 32, device=x.device)
    v[:, :cols] = x.float()
    v = v.view(rows, blocks, 32)
    largest = v.abs().amax(2)
    e = (torch.frexp(largest.double())[1] - 3).clamp(-127, 127)
    e = torch.where(largest > 0, e, torch.full_like(e, -127))
    v = v * _power(-e)[:, :, None]
    a = v.abs().clamp(max=6.0)
    low, high = a < 2.0, a >= 4.0
    # the distance of neighbours is 0.5 up to 2, 1 up to 4, 2 from there on: which multiple, ties to the even one
    n = torch.round(torch.where(low, a * 2.0, torch.where(high, a * 0.5, a))).int()
    code = torch.where(low, n, torch.where(high, n + 4, n + 2)) + torch.where(torch.signbit(v), 8, 0)
    code = code.view(rows, blocks * 16, 2)
    codes = (code[:, :, 0] + code[:, :, 1] * 16).to(torch.uint8)
    scales = torch.zeros(rows, -(-blocks // 4) * 4, dtype=torch.uint8, device=x.device)
    scales[:, :blocks] = (e + 127).to(torch.uint8)
    return codes, scales


def _plain_values(codes, scales, cols):
    """The values that codes and scales stand for, 32 bits."""
    rows = codes.shape[0]
    table = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], 2).view(rows, -1, 32)
    return (v * _power(scales[:, : v.shape[1]].int() - 127)[:, :, None]).view(rows, -1)[:, :cols]


_TANH_C = math.sqrt(2.0 / math.pi)


def _plain_act(act, z):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "gelu":
        return z * 0.5 * torch.erfc(z * -math.sqrt(0.5))
    if act == "gelu_tanh":  # (1 + tanh(a)) / 2 is the logistic function of 2 a
        return z / (1.0 + torch.exp(-2.0 * _TANH_C * (z + 0.044715 * z * z * z)))
    return z


def _plain_mx(s):
    K = s["case"]["K"]
    x, w = _plain_values(*_plain_quantize(s["x"]), K), _plain_values(s["codes"], s["scales"], K)
    z = x @ w.t()
    y = _plain_act(s["case"]["act"], z if s["bias"] is None else z + s["bias"].float())
    return dict(y=(y if s["residual"] is None else y + s["residual"].float()).to(s["x"].dtype))


def _plain_moe(s):
    case = s["case"]
    T, E, k, D, F = (case[n] for n in ("T", "E", "k", "D", "F"))
    x = s["x"].float()
    logits = (s["x"].double() @ s["router"].double().t()).float()
    order = torch.sort(logits, dim=1, descending=True, stable=True)[1][:, :k]  # ties: the lowest index first
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    chosen = e.gather(1, order)
    weights = chosen / (chosen if case["normalize"] else e).sum(1, keepdim=True)
    if T * k < E:  # the chosen experts' weights
        at = order.reshape(-1)
        xs = x.repeat_interleave(k, 0)[:, :, None]
        g, u = torch.bmm(s["wg"][at].float(), xs), torch.bmm(s["wu"][at].float(), xs)
        parts = torch.bmm(s["wd"][at].float(), _plain_act(case["act"], g) * u)
        y = (parts.view(T, k, D) * weights[:, :, None]).sum(1)
    else:  # all experts' products, those that were not chosen with a weight of zero
        spread = torch.zeros(T, E, device=x.device).scatter_(1, order, weights)
        g, u = x @ s["wg"].float().reshape(E * F, D).t(), x @ s["wu"].float().reshape(E * F, D).t()
        h = (_plain_act(case["act"], g) * u).view(T, E, F) * spread[:, :, None]
        y = h.view(T, E * F) @ s["wd"].float().transpose(1, 2).reshape(E * F, D)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return dict(y=y.to(s["x"].dtype), chosen=order.int(), weights=weights)


# ---- one pass, as a program calls it ------------------------------------------------------------

def _own_norm(s):
    s["B"].cct_residual_norm_forward(s["desc"], s["r"], s["b"], s["gate"], s["w_after"], s["c_after"], s["w_before"],
                                     s["c_before"], s["s"], s["h"])
    return dict(s=s["s"], h=s["h"])


def _own_norm_backward(s):
    s["B"].cct_residual_norm_backward(s["desc"], s["s"], s["b"], s["gate"], s["w_after"], s["c_after"], s["w_before"],
                                      s["ds"], s["dh"], s["dr"], s["db"], s["dgate"], s["dw_after"], s["dc_after"],
                                      s["dw_before"], s["dc_before"], s["ws"])
    names = ("dr", "db", "dgate", "dw_after", "dc_after", "dw_before", "dc_before")
    return {n: s[n] for n in names if s[n] is not None}


def _own_quantize(s):
    s["B"].cct_mx_quantize(s["x"], s["mx"])
    s["B"].cct_mx_dequantize(s["mx"], s["values"])
    return dict(values=s["values"])


def _own_mx(s):
    s["B"].cct_mx_linear_forward(s["desc"], s["x"], s["w"], s["bias"], s["residual"], s["y"], None, s["ws"])
    return dict(y=s["y"])


def _own_moe(s):
    s["B"].cct_moe_forward(s["desc"], s["x"], s["router"], s["wg"], s["wu"], s["wd"], s["residual"], s["y"], s["chosen"],
                           s["weights"], s["ws"])
    return dict(y=s["y"], chosen=s["chosen"], weights=s["weights"])


def run(state):
    k = state["case"]["kind"]
    if k == "norm":
        if state["case"]["backward"]:
            return _own_norm_backward(state) if own else _plain_norm_backward(state)
        return _own_norm(state) if own else _plain_norm(state)
    if k == "quantize":
        if own:
            return _own_quantize(state)
        x = state["x"]
        return dict(values=_plain_values(*_plain_quantize(x), x.shape[1]).to(x.dtype))
    if k == "mx":
        return _own_mx(state) if own else _plain_mx(state)
    return _own_moe(state) if own else _plain_moe(state)


# ---- what a pass cannot do without: every input read once, every output written once ------------

def work(case):
    k, e = case["kind"], _SIZE[case["type"]]
    if k == "norm":
        M, D = case["M"], case["D"]
        after = case["after"] != "none"
        groups = -(-M // case["gate"]) if case["gate"] else 0
        vectors = (1 + after) * (1 + case["affine"])
        if case["backward"]:
            return dict(bytes=e * D * (6 * M + 2 * (groups + vectors)), flops=(20 + 15 * after) * M * D)
        return dict(bytes=e * D * (4 * M + groups + vectors), flops=(8 + 5 * after) * M * D)
    if k == "quantize":
        n = case["M"] * case["D"]
        return dict(bytes=int(n * (2 * e + 2 * 17 / 32)), flops=4 * n)
    if k == "mx":
        M, N, K = case["M"], case["N"], case["K"]
        n = M * K + M * N * (1 + case["residual"]) + (N if case["bias"] else 0)
        return dict(bytes=int(e * n + N * K * 17 / 32), flops=2 * M * N * K)
    T, E, c, D, F = (case[n] for n in ("T", "E", "k", "D", "F"))
    used = E * (1.0 - (1.0 - c / E) ** T)  # experts that some token chose, expected
    n = used * 3 * D * F + E * D + T * D * (2 + case["residual"])
    return dict(bytes=int(e * n + 8 * T * c), flops=2 * T * (3 * c * D * F + E * D))


# ---- the same from the definitions in 64 bits ---------------------------------------------------

def _exact_normed(kind, v, w, c):
    import torch.nn.functional as F
    if kind == "none":
        return v
    if kind == "layer":
        return F.layer_norm(v, v.shape[1:], w, c, _EPS)
    n = v / v.square().mean(1, keepdim=True).add(_EPS).sqrt() * w
    return n if c is None else n + c


def _exact_norm(case, s, d):
    """Gradients by differentiating the definition; the plain form has them as formulas."""
    if case["backward"]:
        # the stream is what the forward pass left: r is taken from it, so that r + scale * gate * N(b) is the stream
        wanted = [n for n in ("b", "gate", "w_after", "c_after", "w_before", "c_before") if n in d]
        for n in wanted:
            d[n].requires_grad_()
    rows = torch.arange(case["M"], device="cuda") // case["gate"] if case["gate"] else None
    p = _exact_normed(case["after"], d["b"], d.get("w_after"), d.get("c_after"))
    p = p if rows is None else p * d["gate"][rows]
    if not case["backward"]:
        new = d["r"] + _SCALE * p
        return dict(s=new, h=_exact_normed(case["before"], new, d["w_before"], d.get("c_before")))
    r = (d["s"] - _SCALE * p).detach().requires_grad_()
    new = r + _SCALE * p
    h = _exact_normed(case["before"], new, d["w_before"], d.get("c_before"))
    grads = torch.autograd.grad([new, h], [r] + [d[n] for n in wanted], [d["ds"], d["dh"]])
    return dict(zip(["dr"] + ["d" + n for n in wanted], grads))


def _exact_mx_values(x):
    """A matrix's values rounded to the microscaled format, by comparing with the middles between neighbours."""
    import torch.nn.functional as F
    rows, cols = x.shape
    v = F.pad(x.double(), (0, -cols % 32)).view(rows, -1, 32)
    most = v.abs().amax(2, keepdim=True)
    scale = torch.where(most > 0, 2.0 ** (torch.floor(torch.log2(most)) - 2.0), 1.0)
    a = v.abs() / scale
    # a middle belongs to the neighbour whose last bit is zero
    steps = (0.5 * (a > 0.25) + 0.5 * (a >= 0.75) + 0.5 * (a > 1.25) + 0.5 * (a >= 1.75) + (a > 2.5) + (a >= 3.5) + 2.0 * (a > 5.0))
    return (steps * v.sign() * scale).view(rows, -1)[:, :cols]


def _exact_act(act, z):
    import torch.nn.functional as F
    return {"none": lambda t: t, "relu": F.relu, "silu": F.silu, "gelu": F.gelu,
            "gelu_tanh": lambda t: F.gelu(t, approximate="tanh")}[act](z)


def _exact_moe(case, s):
    x = s["x"].double()
    logits = torch.nn.functional.linear(x, s["router"].double()).float().double()
    # an expert's place: how many are before it, larger ones and equal ones of lower number
    larger = logits[:, None, :] > logits[:, :, None]
    n = torch.arange(case["E"], device="cuda")
    equal = (logits[:, None, :] == logits[:, :, None]) & (n[None, None, :] < n[None, :, None])
    place = (larger | equal).sum(2)
    spread = torch.softmax(logits if not case["normalize"] else logits.masked_fill(place >= case["k"], -math.inf), 1)
    y = s["residual"].double() if s["residual"] is not None else torch.zeros_like(x)
    for e in range(case["E"]):
        at = (place[:, e] < case["k"]).nonzero()[:, 0]
        if len(at):
            h = _exact_act(case["act"], x[at] @ s["wg"][e].double().t()) * (x[at] @ s["wu"][e].double().t())
            y[at] = y[at] + spread[at, e][:, None] * (h @ s["wd"][e].double().t())
    chosen = torch.argsort(place, 1)[:, : case["k"]]
    return dict(y=y, chosen=None, weights=spread.gather(1, chosen))


def exact(case, seed):
    import torch.nn.functional as F
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    k = case["kind"]
    if k == "moe":
        return _exact_moe(case, s)
    d = {n: t.double() for n, t in s.items() if isinstance(t, torch.Tensor) and t.is_floating_point()}
    if k == "norm":
        return _exact_norm(case, s, d)
    if k == "quantize":
        return dict(values=_exact_mx_values(s["x"]))
    scale = 2.0 ** (s["scales"].double() - 127.0)
    code = torch.stack([s["codes"] % 16, s["codes"] // 16], 2).view(case["N"], -1, 32).long()
    m, field = code % 2, code % 8 // 2  # sign, two bits of exponent, one of mantissa
    w = torch.where(field == 0, 0.5 * m, (1.0 + 0.5 * m) * 2.0 ** (field - 1.0)) * torch.where(code >= 8, -1.0, 1.0)
    w = (w.double() * scale[:, : w.shape[1], None]).view(case["N"], -1)[:, : case["K"]]
    y = _exact_act(case["act"], F.linear(_exact_mx_values(s["x"]), w, d.get("bias")))
    return dict(y=y if s["residual"] is None else y + d["residual"])
