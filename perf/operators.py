"""The operators of a feed-forward block in training and in serving, as cases that can be timed and compared.

Four operators that a training step of fully connected layers runs one after the other:

  ``linear``  y = act(x w^T + bias) + residual in one product, and its backward pass (dx, dw, dbias);
  ``gated``   h = act(x wg^T) * (x wu^T), both products in one, and its backward pass (dx, dwg, dwu);
  ``clip``    the 2-norm of all gradients together, and the gradients scaled down to a largest norm;
  ``update``  the same norm, and momentum, weight decay and the clipped step over all parameters.

With ``own`` false a pass is elementary torch operations in 32 bits, rounded once at the end; with
``own`` true it is what a program calls in ``paper_1504_04343_amd.binding``.

x, w, y and their gradients are matrices of one type (fp32, bf16, fp16) whose rows lie ``ld`` elements
apart: ``pad`` elements more than they have, as in slices of wider tensors.  z, g and u are the
products before the activation, in the same type, which a training program keeps for the backward pass.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _linear(name, M, N, K, type, act, backward=False, bias=True, residual=False, save=False, pad=0):
    return dict(name=name, kind="linear", M=M, N=N, K=K, type=type, act=act, backward=backward, bias=bias,
                residual=residual, save=save, pad=pad)


def _gated(name, M, F, K, type, act, backward=False, save=False, pad=0):
    return dict(name=name, kind="gated", M=M, F=F, K=K, type=type, act=act, backward=backward, save=save,
                pad=pad)


def _step(name, kind, params, type, max_norm, copy=False, tight=False):
    case = dict(name=name, kind=kind, params=params, type=type, max_norm=max_norm, tight=tight)
    if kind == "update":
        case["copy"] = copy
    return case


def listed():
    return [
        # serving: one image's features through a classifier's middle layer; the weights are read once
        _linear("linear_one_row", 1, 4096, 4096, "bf16", "relu"),
        # the projection back to the residual stream in training, with the stream's addition
        _linear("linear_forward", 4096, 4096, 4096, "bf16", "none", residual=True),
        # the first fully connected layer of CaffeNet (256 x 6 x 6 features) at batch 1024, fp32 as the
        # convolutions leave it: its gradients
        _linear("linear_backward_f32", 1024, 4096, 9216, "f32", "relu", backward=True),
        # a layer of odd sizes whose rows are slices of wider tensors, gradients in fp16
        _linear("linear_backward_odd", 1531, 1000, 2049, "f16", "gelu", backward=True, pad=3),
        # serving a gated block: a single token
        _gated("gated_one_row", 1, 8192, 4096, "bf16", "silu"),
        # serving a gated block: a batch of sequences, one token each
        _gated("gated_few_rows", 48, 8192, 4096, "bf16", "silu"),
        # training: what the backward pass needs is kept
        _gated("gated_forward", 4096, 8192, 4096, "bf16", "silu", save=True),
        # training: the largest batch
        _gated("gated_backward", 8192, 8192, 4096, "bf16", "silu", backward=True),
        # every gradient of CaffeNet (61 million in 16 tensors), as the fp32 kernels leave them
        _step("clip_caffenet", "clip", "caffenet", "f32", 1.0),
        # a deep model's many tensors, most of them small and of odd sizes, bf16 gradients
        _step("clip_many", "clip", "many-400-1", "bf16", 1.0),
        # CaffeNet's weight update
        _step("update_caffenet", "update", "caffenet", "f32", 1.0),
        # the deep model's: bf16 gradients, fp32 weights, and the bf16 copy that the products read
        _step("update_many", "update", "many-400-2", "bf16", 1.0, copy=True),
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
        if u < 0.75:
            type = rng.choice(["bf16", "bf16", "f16", "f32"])
            M = _log_int(rng, 1, 8192)
            pad = rng.choice([0, 0, 0, 8, 64, 1, 5])
            back = rng.random() < 0.45
            if u < 0.42:
                case = _linear("", M, _size(rng, 10, 16384), _size(rng, 16, 16384), type,
                               rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), back,
                               rng.random() < 0.6, not back and rng.random() < 0.5,
                               not back and rng.random() < 0.3, pad)
            else:
                case = _gated("", M, _size(rng, 64, 16384), _size(rng, 32, 8192), type,
                              rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu"]), back,
                              not back and rng.random() < 0.5, pad)
        else:
            kind = "clip" if u < 0.87 else "update"
            params = "many-%d-%d" % (_log_int(rng, 1, 600), rng.randrange(1 << 20))
            case = _step("", kind, params, rng.choice(["f32", "bf16", "f16"]),
                         rng.choice([0.5, 1.0, 1e6]), rng.random() < 0.5, rng.random() < 0.3)
        del case["name"]
        w = work(case)
        limit = 2.0e12 if case.get("type") != "f32" or case["kind"] in ("clip", "update") else 6.0e11
        if w["flops"] <= limit and w["bytes"] <= 1.2e9:
            return case


# ---- shapes -------------------------------------------------------------------------------------

_CAFFENET = [(96, 3, 11, 11), (96,), (256, 48, 5, 5), (256,), (384, 256, 3, 3), (384,), (384, 192, 3, 3), (384,),
             (256, 192, 3, 3), (256,), (4096, 9216), (4096,), (4096, 4096), (4096,), (1000, 4096), (1000,)]


def _numels(params):
    """The number of values of each parameter."""
    if params == "caffenet":
        return [math.prod(s) for s in _CAFFENET]
    import random
    _, count, seed = params.split("-")
    r = random.Random(int(seed))
    out = []
    while len(out) < int(count):  # of ten tensors, six vectors (scales, biases) and four matrices, of odd sizes too
        n = _log_int(r, 16, 8192) if r.random() < 0.6 else _log_int(r, 2000, 2000000)
        out.append(n)
    return out


# ---- what a program has in hand before the call -------------------------------------------------

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _matrix(g, rows, cols, type, std=1.0, pad=0):
    """rows x cols values, rows cols + pad elements apart."""
    t = torch.empty(rows, cols + pad, dtype=_TYPES[type], device="cuda")
    t.copy_(torch.randn(t.shape, generator=g, device="cuda").mul_(std))
    return t[:, :cols]


def _empty(rows, cols, type, pad=0):
    return torch.empty(rows, cols + pad, dtype=_TYPES[type], device="cuda")[:, :cols]


def _linear_state(case, seed):
    g = _gen(seed)
    M, N, K, ty, pad = (case[k] for k in ("M", "N", "K", "type", "pad"))
    s = dict(x=_matrix(g, M, K, ty, pad=pad), w=_matrix(g, N, K, ty, K ** -0.5, pad),
             bias=_matrix(g, 1, N, ty, 0.1).view(N) if case["bias"] else None)
    s["dims"] = (M, N, K)
    if case["backward"]:
        s["z"] = _empty(M, N, ty, pad) if case["act"] != "none" else None
        if s["z"] is not None:
            s["z"].copy_(_plain_product(s["x"], s["w"], s["bias"]))
        s["dy"] = _matrix(g, M, N, ty, 0.1, pad)
        s["dx"], s["dw"] = _empty(M, K, ty, pad), _empty(N, K, ty, pad)
        s["dbias"] = torch.empty(N, dtype=_TYPES[ty], device="cuda") if case["bias"] else None
    else:
        s["residual"] = _matrix(g, M, N, ty, pad=pad) if case["residual"] else None
        s["y"] = _empty(M, N, ty, pad)
        s["z"] = _empty(M, N, ty, pad) if case["save"] else None
    return s


def _gated_state(case, seed):
    g = _gen(seed)
    M, F, K, ty, pad = (case[k] for k in ("M", "F", "K", "type", "pad"))
    s = dict(x=_matrix(g, M, K, ty, pad=pad), wg=_matrix(g, F, K, ty, K ** -0.5, pad),
             wu=_matrix(g, F, K, ty, K ** -0.5, pad))
    s["dims"] = (M, F, K)
    if case["backward"]:
        s["g"], s["u"] = _empty(M, F, ty, pad), _empty(M, F, ty, pad)
        s["g"].copy_(_plain_product(s["x"], s["wg"]))
        s["u"].copy_(_plain_product(s["x"], s["wu"]))
        s["dh"] = _matrix(g, M, F, ty, 0.1, pad)
        s["dx"], s["dwg"], s["dwu"] = _empty(M, K, ty, pad), _empty(F, K, ty, pad), _empty(F, K, ty, pad)
    else:
        s["h"] = _empty(M, F, ty, pad)
        s["g"], s["u"] = (_empty(M, F, ty, pad), _empty(M, F, ty, pad)) if case["save"] else (None, None)
    return s


def _places(case):
    """Where each parameter begins in one buffer, its size, and the buffer's: at every 64th value as allocations
    do, or tightly one behind the other as in a gradient bucket."""
    at, places = 0, []
    for n in _numels(case["params"]):
        places.append((at, n))
        at += n if case["tight"] else -(-n // 64) * 64
    return places, at


def _step_state(case, seed):
    g = _gen(seed)
    places, total = _places(case)
    here = torch.zeros(total, dtype=torch.bool)
    for at, n in places:
        here[at:at + n] = True
    here = here.cuda()

    def buffer(std, dtype=torch.float32):
        return torch.randn(total, generator=g, device="cuda").mul_(std).mul_(here).to(dtype)

    def views(flat):
        return [flat[at:at + n] for at, n in places]

    s = dict(grads_flat=buffer(0.01, _TYPES[case["type"]]), clip=torch.empty(2, device="cuda"))
    if case["kind"] == "clip":
        s["out_flat"] = torch.zeros_like(s["grads_flat"])
    else:
        s["weights_flat"], s["moments_flat"] = buffer(0.05), buffer(0.001)
        if case["copy"]:
            s["copies_flat"] = s["weights_flat"].to(torch.bfloat16)
    for name in ("grads", "out", "weights", "moments", "copies"):
        s[name] = views(s[name + "_flat"]) if name + "_flat" in s else None
    return s


def prepare(case, seed):
    make = {"linear": _linear_state, "gated": _gated_state, "clip": _step_state, "update": _step_state}
    s = dict(case=case, **make[case["kind"]](case, seed))
    if own:  # the descriptors, lists and workspaces that a program keeps between its calls
        from paper_1504_04343_amd import binding as B
        s["B"] = B
        k = case["kind"]
        if k in ("linear", "gated"):
            types = {"f32": B.TYPE_F32, "bf16": B.TYPE_BF16, "f16": B.TYPE_F16}
            acts = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU,
                    "gelu_tanh": B.ACT_GELU_TANH}
            make_desc = B.make_linear_desc if k == "linear" else B.make_gated_desc
            s["desc"] = make_desc(*s["dims"], type=types[case["type"]], activation=acts[case["act"]])
            p = B.PASS_BACKWARD if case["backward"] else B.PASS_FORWARD
            s["ws"] = B.alloc_linear_workspace(s["desc"], p) if k == "linear" else \
                B.alloc_gated_workspace(s["desc"], p)
        else:
            for name in ("grads", "out", "weights", "moments", "copies"):
                if s.get(name) is not None:
                    s[name + "_list"] = B.make_tensor_list(s[name])
            s["ws"] = B.alloc_norm_workspace(s["grads_list"])
    return s


# ---- one pass, in plain form --------------------------------------------------------------------

def _plain_product(x, w, bias=None):
    z = x.float() @ w.float().t()
    return z if bias is None else z + bias.float()


_TANH_C = math.sqrt(2.0 / math.pi)


def _plain_act(act, z):
    """act(z) and its derivative, 32 bits."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0.0), (z > 0).float()
    if act == "silu":
        e = 1.0 / (1.0 + torch.exp(-z))
        return z * e, e * (1.0 + z * (1.0 - e))
    if act == "gelu":
        cdf = 0.5 * torch.erfc(z * -math.sqrt(0.5))
        return z * cdf, cdf + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    # tanh(a) as 1 - 2 / (1 + exp(2 a)), so that 0.5 * (1 + tanh(a)) is the logistic function of 2 a
    a = _TANH_C * (z + 0.044715 * z * z * z)
    e = 1.0 / (1.0 + torch.exp(-2.0 * a))
    return z * e, e + z * 2.0 * e * (1.0 - e) * _TANH_C * (1.0 + 3.0 * 0.044715 * z * z)


def _plain_linear(s):
    act, ty = s["case"]["act"], s["x"].dtype
    if not s["case"]["backward"]:
        z = _plain_product(s["x"], s["w"], s["bias"])
        y = _plain_act(act, z)[0]
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return dict(y=y.to(ty), **(dict(z=z.to(ty)) if s["z"] is not None else {}))
    dz = s["dy"].float()
    if act != "none":
        dz = dz * _plain_act(act, s["z"].float())[1]
    out = dict(dx=(dz @ s["w"].float()).to(ty), dw=(dz.t() @ s["x"].float()).to(ty))
    if s["dbias"] is not None:
        out["dbias"] = dz.sum(0).to(ty)
    return out


def _plain_gated(s):
    act, ty = s["case"]["act"], s["x"].dtype
    if not s["case"]["backward"]:
        g, u = _plain_product(s["x"], s["wg"]), _plain_product(s["x"], s["wu"])
        h = (_plain_act(act, g)[0] * u).to(ty)
        return dict(h=h, g=g.to(ty), u=u.to(ty)) if s["g"] is not None else dict(h=h)
    dh, u = s["dh"].float(), s["u"].float()
    a, da = _plain_act(act, s["g"].float())
    dg, du = dh * u * da, dh * a
    x = s["x"].float()
    return dict(dx=(dg @ s["wg"].float() + du @ s["wu"].float()).to(ty), dwg=(dg.t() @ x).to(ty),
                dwu=(du.t() @ x).to(ty))


def _whole(tensors):
    """All values of a list of tensors, in 32 bits."""
    return torch.cat(tensors).float()


def _spread(values, tensors):
    """The values back to a list of tensors."""
    torch._foreach_copy_(tensors, list(values.split([t.numel() for t in tensors])))


_LR, _MOMENTUM, _DECAY = 0.01, 0.9, 0.0005


def _plain_step(s):
    grads, most = _whole(s["grads"]), s["case"]["max_norm"]
    norm = grads.square().sum(dtype=torch.float64).sqrt()
    scale = torch.where(norm > most, most / norm, torch.ones_like(norm)).float()
    s["clip"].copy_(torch.stack([norm.float(), scale]))
    grads = grads * scale
    if s["case"]["kind"] == "clip":
        _spread(grads, s["out"])
        return
    w = _whole(s["weights"])
    v = _whole(s["moments"]) * _MOMENTUM + (grads + w * _DECAY) * _LR
    w = w - v
    _spread(v, s["moments"])
    _spread(w, s["weights"])
    if s["copies"] is not None:
        _spread(w, s["copies"])


def _step_outputs(s):
    """The buffers in which the tensors lie, whole."""
    names = ("out",) if s["case"]["kind"] == "clip" else ("weights", "moments", "copies")
    return dict(clip=s["clip"], **{n: s[n + "_flat"] for n in names if n + "_flat" in s})


# ---- one pass, as a program calls it ------------------------------------------------------------

def _own_linear(s):
    B = s["B"]
    if s["case"]["backward"]:
        B.cct_linear_backward(s["desc"], s["x"], s["w"], s["z"], s["dy"], s["dx"], s["dw"], s["dbias"], s["ws"])
        out = dict(dx=s["dx"], dw=s["dw"])
        return dict(out, dbias=s["dbias"]) if s["dbias"] is not None else out
    B.cct_linear_forward(s["desc"], s["x"], s["w"], s["bias"], s["residual"], s["y"], s["z"], s["ws"])
    return dict(y=s["y"], z=s["z"]) if s["z"] is not None else dict(y=s["y"])


def _own_gated(s):
    B = s["B"]
    if s["case"]["backward"]:
        B.cct_gated_backward(s["desc"], s["x"], s["wg"], s["wu"], s["g"], s["u"], s["dh"], s["dx"], s["dwg"],
                             s["dwu"], s["ws"])
        return dict(dx=s["dx"], dwg=s["dwg"], dwu=s["dwu"])
    B.cct_gated_forward(s["desc"], s["x"], s["wg"], s["wu"], s["h"], s["g"], s["u"], s["ws"])
    return dict(h=s["h"], g=s["g"], u=s["u"]) if s["g"] is not None else dict(h=s["h"])


def _own_step(s):
    B = s["B"]
    B.cct_grad_norm(s["grads_list"], s["case"]["max_norm"], s["clip"], s["ws"])
    if s["case"]["kind"] == "clip":
        B.cct_grad_scale(s["grads_list"], s["clip"], s["out_list"])
    else:
        B.cct_sgd_update(s["grads_list"], s["clip"], s["weights_list"], s["moments_list"], s.get("copies_list"),
                         _LR, _MOMENTUM, _DECAY)


def run(state):
    k = state["case"]["kind"]
    if k == "linear":
        return _own_linear(state) if own else _plain_linear(state)
    if k == "gated":
        return _own_gated(state) if own else _plain_gated(state)
    if own:
        _own_step(state)
    else:
        _plain_step(state)
    return _step_outputs(state)


# ---- what a pass cannot do without: every input read once, every output written once ------------

def work(case):
    k, e = case["kind"], _SIZE[case["type"]]
    if k in ("clip", "update"):
        n = sum(_numels(case["params"]))
        if k == "clip":
            return dict(bytes=2 * e * n + 8, flops=3 * n)
        return dict(bytes=(e + 16 + (2 if case["copy"] else 0)) * n + 8, flops=8 * n)
    if k == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        one = M * K + N * K
        if case["backward"]:
            n = 2 * one + M * N * (1 if case["act"] == "none" else 2) + (N if case["bias"] else 0)
            return dict(bytes=e * n, flops=4 * M * N * K)
        n = one + M * N * (1 + case["residual"] + case["save"]) + (N if case["bias"] else 0)
        return dict(bytes=e * n, flops=2 * M * N * K)
    M, F, K = case["M"], case["F"], case["K"]
    one = M * K + 2 * F * K
    if case["backward"]:
        return dict(bytes=e * (2 * one + 3 * M * F), flops=8 * M * F * K)
    return dict(bytes=e * (one + M * F * (3 if case["save"] else 1)), flops=4 * M * F * K)


# ---- the same from the definitions in 64 bits ---------------------------------------------------

def _exact_act(act, z):
    import torch.nn.functional as F
    return {"none": lambda t: t, "relu": F.relu, "silu": F.silu, "gelu": F.gelu,
            "gelu_tanh": lambda t: F.gelu(t, approximate="tanh")}[act](z)


def exact(case, seed):
    """Gradients by differentiating the definition; the plain form has them as formulas."""
    import torch.nn.functional as F
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    k = case["kind"]
    d = {n: t.double() for n, t in s.items() if isinstance(t, torch.Tensor)}
    if k == "linear" and not case["backward"]:
        z = F.linear(d["x"], d["w"], d.get("bias"))
        y = _exact_act(case["act"], z)
        y = y + d["residual"] if "residual" in d else y
        return dict(y=y, z=z) if case["save"] else dict(y=y)
    if k == "linear":
        if case["act"] == "none":
            dz = d["dy"]
        else:
            z = d["z"].requires_grad_()
            dz, = torch.autograd.grad(_exact_act(case["act"], z), z, d["dy"])
        out = dict(dx=torch.mm(dz, d["w"]), dw=torch.mm(d["x"].t(), dz).t())
        return dict(out, dbias=torch.mv(dz.t(), dz.new_ones(dz.shape[0]))) if case["bias"] else out
    if k == "gated" and not case["backward"]:
        g, u = F.linear(d["x"], d["wg"]), F.linear(d["x"], d["wu"])
        h = _exact_act(case["act"], g) * u
        return dict(h=h, g=g, u=u) if case["save"] else dict(h=h)
    if k == "gated":
        g, u = d["g"].requires_grad_(), d["u"].requires_grad_()
        dg, du = torch.autograd.grad(_exact_act(case["act"], g) * u, (g, u), d["dh"])
        dx = torch.addmm(torch.mm(dg, d["wg"]), du, d["wu"])
        return dict(dx=dx, dwg=torch.mm(d["x"].t(), dg).t(), dwu=torch.mm(d["x"].t(), du).t())
    grads = d["grads_flat"]  # what lies between the tensors is zero
    norm = torch.linalg.vector_norm(grads)
    scale = min(1.0, case["max_norm"] / float(norm)) if float(norm) > 0 else 1.0
    clip = torch.stack([norm, torch.full_like(norm, scale)])
    if k == "clip":
        return dict(clip=clip, out=grads * scale)
    v = _MOMENTUM * d["moments_flat"] + _LR * (scale * grads + _DECAY * d["weights_flat"])
    w = d["weights_flat"] - v
    return dict(clip=clip, weights=w, moments=v, **(dict(copies=w) if case["copy"] else {}))
