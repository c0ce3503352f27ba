"""The gradient norm, scaling and weight update over lists of tensors against 64 bits on the CPU.  Bounds: the norm is summed in
64 bits and rounded once to fp32 (and its square's 2^-53 errors): 2^-23 relative; a scaled gradient is one product rounded to
fp32 (if the type is narrower) and to the type, with clip[1] itself known to 2^-23; the update is five fp32 operations."""
import pytest
import torch

import feed_forward_util as ff

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    assert torch.cuda.is_available()
    from paper_1504_04343_amd import binding
    return binding


SIZES = {
    "one": [1],
    "small": [1, 2, 3, 7, 8, 9, 31, 1023, 1024, 1025],
    "runs": [8191, 8192, 8193, 3 * 8192 + 5, 1],
    "many": [((i * 7919) % 300) + 1 for i in range(500)],
    "empty": [0, 5, 0, 0, 8200, 0],
    "one large": [5000011],
}


def make(sizes, dtypes, seed, std, tight):
    """Tensors that lie one behind the other in one buffer per type (tight: at any address), on the GPU."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        dt = dtypes[i % len(dtypes)]
        off = (i % 7) if tight else 0
        flat = (torch.randn(n + off, generator=g) * std).to(dt)
        out.append(flat.cuda()[off:])
    return out


def norm64(grads):
    return float(sum((t.cpu().double() ** 2).sum() for t in grads)) ** 0.5 if grads else 0.0


@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("types", ["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("tight", [False, True])
def test_norm_and_scale(B, sizes, types, tight):
    dtypes = list(ff.TYPES.values()) if types == "mixed" else [ff.TYPES[types]]
    grads = make(SIZES[sizes], dtypes, 1, 0.5, tight)
    lst = B.make_tensor_list(grads)
    want = norm64(grads)
    clip = torch.full((2,), float("nan"), device="cuda")
    ws = B.alloc_norm_workspace(lst)
    for factor in (0.25, 4.0):
        ws.fill_(0xff)
        B.cct_grad_norm(lst, want * factor, clip, ws)
        norm, scale = clip.tolist()
        assert abs(norm - want) <= 2.0 ** -23 * want
        assert abs(scale - min(factor, 1.0)) <= 2.0 ** -22 * min(factor, 1.0)
        outs = [torch.full_like(t, float("nan")) for t in grads]
        B.cct_grad_scale(lst, clip, B.make_tensor_list(outs))
        for t, o in zip(grads, outs):
            v = t.cpu().double() * scale
            ff.check("out", o, ff.rounded(v, v.abs() * ff.EPS32, t.dtype))
    kept = [t.clone() for t in grads]
    B.cct_grad_scale(lst, clip, lst)                        # in place, scale 1: the same bits
    assert all(torch.equal(a, b) for a, b in zip(grads, kept))
    B.cct_grad_norm(lst, want * 0.25, clip, ws)
    B.cct_grad_scale(lst, clip, lst)                        # in place
    for t, k in zip(grads, kept):
        v = k.cpu().double() * float(clip[1])
        ff.check("in place", t, ff.rounded(v, v.abs() * ff.EPS32, t.dtype))


@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("type", list(ff.TYPES))
@pytest.mark.parametrize("copy", [None, "bf16", "f16", "f32"])
def test_update(B, sizes, type, copy):
    grads = make(SIZES[sizes], [ff.TYPES[type]], 2, 0.5, True)
    weights, moments = make(SIZES[sizes], [torch.float32], 3, 1.0, True), make(SIZES[sizes], [torch.float32], 4, 0.1, False)
    copies = None if copy is None else [torch.full_like(t, float("nan"), dtype=ff.TYPES[copy]) for t in weights]
    lists = [B.make_tensor_list(t) for t in (grads, weights, moments)]
    clist = None if copy is None else B.make_tensor_list(copies)
    clip = torch.tensor([7.0, 0.375], device="cuda")
    rate, momentum, decay = 0.125, 0.9, 0.01
    old = [[t.cpu().double() for t in ts] for ts in (grads, weights, moments)]
    for use in (clip, None):
        B.cct_sgd_update(lists[0], use, lists[1], lists[2], clist, rate, momentum, decay)
        s = 1.0 if use is None else 0.375
        for i, (g, w, v) in enumerate(zip(*old)):
            size = (momentum * v).abs() + rate * (s * g).abs() + rate * decay * w.abs()
            nv = float(torch.tensor(momentum)) * v + rate * (s * g + float(torch.tensor(decay)) * w)
            nw = w - nv
            ff.check("moment", moments[i], (nv, 5 * ff.EPS32 * size))
            ff.check("weight", weights[i], (nw, 5 * ff.EPS32 * size + ff.EPS32 * nw.abs()))
            if copies is not None:   # the rounded new weight, bit for bit
                assert torch.equal(copies[i], weights[i].to(copies[i].dtype))
        old = [old[0]] + [[t.cpu().double() for t in ts] for ts in (weights, moments)]


def test_values_at_the_ends(B):
    clip, inf = torch.empty(2, device="cuda"), float("inf")

    def run(values, limit=1.0, dt=torch.float32):
        t = [torch.tensor(values, dtype=dt, device="cuda")]
        lst = B.make_tensor_list(t)
        B.cct_grad_norm(lst, limit, clip, B.alloc_norm_workspace(lst))
        norm, scale = clip.tolist()
        B.cct_grad_scale(lst, clip, lst)
        return norm, scale, t[0].tolist()
    norm, scale, out = run([3e38, 0.0])          # its square is beyond fp32
    assert abs(norm - 3e38) <= 3e38 * 2.0 ** -22 and abs(out[0] - 1.0) <= 2.0 ** -20
    norm, scale, out = run([1e-42, 0.0])         # its square is below fp32
    assert abs(norm - 1e-42) <= 2e-45 and scale == 1.0
    assert run([0.0, 0.0]) == (0.0, 1.0, [0.0, 0.0])
    norm, scale, out = run([inf, 2.0])
    assert norm == inf and scale == 0.0 and out[0] != out[0] and out[1] == 0.0
    norm, scale, out = run([float("nan"), 2.0])
    assert norm != norm and scale != scale and out[1] != out[1]
    assert run([30.0, 40.0], inf) == (50.0, 1.0, [30.0, 40.0])
    assert run([3.0, 4.0], 5.0) == (5.0, 1.0, [3.0, 4.0])          # not above the limit
    empty = B.make_tensor_list([])
    B.cct_grad_norm(empty, 1.0, clip, B.alloc_norm_workspace(empty))
    assert clip.tolist() == [0.0, 1.0]
    B.cct_grad_scale(empty, clip, empty)
    B.cct_sgd_update(empty, clip, empty, empty, None, 0.1)


def test_same_bits_every_time_and_from_a_graph(B):
    grads = make([70000, 13, 400000, 8192], [torch.bfloat16], 7, 1.0, False)
    outs = [torch.empty_like(t) for t in grads]
    lst, olist = B.make_tensor_list(grads), B.make_tensor_list(outs)
    clip, ws = torch.empty(2, device="cuda"), B.alloc_norm_workspace(lst)

    def step():
        B.cct_grad_norm(lst, 1.0, clip, ws)
        B.cct_grad_scale(lst, clip, olist)
    step()
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    for _ in range(3):
        for t in grads:
            t.mul_(1.5)
        torch.cuda.synchronize()
        step()
        torch.cuda.synchronize()
        want, wc = [o.clone() for o in outs], clip.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(clip, wc) and all(torch.equal(a, b) for a, b in zip(outs, want))


def test_a_list_of_more_workgroups_than_a_launch_takes(B):
    """2^37 values and more in one list, which is one tensor 17 times over: two launches."""
    if torch.cuda.mem_get_info()[0] < 40e9:
        pytest.skip("needs 40 GB")
    flat = torch.zeros(1 << 33, dtype=torch.bfloat16, device="cuda")
    flat[::1 << 23] = 2.0
    flat[-1] = 5.0
    lst = B.make_tensor_list([flat] * 17)
    clip = torch.full((2,), float("nan"), device="cuda")
    B.cct_grad_norm(lst, 1e6, clip, B.alloc_norm_workspace(lst))
    want = (17 * (1024 * 4.0 + 25.0)) ** 0.5
    norm, scale = clip.tolist()
    assert abs(norm - want) <= 2.0 ** -23 * want and scale == 1.0
    B.cct_grad_scale(lst, clip, lst)                # scale 1 in place: nothing is written
    assert float(flat[-1]) == 5.0 and float(flat[1 << 23]) == 2.0
    del flat, lst
    torch.cuda.empty_cache()
