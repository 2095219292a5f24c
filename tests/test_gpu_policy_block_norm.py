"""The norms around a residual block against their formula in 64 bits, gradients against autograd on it and against differences.

Tolerances: with u = 2^-24 and D the width, a mean of squares adds at most 16 squares a thread, 5 + 5 partial sums over lanes and warps:
30 u relative; its root 15 u and 2 u of its own. n carries that and 3 roundings, r = alpha x + gate n two more, against the
size |alpha x| + |gate n|: 24 u of it. h carries 24 u of r's size over its root, the root's error 17 u and that of its mean: every r
is off by 24 u of its size, which moves the root by no more than 24 u of the largest share, below 24 u sqrt(mean size^2 / mean r^2). To
all of which half a step of the type is added (2^-8 relative in bf16, 2^-11 in f16, 2^-24 in f32; half of f16's smallest, 2^-25).
The gradients go through two such roots and two means more: each is compared within 400 u of the sum of the magnitudes of
all of its terms, taken with sizes in place of values, which the reference computes alongside; sums over N rows add the depth of
their additions, at most (N + 64) u of the sum of magnitudes.
"""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"float32": U, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
LOW = {"float32": 2.0 ** -140, "bfloat16": 2.0 ** -130, "float16": 2.0 ** -25}


@pytest.fixture(scope="module")
def nb():
    import torch
    from paper_2503_20591_b200 import binding, build as lib_build
    lib_build.build()
    assert torch.cuda.is_available()
    binding.load_library()
    return binding


def make(shape, dtype, gate, seed, pad=0, shift=0, weights="float32", gate_dtype=None):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda s: torch.randn(s, generator=gen, device="cuda")
    dt = getattr(torch, dtype)

    def table(scale):
        rows = math.prod(shape[:-1])
        buf = torch.full((rows * (shape[-1] + pad) + shift,), 7.0, dtype=dt, device="cuda")
        t = buf[shift:].view(*shape[:-1], shape[-1] + pad)[..., :shape[-1]]
        t.copy_(rand(shape) * scale)
        return t

    c = dict(residual=table(2.0), branch=table(0.5))
    gshape = {"none": None, "width": (shape[-1],), "group": (*shape[:-2], 1, shape[-1]), "row": shape}[gate]
    c["gate"] = None if gshape is None else rand(gshape).to(getattr(torch, gate_dtype or dtype))
    w = getattr(torch, weights)
    c["post_weight"], c["pre_weight"] = (1 + 0.3 * rand(shape[-1])).to(w), (1 + 0.3 * rand(shape[-1])).to(w)
    return c, table(1.0), table(0.7)


def reference(c, alpha, eps, dr, dh):
    """Values and tolerances in 64 bits, by name."""
    import torch
    x, y = c["residual"].double(), c["branch"].double()
    one = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device)
    post, pre = (one if c[n] is None else c[n].double() for n in ("post_weight", "pre_weight"))
    gate = one if c["gate"] is None else c["gate"].double()
    mean = lambda v: v.mean(-1, keepdim=True)
    root_y, eps64 = (mean(y * y) + eps) ** -0.5, eps
    y_hat = y * root_y
    n = y_hat * post
    r = alpha * x + gate * n
    size = abs(alpha) * x.abs() + (gate * n).abs()
    root_r = (mean(r * r) + eps64) ** -0.5
    r_hat, size_hat = r * root_r, size * root_r
    grow = 1 + (mean(size * size) / (mean(r * r) + eps64)).sqrt()     # how far r's error can move its root
    out = {"out": (r, 24 * U * size), "normed": (r_hat * pre, (24 * size_hat * grow + 30 * r_hat.abs()) * U * pre.abs())}
    if dr is None and dh is None:
        return out
    zero = torch.zeros_like(x)
    dr, dh = (zero if v is None else v.double() for v in (dr, dh))
    e = dh * pre
    m_r = mean(e * r_hat)
    d = dr + root_r * (e - r_hat * m_r)
    reach = size_hat * grow                                            # r^ with its error's size
    d_size = dr.abs() + root_r * grow * (e.abs() + 2 * reach * mean(e.abs() * reach))
    f, f_size = d * gate * post, d_size * (gate * post).abs()
    y_abs = y_hat.abs()
    dy = root_y * (f - y_hat * mean(f * y_hat))
    dy_size = root_y * (f_size + 2 * y_abs * mean(f_size * y_abs))
    out["residual"] = (alpha * d, 400 * U * abs(alpha) * d_size)
    out["branch"] = (dy, 400 * U * dy_size)

    def over_rows(v, s, like):
        lead = tuple(i for i in range(v.dim() - 1)) if like.dim() == 1 else tuple(i for i in range(v.dim() - 1) if like.shape[i] != v.shape[i])
        count = math.prod(v.shape[i] for i in lead) if lead else 1
        keep = like.dim() > 1
        if lead:
            v, s = v.sum(lead, keepdim=keep), s.sum(lead, keepdim=keep)
        return v, (400 + (count + 64 if lead else 0)) * U * s

    if c["gate"] is not None:
        out["gate"] = over_rows(d * n, d_size * n.abs(), c["gate"])
    out["post_weight"] = over_rows(d * gate * y_hat, d_size * gate.abs() * y_abs, post)
    out["pre_weight"] = over_rows(dh * r_hat, dh.abs() * reach, pre)
    return out


def close(name, got, ref):
    dtype = str(got.dtype)[6:]
    want, tol = ref
    bad = ~((got.double() - want).abs() <= tol * (1 + HALF[dtype]) + HALF[dtype] * want.abs() + LOW[dtype])
    assert got.shape == want.shape
    assert not bad.any(), (name, int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4], want[bad][:4], tol.expand_as(bad)[bad][:4])


NAMES = ("residual", "branch", "gate", "post_weight", "pre_weight")


def run(nb, c, alpha, eps, dr, dh, pad=0):
    import torch
    x = c["residual"]
    like = lambda t, p=0: torch.full((*t.shape[:-1], t.shape[-1] + p), -7.0, dtype=t.dtype, device="cuda")[..., :t.shape[-1]]
    out, normed, stats = like(x, pad), like(x, pad), torch.full((*x.shape[:-1], 2), -7.0, device="cuda")
    nb.nbos_policy_block_norm(*(c[n] for n in NAMES), out, normed, stats, alpha, eps)
    got = {"out": out, "normed": normed}
    if dr is not None or dh is not None:
        grads = {n: None if c[n] is None else like(c[n], pad if n in ("residual", "branch") else 0) for n in NAMES}
        nb.nbos_policy_block_norm_backward(*(c[n] for n in NAMES), stats, dr, dh, *grads.values(), residual_scale=alpha)
        got.update({n: g for n, g in grads.items() if g is not None})
    torch.cuda.synchronize()
    return got


def check(nb, c, alpha, eps, dr, dh, pad=0):
    got, want = run(nb, c, alpha, eps, dr, dh, pad), reference(c, alpha, eps, dr, dh)
    for name in got:
        close(name, got[name], want[name])
    return got


# one value; lanes of a warp, a warp, a block; 8 and 16 values a thread; odd widths; few rows, many rows
SHAPES = [(1, 1, 1), (2, 3, 2), (3, 5, 7), (1, 33, 8), (4, 64, 64), (2, 50, 65), (1, 9, 256), (2, 17, 257), (3, 40, 1000), (1, 7, 1026),
          (2, 9, 4096), (1, 5, 4097), (2, 3, 8192), (1, 3, 8194), (1, 2, 16383), (1, 2, 16384), (1, 3000, 24), (600, 3, 40), (2, 2100, 96)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("gate", ["none", "width", "group", "row"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_matches_the_formula(nb, shape, gate, dtype):
    c, dr, dh = make(shape, dtype, gate, sum(shape))
    check(nb, c, 0.9, 1e-6, dr, dh)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gate", ["width", "group", "row"])
@pytest.mark.parametrize("width,pad,shift", [(64, 8, 0), (64, 2, 2), (63, 0, 1), (1000, 24, 8), (1000, 0, 1), (4100, 2, 0), (9001, 7, 3)])
def test_any_alignment_and_types_of_weights(nb, width, pad, shift, gate, dtype):
    import torch
    for weights, gate_dtype in (("float32", "float32"), (dtype, dtype), ("float32", dtype)):
        c, dr, dh = make((3, 11, width), dtype, gate, width + pad, pad, shift, weights, gate_dtype)
        check(nb, c, 1.0, 1e-5, dr, dh, pad)
    # weights off a 16-byte boundary
    for n in ("post_weight", "pre_weight"):
        c[n] = torch.cat([torch.zeros(1, device="cuda", dtype=c[n].dtype), c[n]])[1:]
    check(nb, c, 1.0, 1e-5, dr, dh)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_what_may_be_left_out(nb, dtype):
    """Weights, either arriving gradient, outputs."""
    import torch
    c, dr, dh = make((2, 30, 200), dtype, "group", 3)
    for a, b in ((dr, None), (None, dh)):
        check(nb, c, 0.5, 1e-6, a, b)
    full = run(nb, c, 0.5, 1e-6, dr, dh)
    stats = torch.empty(2, 30, 2, device="cuda")
    args = [c[n] for n in NAMES]
    nb.nbos_policy_block_norm(*args, None, None, stats, 0.5, 1e-6)
    for i, n in enumerate(NAMES):
        g = torch.full_like(c[n], -7.0)
        nb.nbos_policy_block_norm_backward(*args, stats, dr, dh, *(g if i == j else None for j in range(5)), residual_scale=0.5)
        assert torch.equal(g, full[n]), n
    for only in ("out", "normed"):
        t = torch.full_like(c["residual"], -7.0)
        nb.nbos_policy_block_norm(*args, t if only == "out" else None, t if only == "normed" else None, None, 0.5, 1e-6)
        assert torch.equal(t, full[only])
    c["post_weight"] = c["pre_weight"] = None
    check(nb, c, -1.5, 0.0, dr, dh)


def test_written_over_the_inputs(nb):
    import torch
    for shape in ((2, 30, 200), (3, 2048), (5, 9000), (700, 333), (900, 1001), (5, 9001)):
        c, dr, dh = make(shape, "bfloat16", "row", 4)
        want = run(nb, c, 0.5, 1e-6, dr, dh)
        stats = torch.empty(*shape[:-1], 2, device="cuda")
        a, b = dr.clone(), dh.clone()
        nb.nbos_policy_block_norm(*(c[n] for n in NAMES), None, None, stats, 0.5, 1e-6)
        nb.nbos_policy_block_norm_backward(*(c[n] for n in NAMES), stats, a, b, a, b, residual_scale=0.5)
        assert torch.equal(a, want["residual"]) and torch.equal(b, want["branch"])
        nb.nbos_policy_block_norm(*(c[n] for n in NAMES), c["residual"], c["branch"], None, 0.5, 1e-6)
        assert torch.equal(c["residual"], want["out"]) and torch.equal(c["branch"], want["normed"])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("gate", ["none", "group", "row"])
@pytest.mark.parametrize("width", [24, 200, 333, 1000, 5001])
def test_rows_that_start_anywhere_give_the_same_bits(nb, width, gate, dtype):
    """The same values in tables on 16-byte boundaries and off them, many rows a block: a row's arithmetic is the same. (Sums over rows go
    by how many blocks there are room for, which differs: they are compared with the formula.)"""
    import torch
    shape = (6, 2500 if width < 1000 else 300, width)
    c, dr, dh = make(shape, dtype, gate, width)
    off, dr2, dh2 = make(shape, dtype, gate, width, pad=3, shift=1)

    def aligned(t):
        per16 = 16 // t.element_size()
        room = torch.zeros((*t.shape[:-1], (width + per16 - 1) // per16 * per16), dtype=t.dtype, device="cuda")
        room[..., :width] = t
        return room[..., :width]

    want = run(nb, {n: aligned(t) if t is not None and t.dim() == 3 and t.shape == shape else t for n, t in c.items()}, 0.7, 1e-6, aligned(dr), aligned(dh),
               (-width) % (16 // dr.element_size()))
    got = run(nb, off, 0.7, 1e-6, dr2, dh2, 5)
    rows = [n for n in want if n in ("out", "normed", "residual", "branch") or (n == "gate" and gate == "row")]
    assert [n for n in rows if not torch.equal(got[n], want[n])] == []
    ref = reference(off, 0.7, 1e-6, dr2, dh2)
    for n in set(want) - set(rows):
        close(n, got[n], ref[n])
        close(n, want[n], ref[n])


def test_rows_of_zeros_nan_and_infinity_stay_alone(nb):
    import torch
    for width in (64, 3000):
        c, dr, dh = make((1, 40, width), "float32", "row", 5)
        c["branch"][0, 3] = 0
        c["residual"][0, 4] = c["branch"][0, 4] = 0
        got = check(nb, c, 1.0, 1e-6, dr, dh)
        c["residual"][0, 7, 1], c["branch"][0, 8, 2], c["branch"][0, 9, 5] = math.nan, math.nan, math.inf
        bad = run(nb, c, 1.0, 1e-6, dr, dh)
        rest = [i for i in range(40) if i not in (7, 8, 9)]
        for n in ("out", "normed", "residual", "branch"):
            assert torch.equal(bad[n][0, rest], got[n][0, rest]) and not bad[n][0, 7:10].isfinite().all()
    # without eps a row of zeros has no norm: NaN, in that row alone
    c["residual"][0, 7:10], c["branch"][0, 7:10] = 1.0, 1.0
    got = run(nb, c, 1.0, 0.0, None, None)
    assert got["normed"][0, 4].isnan().all() and got["out"][0, 3].isnan().all() and got["out"][0, 5:].isfinite().all()


def test_differences(nb):
    """Autograd's gradient along random directions against differences in 64 bits."""
    import torch
    from paper_2503_20591_b200 import policy
    c, dr, dh = make((3, 20, 48), "float32", "group", 6)
    leaves = {n: c[n].clone().requires_grad_(True) for n in NAMES}
    out, normed = policy.block_norm(*leaves.values(), residual_scale=0.8, eps=1e-6)
    ((out * dr).sum() + (normed * dh).sum()).backward()

    def value(v):
        r = reference(v, 0.8, 1e-6, None, None)
        return float((r["out"][0] * dr).sum() + (r["normed"][0] * dh).sum())

    for n in NAMES:
        d = torch.randn_like(c[n]).double()
        e = 1e-5
        at = lambda s: dict(c, **{n: c[n].double() + s * d})
        slope = (value(at(e)) - value(at(-e))) / (2 * e)
        got = float((leaves[n].grad.double() * d).sum())
        size = float((leaves[n].grad.double().abs() * d.abs()).sum())
        assert abs(got - slope) <= 1e-5 * size + 1e-6, n     # 32-bit gradients: below 100 u of their size; differences: e^2


def test_autograd_of_parts(nb):
    import torch
    from paper_2503_20591_b200 import policy
    c, dr, dh = make((4, 10, 64), "bfloat16", "width", 7)
    want = run(nb, c, 1.0, 1e-6, dr, None)
    leaves = [c[n].clone().requires_grad_(n != "branch") for n in NAMES]
    out, normed = policy.block_norm(*leaves)
    out.backward(dr)                                   # the normed output is not used
    assert torch.equal(leaves[0].grad, want["residual"]) and leaves[1].grad is None and torch.equal(leaves[2].grad, want["gate"])
    out, normed = policy.block_norm(*(t.detach() for t in leaves))
    assert not out.requires_grad
    x = c["residual"].clone().requires_grad_(True)     # a gradient that is no table: expanded from one value
    policy.block_norm(x, c["branch"])[0].sum().backward()
    assert torch.equal(x.grad, torch.ones_like(x))


def test_empty(nb):
    import torch
    e = lambda *s: torch.full(s, -7.0, device="cuda")
    g = [e(0, 8), e(0, 8), e(8), e(8), e(8)]
    nb.nbos_policy_block_norm(e(0, 8), e(0, 8), e(8), e(8), e(8), e(0, 8), e(0, 8), e(0, 2))
    nb.nbos_policy_block_norm_backward(e(0, 8), e(0, 8), e(8), e(8), e(8), e(0, 2), e(0, 8), e(0, 8), *g)
    assert all((t == 0).all() for t in g)


def test_same_bits_every_time_streams_and_graphs(nb):
    import torch
    from paper_2503_20591_b200 import policy
    for shape, gate in (((5, 700, 96), "group"), ((1, 900, 2048), "width"), ((1500, 2, 64), "group")):
        c, dr, dh = make(shape, "bfloat16", gate, 8)
        d, dr2, dh2 = make(shape, "bfloat16", gate, 9)
        first, second = run(nb, c, 1.0, 1e-6, dr, dh), run(nb, d, 1.0, 1e-6, dr2, dh2)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = run(nb, c, 1.0, 1e-6, dr, dh)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(again[n], first[n]) for n in first)
        leaves = [c[n].clone().requires_grad_(True) for n in NAMES]
        alive = policy.block_norm(*leaves)[0].sum()      # an eager graph of the same leaves
        graphs = []
        for _ in range(2):
            outs = [torch.empty_like(c["residual"]) for _ in range(2)]
            stats, grads = torch.empty(*shape[:-1], 2, device="cuda"), [torch.empty_like(t) for t in leaves]
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                args = [t.detach() for t in leaves]
                nb.nbos_policy_block_norm(*args, *outs, stats)
                nb.nbos_policy_block_norm_backward(*args, stats, dr, dh, *grads)
            graphs.append((graph, outs + grads))
        with torch.no_grad():
            for t, n in zip(leaves, NAMES):
                t.copy_(d[n])
            dr.copy_(dr2), dh.copy_(dh2)
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, got in graphs:
            assert all(torch.equal(g, second[n]) for g, n in zip(got, ("out", "normed", *NAMES)))
        del alive


def test_the_binding_refuses_wrong_tensors(nb):
    import torch
    x, w = torch.ones(2, 3, 8, device="cuda"), torch.ones(8, device="cuda")
    call = lambda **kw: nb.nbos_policy_block_norm(**dict(dict(residual=x, branch=x, gate=None, post_weight=w, pre_weight=w, out_residual=x.clone()), **kw))
    for kw, error, word in ((dict(residual=x.double()), TypeError, "float32"), (dict(residual=x.cpu()), ValueError, "cuda"),
                            (dict(branch=x[:1]), ValueError, "shape"), (dict(branch=x.half()), ValueError, "type"), (dict(branch=None), ValueError, "None"),
                            (dict(gate=x[:, :2]), ValueError, "gate"), (dict(gate=torch.ones(1, 3, 8, device="cuda")), ValueError, "gate"),
                            (dict(gate=w[:4]), ValueError, "gate"), (dict(gate=w.half()), TypeError, "gate"), (dict(gate=w.cpu()), ValueError, "live on"),
                            (dict(post_weight=w[:7]), ValueError, "hold"), (dict(pre_weight=w.double()), TypeError, "pre_weight"),
                            (dict(out_residual=x[..., :4]), ValueError, "shape"), (dict(out_stats=w), ValueError, "hold")):
        with pytest.raises(error, match=word):
            call(**kw)
