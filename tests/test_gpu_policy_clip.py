"""The global norm over many tensors and clipping by it, against the formula in 64 bits.

Tolerances: a norm is the root of sums of squares in which a thread adds at most 64 values in 32 bits, 16 to a running sum and
four of those: relative 20 2^-24 of the sum, half of that of its root, and the rounding to a float, 2^-24: 11 2^-24. A
clipped value carries that of the factor, its rounding to 32 bits and the product's (13 2^-24 together) and half a step of its
type: 2^-8 in bf16, 2^-11 in f16 (half of 2^-24 below its normal numbers), 2^-24 in f32.
"""
from __future__ import annotations

import math

import pytest

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
HALF = {"float32": E, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}
INF = math.inf


@pytest.fixture(scope="module")
def nb():
    import torch
    from paper_2503_20591_b200 import binding, build as lib_build
    lib_build.build()
    assert torch.cuda.is_available()
    binding.load_library()
    return binding


def make(sizes, dtypes, seed, shift=0, scale=1.0):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        dtype = getattr(torch, dtypes[i % len(dtypes)])
        buf = torch.zeros(n + shift, dtype=dtype, device="cuda")
        buf[shift:] = (torch.randn(n, generator=gen, device="cuda") * scale * 4.0 ** (i % 3)).to(dtype)
        out.append(buf[shift:])
    return out


def formula(tensors, max_norm, kind):
    """norm and factor in 64 bits."""
    import torch
    if kind == "inf":
        norm = max(float(m) for m in torch.stack([t.abs().max().double() for t in tensors if t.numel()]))
    else:
        norm = math.sqrt(sum(float((torch.cat(same).double() ** 2).sum()) for same in
                             ([t.reshape(-1) for t in tensors if t.dtype == d] for d in {t.dtype for t in tensors})))
    return norm, min(1.0, max_norm / (norm + 1e-6))


def check(nb, tensors, max_norm, kind="2", in_place=False):
    import torch
    by_type = {}
    for i, t in enumerate(tensors):
        by_type.setdefault(t.dtype, []).append(i)
    values = {d: torch.cat([tensors[i] for i in at]).double() for d, at in by_type.items()}
    # max_norm is a 32-bit float at the C entry: 1.5e40 arrives there as infinity
    want, factor = formula(tensors, float(torch.tensor(max_norm, dtype=torch.float32)), kind)
    norm = torch.full((), -7.0, device="cuda")
    outs = tensors if in_place else [torch.full_like(t, -7.0) for t in tensors]
    nb.nbos_policy_clip(tensors, max_norm, norm, outs, norm_kind=nb.NBOS_NORM_2 if kind == "2" else nb.NBOS_NORM_INF)
    tol = (11 if kind == "2" else 1) * E
    if want > torch.finfo(torch.float32).max:   # 6.2e38, say: the nearest 32-bit float is infinity
        assert float(norm) == INF
    else:
        assert abs(float(norm) - want) <= tol * want, (float(norm), want)
    for dtype, x in values.items():
        got = torch.cat([outs[i] for i in by_type[dtype]])
        half = HALF[str(dtype)[6:]]
        low = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}[dtype]
        err = (got.double() - x * factor).abs() - (13 * E + half * (1 + 13 * E)) * (x * factor).abs() - low
        assert got.numel() == 0 or float(err.max()) <= 0
    return norm, outs


# one value; around a 16-byte piece, a thread's and a block's chunk (8,192 16-bit values), one cluster's share (32 chunks), beyond
SIZES = [[1], [3, 1, 2], [7, 8, 9], [8191, 8192, 8193], [1 << 18, 5], [(1 << 18) + 1], [1 << 20, 1, 77777], [0, 5, 0], [1] * 64, [1] * 65,
         [13] * 1100, [13] * 1101 + [4001], [100] * 2500, [9_000_001]]


@pytest.mark.parametrize("kind", ["2", "inf"])
@pytest.mark.parametrize("dtypes", [["float32"], ["bfloat16"], ["float16"], ["bfloat16", "float32", "float16"]])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_matches_the_formula(nb, sizes, dtypes, kind):
    import torch
    tensors = make(sizes, dtypes, len(sizes) + max(sizes))
    norm, _ = formula(tensors, 1.0, kind)
    for share in (0.37, 5.0):
        check(nb, tensors, share * norm, kind)
    before = [t.clone() for t in tensors]
    check(nb, tensors, 5.0 * norm, kind, in_place=True)
    assert all(torch.equal(a, b) for a, b in zip(tensors, before))
    check(nb, tensors, 0.37 * norm, kind, in_place=True)


@pytest.mark.parametrize("dtype,shift", [("float32", 1), ("float32", 3), ("bfloat16", 1), ("float16", 7), ("bfloat16", 8)])
def test_tensors_that_start_anywhere(nb, dtype, shift):
    import torch
    tensors = make([5, 8195, 300_001], [dtype], 1, shift)
    norm = formula(tensors, 1.0, "2")[0]
    check(nb, tensors, 0.3 * norm)
    # only the outputs off their boundary, with what lies around them left alone
    aligned = [t.clone() for t in tensors]
    bufs = [torch.full((t.numel() + 2 * shift,), -7.0, dtype=t.dtype, device="cuda") for t in tensors]
    outs = [b[shift:-shift] for b in bufs]
    nb.nbos_policy_clip(aligned, 0.3 * norm, None, outs)
    want = [torch.empty_like(t) for t in aligned]
    nb.nbos_policy_clip(aligned, 0.3 * norm, None, want)
    for b, o, w in zip(bufs, outs, want):
        assert torch.equal(o, w) and (b[:shift] == -7.0).all() and (b[-shift:] == -7.0).all()


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-22, 1e-10, 1e10, 1e22, 1e37])
def test_squares_beyond_32_bits(nb, scale):
    """Values whose squares overflow a float or vanish, among zeros and among ordinary ones."""
    import torch
    for n in (200, 500_000):
        tensors = make([n, n], ["float32", "bfloat16"], 2, scale=scale)
        tensors[0][::2] = 0
        norm, _ = formula(tensors, 1.0, "2")
        check(nb, tensors, max(0.5 * norm, 1e-38))
        mixed = [tensors[0], torch.ones(7, device="cuda")]
        check(nb, mixed, 0.5)


def test_norm_beyond_a_float(nb):
    """The norm overflows to infinity; the factor, taken in 64 bits, is still right."""
    import torch
    t = torch.full((100,), 3e38, device="cuda")
    norm, out = torch.empty((), device="cuda"), torch.empty_like(t)
    nb.nbos_policy_clip([t], 1e38, norm, [out])
    assert float(norm) == INF
    torch.testing.assert_close(out, torch.full_like(t, 1e37), rtol=2 * E, atol=0.0)


@pytest.mark.parametrize("n", [50, 2_000_000])
@pytest.mark.parametrize("kind", ["2", "inf"])
def test_nan_and_infinity(nb, n, kind):
    import torch
    k = nb.NBOS_NORM_2 if kind == "2" else nb.NBOS_NORM_INF
    norm = torch.empty((), device="cuda")
    t = torch.ones(n, device="cuda")
    t[n // 3] = -INF
    out = torch.empty_like(t)
    nb.nbos_policy_clip([t], 1.0, norm, [out], norm_kind=k)
    assert float(norm) == INF and out[n // 3].isnan() and int((out == 0).sum()) == n - 1
    t[n // 2] = math.nan
    nb.nbos_policy_clip([t], 1.0, norm, [out], norm_kind=k)
    assert norm.isnan() and out.isnan().all()


def test_norm_alone_empty_and_zero(nb):
    import torch
    norm = torch.full((), -7.0, device="cuda")
    nb.nbos_policy_clip([], 1.0, norm)
    assert float(norm) == 0.0
    nb.nbos_policy_clip([torch.empty(0, device="cuda")], 1.0, norm.fill_(-7.0))
    assert float(norm) == 0.0
    z = torch.zeros(1_000_000, device="cuda")
    check(nb, [z], 1.0)
    tensors = make([1000, 3_000_000], ["bfloat16"], 3)
    before = [t.clone() for t in tensors]
    nb.nbos_policy_clip(tensors, 0.0, norm)
    assert abs(float(norm) - formula(tensors, 1.0, "2")[0]) <= 11 * E * float(norm)
    assert all(torch.equal(a, b) for a, b in zip(tensors, before))
    nb.nbos_policy_clip(tensors, 0.0, None, tensors)
    assert all((t == 0).all() for t in tensors)
    out = [torch.empty_like(t) for t in before]
    nb.nbos_policy_clip(before, INF, None, out)
    assert all(torch.equal(a, b) for a, b in zip(out, before))


def test_offsets_beyond_31_bits(nb):
    import torch
    t = torch.zeros((1 << 31) + 77, dtype=torch.bfloat16, device="cuda")
    t[-5:] = 2.0
    t[5] = 1.0
    norm = torch.empty((), device="cuda")
    nb.nbos_policy_clip([t], math.sqrt(21.0) / 2, norm, [t][:1])
    assert abs(float(norm) - math.sqrt(21.0)) <= 11 * E * float(norm)
    assert (t[-5:] == 1.0).all() and float(t[5]) == 0.5


def test_same_bits_every_time_and_in_graphs(nb):
    import torch
    tensors = make([5_000_000, 17, 400_000], ["float32", "bfloat16"], 4)
    small = make([64, 64 * 64], ["float32"], 5)
    for group in (tensors, small):
        outs, norm = [torch.empty_like(t) for t in group], torch.empty((), device="cuda")
        nb.nbos_policy_clip(group, 3.0, norm, outs)
        want = [norm.clone()] + [o.clone() for o in outs]
        graphs = []
        for _ in range(2):
            o, n = [torch.empty_like(t) for t in group], torch.empty((), device="cuda")
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                nb.nbos_policy_clip(group, 3.0, n, o)
            graphs.append((graph, [n] + o))
        for graph, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, got in graphs:
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_clip_gradients(nb):
    import torch
    from paper_2503_20591_b200 import policy
    net = torch.nn.Sequential(torch.nn.Linear(40, 50), torch.nn.Linear(50, 60)).cuda()
    unused = torch.nn.Parameter(torch.ones(3, device="cuda"))
    net(torch.randn(20, 40, device="cuda")).square().sum().backward()
    params = [*net.parameters(), unused]
    before = [p.grad.clone() for p in net.parameters()]
    norm = policy.clip_gradients(params, 0.5)
    want, factor = formula(before, 0.5, "2")
    assert abs(float(norm) - want) <= 11 * E * want and unused.grad is None
    for p, b in zip(net.parameters(), before):
        torch.testing.assert_close(p.grad.double(), b.double() * factor, rtol=14 * E, atol=0.0)
    assert float(policy.clip_gradients(unused, 1.0)) == 0.0
    # a shared parameter counts once; a gradient that is laid out otherwise is clipped as it lies
    p, q = torch.nn.Parameter(torch.ones(3, 5, device="cuda")), torch.nn.Parameter(torch.ones(4, 6, device="cuda"))
    p.grad, q.grad = torch.full((3, 5), 2.0, device="cuda"), torch.full((6, 4), 3.0, device="cuda").t()
    norm = policy.clip_gradients([p, q, p], 1.0)
    want = math.sqrt(15 * 4.0 + 24 * 9.0)
    assert abs(float(norm) - want) <= 11 * E * want and not q.grad.is_contiguous()
    torch.testing.assert_close(p.grad, torch.full_like(p.grad, 2.0 / want), rtol=1e-6, atol=0.0)
    torch.testing.assert_close(q.grad, torch.full_like(q.grad, 3.0 / want), rtol=1e-6, atol=0.0)
    assert float(policy.clip_gradients(net.parameters(), 1.0, math.inf)) == max(float(p.grad.abs().max()) for p in net.parameters())


def test_the_binding_refuses_wrong_tensors(nb):
    import torch
    x, norm = torch.ones(4, 4, device="cuda"), torch.empty((), device="cuda")
    for bad, error, word in (([x, x.cpu()], ValueError, "live on"), ([x.t()[:, 1:]], ValueError, "contiguous"), ([x.double()], TypeError, "float64"),
                             ([x, 3.0], TypeError, "get_device"), ([x.cpu()], ValueError, "cuda")):
        with pytest.raises(error, match=word):
            nb.nbos_policy_clip(bad, 1.0, norm)
    with pytest.raises(ValueError, match="twice"):
        nb.nbos_policy_clip([x, x], 1.0, norm, [x, x])
    two = [x, x]
    with pytest.raises(ValueError, match="twice"):
        nb.nbos_policy_clip(two, 1.0, norm, two)
    nb.nbos_policy_clip(two, 1.0, norm)   # reading it twice is a sum like any other
    assert abs(float(norm) - math.sqrt(32.0)) <= 11 * E * 6
    empty = torch.empty(0, device="cuda")
    nb.nbos_policy_clip([empty, x, empty], 1.0, norm, [empty, x.clone(), empty])
    for outs, word in (([x, x], "each"), ([x[:2]], "sizes"), ([x.half()], "sizes"), ([x.cpu()], "live on")):
        with pytest.raises(ValueError, match=word):
            nb.nbos_policy_clip([x], 1.0, norm, outs)
    with pytest.raises(nb.NbosError, match="max_norm"):
        nb.nbos_policy_clip([x], -1.0, norm)


def test_outputs_that_are_other_inputs(nb):
    import torch
    x, y, z = (torch.ones(32, device="cuda") for _ in range(3))
    norm = torch.empty((), device="cuda")
    for tensors, outs in (([x, y], [y, x]), ([x, y], [z, x]), ([x, x], [x, z])):
        with pytest.raises(ValueError, match="another of the tensors"):
            nb.nbos_policy_clip(tensors, 1.0, norm, outs)
    nb.nbos_policy_clip([x, y], 1.0, norm, [x, z])   # one in place, one not
    assert torch.equal(x, z) and float(x[0]) < 1 and (y == 1).all()
