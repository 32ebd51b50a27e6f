"""The global norm of many gradients and clipping, against 64 bits.

Bars: the squares of float32 numbers are exact in 64 bits and their sum is good to n 2^-53, so the norm is the exact one rounded to float32
once.  A clipped element is the product with a factor rounded to float32 (2^-24), itself rounded in float32 (2^-24) and to its
type (half a step)."""
import math

import pytest
import torch

import paper_2602_17206_amd as pkg

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
LEAST = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -126}
INF, NAN = float("inf"), float("nan")


def norm_of(tensors):
    return math.sqrt(sum(float(t.double().square().sum()) for t in tensors))


def check(grads, max_norm, outs=None):
    before = [g.clone() for g in grads]
    want = norm_of(before)
    norm = pkg.sdtw_gradient_clip(grads, max_norm, out=outs)
    assert norm.shape == () and norm.dtype == torch.float32
    assert abs(float(norm) - want) <= 2.0 ** -24 * want * 1.001 + 2.0 ** -149
    factor = min(1.0, max_norm / want) if want else 1.0
    for b, g, o in zip(before, grads, grads if outs is None else outs):
        if outs is not None:
            assert torch.equal(b, g)
        x = b.double().reshape(-1) if outs is not None and b.shape != o.shape else b.double()
        bar = (2.1 * 2.0 ** -24 + 1.001 * HALF_ULP[o.dtype]) * (x * factor).abs() + LEAST[o.dtype]
        if factor == 1.0 and o.dtype == b.dtype:
            assert torch.equal(o.reshape(b.shape), b)
        assert ((o.double().reshape(x.shape) - x * factor).abs() <= bar).all()
    return norm


def some(sizes, kinds, seed=0, size=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(size * torch.randn(n, generator=gen, device="cuda")).to(TYPES[kinds[i % len(kinds)]]) for i, n in enumerate(sizes)]


@pytest.mark.parametrize("kinds", [["f32"], ["f16"], ["bf16"], ["f32", "bf16", "f16"]])
@pytest.mark.parametrize("share", [0.1, 0.999, 1.001, 100.0])
@pytest.mark.parametrize("sizes", [[1], [7], [8192], [8191, 8193, 1, 2, 3], [0, 5, 0, 100000, 0], [3 * 8192 + 5], [1000003, 17]])
def test_clipping(sizes, share, kinds):
    grads = some(sizes, kinds)
    check(grads, share * norm_of(grads))


@pytest.mark.parametrize("out", sorted(TYPES))
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("share", [0.3, 3.0])
def test_clipping_into_other_tensors(kind, out, share):
    sizes = [1, 3, 8, 100, 8192, 20001, 0, 300007]
    grads = some(sizes, [kind])
    room = torch.full((sum(sizes) + 2 * len(sizes),), 7.0, dtype=TYPES[out], device="cuda")
    outs, at, used = [], 1, torch.zeros(room.shape, dtype=torch.bool, device="cuda")
    for n in sizes:  # one behind the other, from odd elements on
        outs.append(room[at:at + n])
        used[at:at + n] = True
        at += n + 1
    check(grads, share * norm_of(grads), outs)
    assert (room[~used] == 7.0).all()


@pytest.mark.parametrize("count", [127, 128, 129, 600])
def test_many_tensors(count):
    check(some([(i * 37) % 5000 + (i % 9 == 0) * 20000 for i in range(count)], ["bf16", "f32"]), 1.0)
    check(some([3] * count, ["f16"]), 1.0)


def test_large_tensors():
    grads = some([40000003, 100, 33000001], ["bf16", "f32"])
    check(grads, 10.0)


def test_views_that_begin_anywhere_and_other_orders_of_the_dimensions():
    room = some([50000], ["bf16"])[0]
    check([room[1:20000], room[20003:20010], room[30001:]], 0.5)
    assert torch.equal(room[20000:20003], some([50000], ["bf16"])[0][20000:20003])
    x = some([24000], ["f32"])[0].view(20, 30, 40)
    check([x.permute(2, 0, 1), x.new_ones(7, 1, 5).transpose(0, 2)], 0.5)
    y = torch.empty((20, 30, 40), dtype=torch.bfloat16, device="cuda").permute(2, 0, 1)
    check([x.permute(2, 0, 1)], 0.5, [y])
    check([x], 0.25, [torch.empty(24000, device="cuda")])  # (as many elements)


@pytest.mark.parametrize("size", [1e-30, 1e-20, 1e20, 1e30])
def test_gradients_of_any_size(size):
    """Squares beyond float32 on either side."""
    grads = some([5000, 77], ["f32", "bf16"], size=size)
    check(grads, 0.01 * size)
    check(grads, 100.0 * size)


@pytest.mark.parametrize("sizes", [[2], [60000, 500]])
@pytest.mark.parametrize("out", sorted(TYPES))
@pytest.mark.parametrize("max_norm", [1.0, 1e-6, 1e-10, 2.0 ** -100, 1e20])
def test_norms_beyond_float32(max_norm, out, sizes):
    """Every element is finite, their norm is above float32's largest number: that is what is returned, and they are clipped by the norm itself.
    Where the factor is below 2^-126 it has a power of two of its own, so that it keeps its digits.  Bars as above; float16's results may
    be beyond its largest number."""
    grads = [(3e38 * torch.sign(t)).float() for t in some(sizes, ["f32"])]
    want = norm_of(grads)
    assert want > torch.finfo(torch.float32).max
    outs = [torch.empty(g.shape, dtype=TYPES[out], device="cuda") for g in grads]
    norm = pkg.sdtw_gradient_clip(grads, max_norm, out=outs)
    assert float(norm) == torch.finfo(torch.float32).max
    assert float(pkg.sdtw_gradient_norm(grads)) == torch.finfo(torch.float32).max
    for g, o in zip(grads, outs):
        x = g.double() * (max_norm / want)
        bar = (2.1 * 2.0 ** -24 + 1.001 * HALF_ULP[o.dtype]) * x.abs() + LEAST[o.dtype]
        beyond = x.abs() > torch.finfo(o.dtype).max
        assert torch.equal(o[beyond].double(), INF * torch.sign(x[beyond]))
        assert ((o.double() - x).abs() <= bar)[~beyond].all()


@pytest.mark.parametrize("max_norm", [1e-9, 1e-30])
def test_factors_below_the_normal_numbers(max_norm):
    grads = some([5000, 77], ["f32", "bf16"], size=1e32)
    check(grads, max_norm)


@pytest.mark.parametrize("bad", [INF, -INF, NAN])
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("n", [3000, 90000])
def test_what_is_not_finite_is_passed_on(n, kind, bad):
    grads = some([n, 50], [kind])
    grads[0][n // 2:n // 2 + 3] = bad
    before = [g.clone() for g in grads]
    outs = [torch.zeros_like(g) for g in grads]
    norms = [pkg.sdtw_gradient_clip(grads, 1.0, out=outs), pkg.sdtw_gradient_clip(grads, 1.0)]
    for norm in norms:
        assert torch.isnan(norm) if bad != bad else float(norm) == INF
    for b, g, o in zip(before, grads, outs):
        for after in (g, o):
            assert torch.equal(torch.isnan(after), torch.isnan(b)) and torch.equal(after[~torch.isnan(b)], b[~torch.isnan(b)])


@pytest.mark.parametrize("bad", [INF, -INF, NAN])
@pytest.mark.parametrize("kind", sorted(TYPES))
def test_a_norm_that_is_not_finite_leaves_the_gradients(kind, bad):
    grads = some([9000, 50], [kind])
    grads[0][8200] = bad
    before = [g.clone() for g in grads]
    norm = pkg.sdtw_gradient_clip(grads, 1.0)
    assert not torch.isfinite(norm)
    outs = [torch.zeros_like(g) for g in grads]
    pkg.sdtw_gradient_clip(grads, 1.0, out=outs)
    for b, g, o in zip(before, grads, outs):
        assert torch.equal(torch.nan_to_num(b), torch.nan_to_num(g)) and torch.equal(torch.nan_to_num(b), torch.nan_to_num(o))


def test_edges_of_the_largest_norm():
    grads = some([100, 9000], ["f32"])
    want = norm_of(grads)
    before = [g.clone() for g in grads]
    assert abs(float(pkg.sdtw_gradient_norm(grads)) - want) <= 2.0 ** -24 * want * 1.001
    check(grads, INF)
    for b, g in zip(before, grads):
        assert torch.equal(b, g)
    pkg.sdtw_gradient_clip(grads, 0.0)
    assert all((g == 0).all() for g in grads)
    assert float(pkg.sdtw_gradient_clip(grads, 0.0)) == 0.0 and float(pkg.sdtw_gradient_clip(grads, 1.0)) == 0.0
    norm = torch.full((), 5.0, device="cuda")
    assert pkg.sdtw_gradient_clip([], 1.0, norm=norm) is norm and float(norm) == 0.0
    assert float(pkg.sdtw_gradient_norm([torch.empty(0, device="cuda")])) == 0.0
    outs = [torch.zeros_like(g) for g in before]
    pkg.sdtw_gradient_clip(before, INF, out=outs)  # copied
    assert all(torch.equal(a, b) for a, b in zip(before, outs))


def test_the_same_gradients_give_the_same_bits():
    grads = some([1000003, 333, 8192 * 40] * 60, ["bf16", "f32"])
    first, outs = None, [torch.empty_like(g) for g in grads]
    for _ in range(4):
        norm = pkg.sdtw_gradient_clip(grads, 1.0, out=outs)
        now = [norm] + [o.clone() for o in outs]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
        first = now


def test_clipping_in_a_graph():
    grads = some([9000, 77, 100001], ["bf16", "f32"])
    gen = torch.Generator(device="cuda").manual_seed(1)
    pkg.sdtw_gradient_clip(grads, 1.0)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = pkg.sdtw_gradient_clip(grads, 1.0)
    for step in range(4):
        fresh = [torch.randn(g.shape, generator=gen, device="cuda").to(g.dtype) * 10.0 ** -step for g in grads]
        for g, f in zip(grads, fresh):
            g.copy_(f)
        graph.replay()
        other = pkg.sdtw_gradient_clip(fresh, 1.0)
        assert torch.equal(norm, other) and all(torch.equal(a, b) for a, b in zip(grads, fresh))
        torch.cuda.synchronize()


def test_clipping_on_the_stream_it_is_given():
    grads = some([100001] * 5, ["f32"])
    want = [g.clone() for g in grads]
    pkg.sdtw_gradient_clip(want, 1.0)
    late = [torch.zeros_like(g) for g in grads]
    busy = torch.randn((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            busy = busy @ busy * 1e-3
        for a, b in zip(late, grads):
            a.copy_(b)
    pkg.sdtw_gradient_clip(late, 1.0, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(late, want))


def test_refusals():
    g = some([100], ["f32"])[0]
    h = some([100], ["f16"])[0]
    for grads, kw in [([g, g.cpu()], {}), ([g.double()], {}), ([], {}), ([g], dict(out=[])), ([g], dict(out=[h[:50]])), ([g.view(10, 10)[:, :5]], {}),
                      ([g.view(10, 10).t()], dict(out=[g.new_empty(10, 10)])), ([g[:1].expand(5)], {}), ([g], dict(norm=h[0])),
                      ([g], dict(norm=g[:1]))]:
        with pytest.raises(ValueError):
            pkg.sdtw_gradient_clip(grads, 1.0, **kw)
    before = g.clone()
    for grads, kw in [([g, g], {}), ([g[:60], g[50:]], {}), ([g[:50], g[50:]], dict(out=[g[50:], g[:50]])), ([g[:50]], dict(out=[g[10:60]])),
                      ([g[:50], h[:50]], dict(out=[torch.empty_like(g[:50]), g[:50]])), ([h[:50]], dict(out=[h.view(torch.bfloat16)[:50]]))]:
        with pytest.raises(pkg.SdtwError):
            pkg.sdtw_gradient_clip(grads, 1.0, **kw)
    for bad in (-1.0, NAN, -INF):
        with pytest.raises(pkg.SdtwError):
            pkg.sdtw_gradient_clip([g], bad)
    small = pkg.Workspace(256)
    with pytest.raises(pkg.SdtwError):
        pkg.sdtw_gradient_clip([g], 1.0, workspace=small)
    assert torch.equal(g, before)
    both = [torch.empty_like(g), torch.empty_like(g)]
    norm = pkg.sdtw_gradient_clip([g, g], 1.0, out=both)  # what is only read may be read twice
    assert abs(float(norm) - math.sqrt(2.0) * norm_of([g])) < 1e-5
