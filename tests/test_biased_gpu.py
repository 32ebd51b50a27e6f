"""Soft-DTW under a learned position penalty against the float64 oracle on the cost matrix written out here, and the
small training example that runs the operators together.  Bars: the path's own (1e-4 relative for the values, 1e-3 of the
largest entry for gradients), the table's gradient as one of them."""
import numpy as np
import pytest
import torch

import oracle
import paper_2602_17206_amd as pkg
from paper_2602_17206_amd import binding
from paper_2602_17206_amd.workloads import normal_pairs, ragged_lengths

pytestmark = pytest.mark.gpu


def bucket_line(lo, hi, buckets, D, two_sided):
    """bucket of r = lo .. hi - 1, from the library's whole-number starts (held against whole numbers elsewhere)"""
    first = np.array(pkg.sdtw_position_bias_starts(buckets, D, two_sided))
    r = np.arange(lo, hi)
    d = np.abs(r) if two_sided else np.maximum(0, -r)
    u = np.searchsorted(first, d, side="right") - 1
    return u + (buckets // 2) * (r > 0) if two_sided else u


@pytest.mark.parametrize("B,H,N,M,D,gamma,extra", [
    (2, 1, 1, 1, 3, 1.0, {}), (4, 2, 40, 55, 8, 1.0, {}), (6, 3, 130, 97, 16, 0.1, {}), (3, 3, 64, 300, 200, 0.5, {}),
    (4, 1, 150, 160, 20, 0.1, {"bandwidth": 30}), (4, 2, 200, 170, 8, 0.5, {"ragged": True}), (4, 2, 220, 190, 8, 0.1, {"min_memory": True}),
    (70, 1, 800, 790, 4, 0.5, {"check": 3}),  # too many bands for the tables of both sweeps: the recomputing sweep
])
@pytest.mark.parametrize("two_sided", [True, False])
def test_values_and_gradients(B, H, N, M, D, gamma, extra, two_sided):
    x, y = normal_pairs(31, B, N, M, D)
    rng = np.random.default_rng(B + N)
    buckets, far = 16, 60
    table = np.abs(rng.standard_normal((H, buckets))).astype(np.float32) * 2
    table[:, 3] = -1.0  # counts as 0
    g = rng.uniform(0.5, 2.0, B).astype(np.float32)
    xl = yl = None
    if extra.get("ragged"):
        xl, yl = ragged_lengths(1, B, N), ragged_lengths(2, B, M)
    to = lambda a: None if a is None else torch.from_numpy(a).cuda()  # noqa: E731
    xd, yd, td, gd = to(x), to(y), to(table), to(g)
    kw = {k: v for k, v in extra.items() if k in ("bandwidth", "min_memory")}
    value, state, ws = pkg.sdtw_forward_biased(xd, yd, td, gamma, max_distance=far, two_sided=two_sided, offset=2, x_len=to(xl), y_len=to(yl), **kw)
    dx, dy, dt, E = pkg.sdtw_backward_biased(state, xd, yd, td, ws, grad_value=gd, x_len=to(xl), y_len=to(yl), want_E=True)
    assert binding.workspace_status(ws) == 0
    value2, state2, ws2 = pkg.sdtw_forward_biased(xd, yd, td, gamma, max_distance=far, two_sided=two_sided, offset=2, x_len=to(xl), y_len=to(yl), **kw)
    again = pkg.sdtw_backward_biased(state2, xd, yd, td, ws2, grad_value=gd, x_len=to(xl), y_len=to(yl))
    assert torch.equal(value, value2) and torch.equal(again[2], dt) and again[3] is None
    line = bucket_line(-(N - 1) - 2, M - 2, buckets, far, two_sided)
    at = line[np.arange(M)[None] - np.arange(N)[:, None] + N - 1]
    want_dt, largest = np.zeros((H, buckets)), 0.0
    for b in range(B):
        n, m = (N if xl is None else int(xl[b])), (M if yl is None else int(yl[b]))
        if b >= extra.get("check", B):
            e = E[b].double().cpu().numpy()
        else:
            a, c = x[b, :n].astype(np.float64), y[b, :m].astype(np.float64)
            d = ((a[:, None] - c[None]) ** 2).sum(2) + np.maximum(table[b % H].astype(np.float64), 0)[at[:n, :m]]
            ref = oracle.from_cost(d, gamma, bandwidth=extra.get("bandwidth"))
            assert abs(float(value[b]) - ref["value"]) <= 1e-4 * max(1.0, abs(ref["value"]))
            e = np.zeros((N, M))
            e[:n, :m] = ref["E"]
            want_x = 2 * g[b] * (a * ref["E"].sum(1)[:, None] - ref["E"] @ c)
            want_y = 2 * g[b] * (c * ref["E"].sum(0)[:, None] - ref["E"].T @ a)
            for got, want, k in ((dx[b], want_x, n), (dy[b], want_y, m)):
                got = got.double().cpu().numpy()
                assert np.abs(got[:k] - want).max() <= 1e-3 * np.abs(want).max() + 1e-12 and (got[k:] == 0).all()
            assert np.abs(E[b].double().cpu().numpy() - e).max() <= 1e-3
        want_dt[b % H] += g[b] * np.bincount(at.ravel(), weights=e.ravel(), minlength=buckets)
    want_dt[:, 3] = 0
    got = dt.double().cpu().numpy()
    assert np.abs(got - want_dt).max() <= 1e-3 * np.abs(want_dt).max() and (got[:, 3] == 0).all()


def test_a_table_of_zeros_changes_nothing():
    x, y = (torch.from_numpy(a).cuda() for a in normal_pairs(5, 8, 100, 90, 16))
    value, desc, ws = pkg.sdtw_forward(x, y, 0.5, pkg.UNFUSED)
    dx, dy, E = pkg.sdtw_backward(desc, x, y, ws, want_E=True)
    table = torch.zeros((2, 32), device="cuda", dtype=torch.bfloat16)
    v, state, w = pkg.sdtw_forward_biased(x, y, table, 0.5)
    bx, by, bt, bE = pkg.sdtw_backward_biased(state, x, y, table, w, want_E=True)
    assert torch.equal(v, value) and torch.equal(bx, dx) and torch.equal(by, dy) and torch.equal(bE, E)
    # every pair's E is somewhere in the table: with weights of one the sums agree
    assert abs(float(bt.double().sum()) - float(E.double().sum())) <= 1e-6 * float(E.double().sum())


def test_table_gradient_against_differences():
    """Central differences of the oracle's values in the table's entries: with h = 1e-4 their own error is some 1e-7 of the
    gradient here, so the path's bar, 1e-3 of the largest entry, is the kernels' alone."""
    x, y = normal_pairs(6, 2, 30, 30, 4)
    rng = np.random.default_rng(1)
    table = np.abs(rng.standard_normal((1, 8))).astype(np.float32) + np.float32(0.2)
    xd, yd, td = (torch.from_numpy(a).cuda() for a in (x, y, table))
    _, state, ws = pkg.sdtw_forward_biased(xd, yd, td, 2.0, max_distance=20)
    dt = pkg.sdtw_backward_biased(state, xd, yd, td, ws)[2].double().cpu().numpy()[0]
    at = bucket_line(-29, 30, 8, 20, True)[np.arange(30)[None] - np.arange(30)[:, None] + 29]

    def value(line):
        cost = ((x.astype(np.float64)[:, :, None] - y.astype(np.float64)[:, None]) ** 2).sum(3) + line[at]
        return sum(oracle.from_cost(c, 2.0)["value"] for c in cost)
    step = 1e-4 * np.eye(8)
    line = table[0].astype(np.float64)
    want = np.array([(value(line + e) - value(line - e)) / 2e-4 for e in step])
    assert np.abs(dt - want).max() <= 1e-3 * np.abs(want).max()


def test_refusals():
    x, y = (torch.from_numpy(a).cuda() for a in normal_pairs(6, 4, 30, 30, 4))
    table = torch.zeros((2, 32), device="cuda")
    with pytest.raises(ValueError):
        pkg.sdtw_forward_biased(x, y, torch.zeros((3, 32), device="cuda"), 1.0)
    with pytest.raises(pkg.SdtwError):
        pkg.sdtw_forward_biased(x, y, torch.zeros((2, 31), device="cuda"), 1.0)
    value, state, ws = pkg.sdtw_forward_biased(x, y, table, 1.0, value_only=True)
    with pytest.raises(pkg.SdtwError) as e:
        pkg.sdtw_backward_biased(state, x, y, table, ws)
    assert e.value.status == binding.STATUS_STATE


def biased_on(stream, x, y, table, **kw):
    """(value, dx, dy, dtable, E) of both calls on a stream given by its handle, or the current one"""
    value, state, ws = pkg.sdtw_forward_biased(x, y, table, 0.5, stream=stream, **kw)
    return (value, *pkg.sdtw_backward_biased(state, x, y, table, ws, want_E=True, stream=stream))


def test_memory_of_a_call_on_another_stream_belongs_to_it():
    """What a call allocates is not the current stream's to give away, nor to take from what its pending kernels use."""
    x, y = (torch.from_numpy(a).cuda() for a in normal_pairs(5, 8, 300, 290, 16))
    table = torch.rand((2, 32), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = biased_on(side.cuda_stream, x, y, table)
    torch.cuda.synchronize()
    sizes = [t.numel() for t in out]
    places = {t.data_ptr() for t in out}
    del out
    taken = [torch.empty(n, device="cuda") for n in sizes for _ in range(8)]
    assert not places & {t.data_ptr() for t in taken}


def test_calls_on_a_busy_stream_keep_their_memory():
    x, y = (torch.from_numpy(a).cuda() for a in normal_pairs(5, 8, 300, 290, 16))
    table = torch.rand((2, 32), device="cuda")
    want = biased_on(None, x, y, table)
    busy = torch.randn((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(4):
                busy @ busy
        got = biased_on(side.cuda_stream, x, y, table)
        alone = pkg.sdtw_forward_biased(x, y, table, 0.5, value_only=True, stream=side.cuda_stream)[0]  # (its workspace is let go)
        kept = [torch.full((t.numel(),), 7.0, device="cuda") for t in got for _ in range(4)] + [torch.full((1 << k,), 7.0, device="cuda") for k in (20, 22, 23)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(alone, want[0])
        assert all((k == 7.0).all() for k in kept)
    assert all(torch.equal(a, b) for a, b in zip(biased_on(0, x, y, table), want))  # the default stream by its handle


def test_the_gradient_call_looks_at_the_tensors_it_is_given():
    """The table's place in memory is that of the tensor at hand, not of the one that the values were computed with."""
    x, y = (torch.from_numpy(a).cuda() for a in normal_pairs(6, 4, 30, 40, 4))
    table = (torch.randint(0, 8, (2, 32), device="cuda") - 2).float() / 4  # (whole quarters: the same in 16 bits)
    value, state, ws = pkg.sdtw_forward_biased(x, y, table, 1.0)
    want = pkg.sdtw_backward_biased(state, x, y, table, ws, want_E=True)
    wide = torch.zeros((32, 5), device="cuda")
    wide[:, 1:5:3] = table.t()
    for same in (table.half(), table.bfloat16(), table.t().contiguous().t(), wide[:, 1:5:3].t()):
        value, state, ws = pkg.sdtw_forward_biased(x, y, table, 1.0)
        got = pkg.sdtw_backward_biased(state, x, y, same, ws, want_E=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    for bad in (table.cpu(), table[:1], table[:, :31], table.t(), table.reshape(-1), table.int(), torch.zeros((1, 2, 32), device="cuda")):
        with pytest.raises(ValueError):
            pkg.sdtw_backward_biased(state, x, y, bad, ws)
    for a, b in ((x[:, :29].contiguous(), y), (x, y[:3]), (x[0], y), (x, y[..., :3].contiguous()), (x.cpu(), y), (x, y.cpu()), (x.half(), y)):
        with pytest.raises(ValueError):
            pkg.sdtw_backward_biased(state, a, b, table, ws)
    # a sequence that all pairs share
    value, state, ws = pkg.sdtw_forward_biased(x[0], y, table, 1.0)
    assert pkg.sdtw_backward_biased(state, x[0], y, table, ws)[0].shape == (4, 30, 4)
    with pytest.raises(ValueError):
        pkg.sdtw_backward_biased(state, x, y, table, ws)


@pytest.mark.parametrize("B,N,M,D,gamma,min_memory", [(4, 40, 45, 8, 0.5, False), (3, 300, 290, 16, 0.1, False), (4, 260, 270, 8, 0.5, True), (70, 800, 790, 4, 0.5, False)])
@pytest.mark.parametrize("kind", [torch.float32, torch.float16, torch.bfloat16])
def test_an_infinite_penalty_forbids_its_cells(B, N, M, D, gamma, min_memory, kind):
    """Nothing on distances up to 15 and +inf beyond is the band |i - j| <= 15."""
    x, y = (torch.from_numpy(a).cuda() for a in normal_pairs(9, B, N, M, D))
    w, last = 15, [16, 33]
    assert pkg.sdtw_position_bias_starts(34, 17)[16] == w + 1
    table = torch.zeros((1, 34), device="cuda", dtype=kind)
    table[0, last] = float("inf")
    value, desc, ws = pkg.sdtw_forward(x, y, gamma, pkg.UNFUSED, bandwidth=w, min_memory=min_memory)
    dx, dy, E = pkg.sdtw_backward(desc, x, y, ws, want_E=True)
    v, state, ws = pkg.sdtw_forward_biased(x, y, table, gamma, max_distance=17, min_memory=min_memory)
    bx, by, bt, bE = pkg.sdtw_backward_biased(state, x, y, table, ws, want_E=True)
    assert binding.workspace_status(ws) == 0
    assert ((v - value).abs() <= 1e-4 * value.abs().clamp(min=1.0)).all()
    outside = (torch.arange(N, device="cuda")[:, None] - torch.arange(M, device="cuda")).abs() > w
    assert (bE[:, outside] == 0).all() and float((bE - E).abs().max()) <= 1e-3
    for got, want in ((bx, dx), (by, dy)):
        assert float((got - want).abs().max()) <= 1e-3 * float(want.abs().max())
    assert torch.isfinite(bt).all() and (bt[0, last] == 0).all()
