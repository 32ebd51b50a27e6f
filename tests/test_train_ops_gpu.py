"""Distillation from a teacher's top logits and the bucketed position bias against plain implementations in 64 bits.

Bars, from the arithmetic.  Loss: the kernels sum exp((z - max) / tau) in float32, an exponential being off by about an ulp of
itself and 2^-24 of its argument, chains and trees of sums by a few ulps more: the logarithm of a sum is off by less than 2e-6
here; there are two of them with a tail, and the loss is rounded once: 4e-6 + 2^-23 |loss|.  Gradient: the same relative error on each of
its terms, 4e-6 (p (Q + q_r / p_r) + q) g / tau, and one rounding to its type.  The bias is one float32 addition and one rounding:
the same bits.  Its gradient is compared on whole numbers, whose sums are exact in float32: the same bits again."""
import math

import numpy as np
import pytest
import torch

import paper_2602_17206_amd as pkg

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = {"f32": 2.0 ** -149, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


# ---------------------------------------------------------------- distillation: the definition, row by row, in numpy

def reference(z, t, ids, tau, lse=None, at=None, g=None):
    """(loss, gradient, the size that its error is measured by), float64"""
    T, V = z.shape
    loss, grad, scale = np.zeros(T), np.zeros((T, V)), np.zeros((T, V))
    for i in range(T):
        r = i if at is None else at[i]
        if r < 0:
            continue
        gi = (1.0 if g is None else g[i]) / tau
        if r >= len(t) or (ids[r] >= V).any():
            loss[i], grad[i] = np.nan, np.nan
            continue
        used = ids[r] >= 0
        if lse is None:
            used = used & (t[r] != -np.inf)
        if not used.any():
            continue
        a, b, v = z[i] / tau, t[r][used] / tau, ids[r][used]
        with np.errstate(all="ignore"):
            a = a - a.max()  # (not added back: a maximum of 1e38 would swallow the logarithm even in 64 bits)
            log_sum = np.log(np.exp(a).sum())
            log_q = b - (b.max() + np.log(np.exp(b - b.max()).sum()) if lse is None else lse[r])
            q = np.exp(log_q)
            on = q > 0
            loss[i] = (q[on] * (log_q[on] - a[v[on]] + log_sum)).sum()
            p = np.exp(a - log_sum)
        kept = np.zeros(V, bool)
        kept[v] = True
        Q, over = q.sum(), 0.0
        if lse is None:
            Q = 1.0
        elif not kept.all():
            rest = max(0.0, 1.0 - q.sum())
            Q += rest
            out = a[~kept]
            if rest > 0:
                with np.errstate(all="ignore"):
                    log_out = out.max() + np.log(np.exp(out - out.max()).sum()) if out.max() > -np.inf else -np.inf
                loss[i] += rest * (math.log(rest) - log_out + log_sum)
                over = rest / math.exp(log_out - log_sum) if log_out > -np.inf else 0.0
        d = np.where(kept, Q * p, p * (Q - over))
        size = p * (Q + over)
        np.add.at(d, v, -q)
        np.add.at(size, v, q)
        grad[i], scale[i] = gi * d, abs(gi) * size
    return loss, grad, scale


def f64(x):
    return x.double().cpu().numpy()


def check_loss(got, want):
    got = f64(got)
    fine = np.isfinite(want)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(got[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    off = np.abs(got[fine] - want[fine])
    assert np.all(off <= 4e-6 + 2.0 ** -23 * np.abs(want[fine])), off.max()


def check_grad(got, want, scale, kind):
    got = f64(got)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    bar = 4e-6 * scale + 1.01 * HALF_ULP[kind] * np.abs(want) + LEAST[kind]
    if kind != "f16":
        bar = bar + 2.0 ** -126  # products below the normal numbers may be taken as 0
    off = np.abs(got - want)
    assert np.all(off[ok] <= bar[ok]), (off[ok] - bar[ok]).max()


def problem(T, V, K, kind, tail, tau, seed, mapped=False, ragged=False, pad=0, id_type=torch.int64, teacher_kind=None):
    gen = np.random.default_rng(seed)
    rows = max(1, 2 * T // 3) if mapped else T
    K = min(K, V)
    z = 3.0 * gen.standard_normal((T, V))
    ids = np.stack([gen.permutation(V)[:K] for _ in range(rows)])
    t = 2.0 * gen.standard_normal((rows, K)) + 3.0
    at = None
    if mapped:
        at = gen.integers(-1, rows, T).astype(np.int32)
    if ragged:
        for r in range(rows):
            ids[r, gen.integers(0, K + 1):] = -1
    big = torch.zeros((T, V + pad), dtype=TYPES[kind], device="cuda")
    big[:, :V] = torch.from_numpy(z).cuda()
    s = {"z": big[:, :V], "t": torch.from_numpy(t).to(TYPES[teacher_kind or kind]).cuda(), "ids": torch.from_numpy(ids).to(id_type).cuda(),
         "at": None if at is None else torch.from_numpy(at).cuda(), "lse": None,
         "g": torch.from_numpy(gen.uniform(0.2, 2.0, T).astype(np.float32)).cuda()}
    if tail:
        td = np.where(ids < 0, -np.inf, f64(s["t"])) / tau
        with np.errstate(all="ignore"):
            top = np.where((ids >= 0).any(1), np.log(np.exp(td - 20).sum(1)) + 20, 0.0)
        s["lse"] = torch.from_numpy((top + gen.uniform(0.01, 0.5, rows)).astype(np.float32)).cuda()
    return s


def run_both(s, tau, kind):
    """The two calls and the one call against the definition."""
    more = {"temperature": tau, "teacher_lse": s["lse"], "teacher_row": s["at"]}
    loss, stats = pkg.sdtw_distill_forward(s["z"], s["t"], s["ids"], **more)
    dz = pkg.sdtw_distill_backward(s["z"], s["t"], s["ids"], stats, grad_loss=s["g"], **more)
    loss2, dz2 = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], grad_loss=s["g"], **more)
    want = reference(f64(s["z"]), f64(s["t"]), s["ids"].cpu().numpy(), float(np.float32(tau)), None if s["lse"] is None else f64(s["lse"]),
                     None if s["at"] is None else s["at"].cpu().numpy(), f64(s["g"]))
    for lo, d in ((loss, dz), (loss2, dz2)):
        check_loss(lo, want[0])
        check_grad(d, want[1], want[2], kind)
    return loss, dz, want


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,V,K", [(1, 1, 1), (2, 2, 1), (3, 7, 7), (5, 8, 3), (4, 9, 4), (7, 63, 20), (3, 257, 64), (9, 1000, 10), (2, 4097, 65),
                                   (1, 33001, 128), (300, 515, 33), (2, 2500, 1024)])
def test_distillation_matches_the_definition(T, V, K, kind, tail):
    run_both(problem(T, V, K, kind, tail, 1.0, 10 * T + V), 1.0, kind)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("tau,pad,id_type,teacher_kind", [(2.0, 0, torch.int32, "f32"), (0.5, 3, torch.int64, "bf16"), (1.7, 64, torch.int32, "f16")])
def test_distillation_with_maps_ragged_teachers_strides_and_types(kind, tail, tau, pad, id_type, teacher_kind):
    s = problem(41, 3001, 50, kind, tail, tau, 5, mapped=True, ragged=True, pad=pad, id_type=id_type, teacher_kind=teacher_kind)
    run_both(s, tau, kind)


@pytest.mark.parametrize("kind,V", [("f32", 70001), ("bf16", 140003), ("f16", 300007)])
@pytest.mark.parametrize("T", [3, 700])
@pytest.mark.parametrize("tail", [False, True])
def test_distillation_of_long_rows(kind, V, T, tail):
    """Few long rows and many: the definition is held against a sample of the rows."""
    gen = torch.Generator(device="cuda").manual_seed(V)
    z = (2.0 * torch.randn((T, V), generator=gen, device="cuda")).to(TYPES[kind])
    ids = (torch.arange(40, device="cuda") * 977 + torch.arange(T, device="cuda")[:, None]) % V
    t = torch.randn((T, 40), generator=gen, device="cuda") + 6.0
    z.scatter_add_(1, ids, torch.full((T, 40), 6.0, device="cuda").to(z.dtype))
    lse = torch.logsumexp(t.double(), 1).float() + 0.1 if tail else None
    g = torch.rand(T, generator=gen, device="cuda")
    loss, stats = pkg.sdtw_distill_forward(z, t, ids, teacher_lse=lse)
    dz = pkg.sdtw_distill_backward(z, t, ids, stats, grad_loss=g, teacher_lse=lse)
    loss2, dz2 = pkg.sdtw_distill_step(z, t, ids, grad_loss=g, teacher_lse=lse)
    rows = torch.tensor([0, T // 2, T - 1])
    pick = lambda x: None if x is None else f64(x[rows.cuda()])  # noqa: E731
    want = reference(pick(z), pick(t), ids[rows.cuda()].cpu().numpy(), 1.0, pick(lse), None, pick(g))
    for lo, d in ((loss, dz), (loss2, dz2)):
        check_loss(lo[rows.cuda()], want[0])
        check_grad(d[rows.cuda()], want[1], want[2], kind)
    # every row's gradient sums to 0 where Q = 1: to the rounding of its elements
    if kind == "f32":
        assert float(dz.double().sum(1).abs().max()) < 1e-5 and float(dz2.double().sum(1).abs().max()) < 1e-5


@pytest.mark.parametrize("tail", [False, True])
def test_offsets_beyond_32_bits(tail):
    """2^31 elements and more: the last row is the one that a 32-bit offset would miss."""
    T, V, K = 70000, 32768, 8
    z = torch.zeros((T, V), dtype=torch.bfloat16, device="cuda")
    z[-1] = torch.linspace(-4, 4, V, device="cuda").to(torch.bfloat16)
    ids = torch.arange(K, device="cuda").repeat(T, 1) * 4001 + 7
    t = torch.linspace(0, 3, K, device="cuda").repeat(T, 1)
    lse = torch.logsumexp(t, 1) + 0.3 if tail else None
    loss, stats = pkg.sdtw_distill_forward(z, t, ids, teacher_lse=lse)
    dz = pkg.sdtw_distill_backward(z, t, ids, stats, teacher_lse=lse)
    del stats
    pick = lambda x: None if x is None else f64(x[-2:])  # noqa: E731
    want = reference(pick(z), pick(t), ids[-2:].cpu().numpy(), 1.0, pick(lse))
    check_loss(loss[-2:], want[0])
    check_grad(dz[-2:], want[1], want[2], "bf16")
    assert torch.equal(loss[:-1], loss[:1].expand(T - 1))
    assert torch.equal(dz[1000:1002], dz[:1].expand(2, V))
    loss2, _ = pkg.sdtw_distill_step(z, t, ids, teacher_lse=lse, dlogits=dz)
    check_loss(loss2[-2:], want[0])
    check_grad(dz[-2:], want[1], want[2], "bf16")


def edge(z, t, ids, tail=None, at=None):
    z, t = torch.tensor(z, device="cuda"), torch.tensor(t, device="cuda")
    n = len(z)
    s = {"z": z, "t": t, "ids": torch.tensor(ids, device="cuda"), "at": None if at is None else torch.tensor(at, dtype=torch.int32, device="cuda"),
         "lse": None if tail is None else torch.tensor(tail, device="cuda"), "g": torch.full((n,), 0.5, device="cuda")}
    return run_both(s, 1.0, "f32")


INF, NAN, LOW = float("inf"), float("nan"), -3.4028234663852886e38


def test_masked_tokens_of_the_student():
    # -inf and the type's lowest value on tokens that the teacher does not keep: they only lose their share
    loss, dz, want = edge([[1.0, -INF, 2.0, 0.5, LOW, -1.0]] * 2, [[1.0, 0.0]] * 2, [[0, 2]] * 2)
    assert np.isfinite(want[0]).all() and (f64(dz)[:, [1, 4]] == 0).all()
    edge([[1.0, -INF, 2.0, 0.5, LOW, -1.0]], [[1.0, 0.0]], [[0, 2]], tail=[1.5])
    # a kept token without mass: an infinite loss, a finite gradient
    loss, dz, want = edge([[1.0, -INF, 2.0, 0.5]], [[1.0, 0.0]], [[1, 2]])
    assert float(loss[0]) == INF and torch.isfinite(dz).all()
    # no mass outside the kept tokens although the teacher has some there
    loss, dz, _ = edge([[1.0, 2.0, -INF, -INF]], [[1.0, 0.0]], [[0, 1]], tail=[2.0])
    assert float(loss[0]) == INF and torch.isfinite(dz).all() and (f64(dz)[0, 2:] == 0).all()
    # the lowest value everywhere is a uniform distribution
    loss, dz, want = edge([[LOW] * 5], [[1.0, 0.0]], [[0, 3]])
    assert abs(float(loss[0]) - want[0][0]) < 1e-5


def test_rows_that_are_masked_as_a_whole():
    z = [[NAN, INF, 1.0], [-INF, -INF, -INF], [NAN, 0.0, 1.0], [0.0, INF, 1.0], [NAN, NAN, NAN]]
    t, ids = [[1.0, 0.0]] * 5, [[-1, -1], [0, 1], [1, 2], [0, 2], [0, 1]]
    at = [0, 1, 2, 3, -1]
    z_d, t_d, i_d = torch.tensor(z, device="cuda"), torch.tensor(t, device="cuda"), torch.tensor(ids, device="cuda")
    at_d = torch.tensor(at, dtype=torch.int32, device="cuda")
    for lse in (None, torch.full((5,), 2.0, device="cuda")):
        loss, stats = pkg.sdtw_distill_forward(z_d, t_d, i_d, teacher_lse=lse, teacher_row=at_d)
        dz = pkg.sdtw_distill_backward(z_d, t_d, i_d, stats, teacher_lse=lse, teacher_row=at_d)
        loss2, dz2 = pkg.sdtw_distill_step(z_d, t_d, i_d, teacher_lse=lse, teacher_row=at_d)
        for lo, d in ((loss, dz), (loss2, dz2)):
            assert float(lo[0]) == 0 and float(lo[4]) == 0 and (d[[0, 4]] == 0).all()   # no target
            assert torch.isnan(lo[1:4]).all() and torch.isnan(d[1:4]).all()


def test_teacher_rows_that_leave_nothing_or_name_nothing():
    z = [[0.3, -0.2, 1.0, 0.1]] * 4
    # masked teacher logits have no probability; a row of them alone no target
    edge(z, [[1.0, -INF, 0.0], [-INF, -INF, -INF], [2.0, 1.0, 0.5], [LOW, 0.0, 1.0]], [[0, 1, 2], [0, 1, 2], [3, -1, -7], [0, 1, 2]])
    edge(z, [[1.0, -INF, 0.0], [-INF, -INF, -INF], [2.0, 1.0, 0.5], [LOW, 0.0, 1.0]], [[0, 1, 2], [0, 1, 2], [3, -1, -7], [-1, 1, 2]], tail=[1.6, 0.0, 2.5, 1.6])
    # ids and rows that do not exist
    loss, dz, _ = edge(z, [[1.0, 0.0]] * 3 + [[0.0, 0.0]], [[0, 4], [0, 1], [1 << 40, 0], [2, 3]], at=[0, 1, 2, 4])
    assert torch.isnan(loss[[0, 2, 3]]).all() and torch.isnan(dz[[0, 2, 3]]).all() and torch.isfinite(loss[1])
    # the whole vocabulary kept: no tail, whatever the rounding of the normaliser
    loss, _, _ = edge(z, [[1.0, 0.0, 0.5, -1.0]] * 4, [[0, 1, 2, 3]] * 4, tail=[1.9] * 4)
    assert torch.isfinite(loss).all()


def test_slots_of_one_token_add_up():
    rng = np.random.default_rng(3)
    for V, K in ((5, 4), (300, 100), (900, 1000)):
        z = rng.standard_normal((3, V)).astype(np.float32)
        t = rng.standard_normal((3, K)).astype(np.float32)
        ids = rng.integers(0, max(2, V // 3), (3, K))
        top = np.log(np.exp(t.astype(np.float64)).sum(1))
        edge(z.tolist(), t.tolist(), ids.tolist())
        edge(z.tolist(), t.tolist(), ids.tolist(), tail=(top + 0.2).tolist())


def test_a_confident_student_keeps_its_tail():
    """Nearly all mass on the kept token: the rest, 1e-12 of it, is not the difference of two sums."""
    z = np.full((1, 200), -28.0, np.float32)
    z[0, 17] = 5.0
    z[0, 3:9] = [-25, -26, -27, -24, -23, -22.5]
    edge(z.tolist(), [[9.0, 3.0]], [[17, 5]], tail=[math.log(math.exp(9.0) + math.exp(3.0)) + 1e-3])


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,V", [(5, 9001), (600, 2003)])
def test_gradient_in_place_of_the_logits(kind, T, V):
    s = problem(T, V, 30, kind, True, 1.0, 77, mapped=True)
    more = {"teacher_lse": s["lse"], "teacher_row": s["at"]}
    loss, stats = pkg.sdtw_distill_forward(s["z"], s["t"], s["ids"], **more)
    want = pkg.sdtw_distill_backward(s["z"], s["t"], s["ids"], stats, grad_loss=s["g"], **more)
    loss_s, want_s = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], grad_loss=s["g"], **more)
    a, b = s["z"].clone(), s["z"].clone()
    assert pkg.sdtw_distill_backward(a, s["t"], s["ids"], stats, grad_loss=s["g"], dlogits=a, **more) is a
    assert torch.equal(a, want)
    loss_b, _ = pkg.sdtw_distill_step(b, s["t"], s["ids"], grad_loss=s["g"], dlogits=b, **more)
    assert torch.equal(b, want_s) and torch.equal(loss_b, loss_s)


@pytest.mark.parametrize("tail", [False, True])
def test_gradient_against_differences_of_the_loss(tail):
    """(L(z + h u) - L(z - h u)) / 2 h against <dz, u>, |u| <= 1, h = 2^-5: the two losses' errors over 2 h, 1.3e-4, and
    h^2 / 6 times a third derivative of at most 1: 1.7e-4 more."""
    s = problem(16, 700, 40, "f32", tail, 1.0, 8)
    loss, stats = pkg.sdtw_distill_forward(s["z"], s["t"], s["ids"], teacher_lse=s["lse"])
    dz = pkg.sdtw_distill_backward(s["z"], s["t"], s["ids"], stats, teacher_lse=s["lse"])
    gen = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(4):
        u = torch.rand(dz.shape, generator=gen, device="cuda") * 2 - 1
        h = 2.0 ** -5
        up, _ = pkg.sdtw_distill_forward(s["z"] + h * u, s["t"], s["ids"], teacher_lse=s["lse"])
        down, _ = pkg.sdtw_distill_forward(s["z"] - h * u, s["t"], s["ids"], teacher_lse=s["lse"])
        slope = (up.double() - down.double()) / (2 * h)
        assert float((slope - (dz.double() * u.double()).sum(1)).abs().max()) < 5e-4


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("T,V", [(1030, 1500), (1027, 700), (1025, 3), (1026, 2047), (3, 2048), (2, 4090)])
def test_short_rows_many_and_few(T, V, kind, tail):
    run_both(problem(T, V, 24, kind, tail, 1.3, T + V, mapped=True, ragged=True, pad=1), 1.3, kind)


@pytest.mark.parametrize("copies", [1, 300])
@pytest.mark.parametrize("width", [9, 1900, 2100, 9001, 60001])
def test_masks_in_rows_of_every_length(width, copies):
    """The masked rows above in rows that are padded with -inf, one of each and many of each."""
    z = [[1.0, -INF, 2.0, 0.5, LOW, -1.0], [1.0, -INF, 2.0, 0.5, LOW, -1.0], [LOW] * 5 + [-INF], [1.0, -INF, 2.0, 0.5, 3.0, -INF],
         [-INF] * 6, [NAN, 0.0, 1.0, 2.0, 0.0, 0.0]]
    t, ids = [[1.0, 0.0], [0.0, 0.5], [1.0, 0.0], [1.0, 0.0], [1.0, 0.0], [1.0, 0.0]], [[0, 2], [3, -1], [0, 3], [1, 2], [0, 1], [1, 2]]
    wide = torch.full((6, width), -INF)
    wide[:, :6] = torch.tensor(z)
    wide[:, [1, width - 1]] = wide[:, [width - 1, 1]]  # a kept place at the row's end
    ids = [[width - 1 if i == 1 else i for i in row] for row in ids]
    z_d, t_d, i_d = wide.cuda().repeat(copies, 1), torch.tensor(t, device="cuda").repeat(copies, 1), torch.tensor(ids, device="cuda").repeat(copies, 1)
    for lse in (None, torch.full((6 * copies,), 1.9, device="cuda")):
        want = reference(f64(z_d[:4]), f64(t_d[:4]), i_d[:4].cpu().numpy(), 1.0, None if lse is None else f64(lse[:4]))
        loss, stats = pkg.sdtw_distill_forward(z_d, t_d, i_d, teacher_lse=lse)
        dz = pkg.sdtw_distill_backward(z_d, t_d, i_d, stats, teacher_lse=lse)
        for lo, d in ((loss, dz), pkg.sdtw_distill_step(z_d, t_d, i_d, teacher_lse=lse)):
            for c in {0, 1 % copies, copies // 2, copies - 1}:
                check_loss(lo[6 * c:6 * c + 4], want[0])
                check_grad(d[6 * c:6 * c + 4], want[1], want[2], "f32")
            assert torch.isnan(lo.view(copies, 6)[:, 4:]).all() and torch.isnan(d.view(copies, 6, width)[:, 4:]).all()
            assert not torch.isnan(lo.view(copies, 6)[:, :4]).any() and not torch.isnan(d.view(copies, 6, width)[:, :4]).any()


# ---------------------------------------------------------------- position bias

def buckets_of(n, D):
    """side(d) in whole numbers"""
    e, m = n // 2, n - n // 2

    def side(d):
        if d < e:
            return d
        d = min(d, D)
        k = 0
        while k + 1 < m and d ** m >= e ** (m - k - 1) * D ** (k + 1):
            k += 1
        return e + k
    return side


def bucket_matrix(N, M, buckets, D, two_sided, offset):
    n = buckets // 2 if two_sided else buckets
    side = buckets_of(n, D)
    seen = {}

    def bucket(r):
        if r not in seen:
            seen[r] = (side(abs(r)) + (n if r > 0 else 0)) if two_sided else side(max(0, -r))
        return seen[r]
    line = np.array([bucket(r - offset) for r in range(-(N - 1), M)], dtype=np.int64)
    return line[np.arange(M)[None, :] - np.arange(N)[:, None] + N - 1]


RULES = [(32, 128, True), (32, 128, False), (4, 2, True), (2, 5, False), (128, 4096, False), (256, 300, True), (10, 77, True)]
SHAPES = [(1, 1, 1, 1), (2, 3, 1, 700), (3, 2, 700, 1), (2, 2, 5, 9), (1, 3, 64, 64), (2, 1, 130, 515), (1, 2, 300, 2100), (1, 1, 2050, 33)]


def whole_numbers(shape, kind, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-8, 9, shape, generator=gen, device="cuda").to(TYPES[kind])


@pytest.mark.parametrize("buckets,D,two_sided", RULES)
@pytest.mark.parametrize("B,H,N,M", SHAPES)
def test_bias_and_its_gradient(B, H, N, M, buckets, D, two_sided):
    for kind in sorted(TYPES):
        gen = torch.Generator(device="cuda").manual_seed(N + M)
        plane = torch.randn((B, H, N, M), generator=gen, device="cuda").to(TYPES[kind])
        table = torch.randn((H, buckets), generator=gen, device="cuda")
        at = bucket_matrix(N, M, buckets, D, two_sided, 0)
        at_d = torch.from_numpy(at).cuda()
        out = pkg.sdtw_position_bias_forward(table, plane, max_distance=D, two_sided=two_sided)
        assert torch.equal(out, (plane.float() + table[:, at_d]).to(plane.dtype)), kind
        g = whole_numbers((B, H, N, M), kind, N * M)
        dt = pkg.sdtw_position_bias_backward(g, buckets, max_distance=D, two_sided=two_sided)
        want = np.zeros((H, buckets))
        total = f64(g).sum(0)
        for h in range(H):
            want[h] = np.bincount(at.ravel(), weights=total[h].ravel(), minlength=buckets)
        np.testing.assert_array_equal(f64(dt), want)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("two_sided", [True, False])
@pytest.mark.parametrize("N,M", [(1, 333), (4, 1000), (70, 90), (257, 300)])
def test_bias_of_sequences_with_lengths_and_offsets_of_their_own(kind, two_sided, N, M):
    B, H, buckets, D = 5, 3, 32, 100
    gen = torch.Generator(device="cuda").manual_seed(9)
    plane = torch.randn((B, H, N, M), generator=gen, device="cuda").to(TYPES[kind])
    g = whole_numbers((B, H, N, M), kind, 4)
    offset = torch.tensor([0, 5, -40, M, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    rlen = torch.tensor([N, 0, max(1, N // 2), N + 5, 1], dtype=torch.int32, device="cuda")
    clen = torch.tensor([M // 2, M, 1, -3, M - 1], dtype=torch.int32, device="cuda")
    scale = torch.tensor([1.0, 0.5, -2.0, 4.0, 0.25], device="cuda")
    table = torch.randn((buckets, H), generator=gen, device="cuda").to(TYPES[kind]).t()  # an embedding's layout
    inside = torch.zeros((B, 1, N, M), dtype=torch.bool, device="cuda")
    want_dt = np.zeros((H, buckets))
    want = plane.clone()
    for b in range(B):
        r, c = min(max(int(rlen[b]), 0), N), min(max(int(clen[b]), 0), M)
        inside[b, :, :r, :c] = True
        at = bucket_matrix(N, M, buckets, D, two_sided, int(offset[b]))
        y = (plane[b].float() + table.float()[:, torch.from_numpy(at).cuda()]).to(plane.dtype)
        want[b] = torch.where(inside[b], y, plane[b])
        for h in range(H):
            want_dt[h] += float(scale[b]) * np.bincount(at[:r, :c].ravel(), weights=f64(g[b, h, :r, :c]).ravel(), minlength=buckets)
    # what lies outside takes no part: NaN and infinities there are copied, and not summed
    plane = torch.where(inside, plane, math.nan)
    want = torch.where(inside, want, math.nan)
    g = torch.where(inside, g, math.inf)
    more = dict(max_distance=D, two_sided=two_sided, offset=offset, row_len=rlen, col_len=clen)
    out = pkg.sdtw_position_bias_forward(table, plane, **more)
    assert torch.equal(torch.isnan(out), ~inside.expand_as(out)) and torch.equal(out.nan_to_num(7.0), want.nan_to_num(7.0))
    np.testing.assert_array_equal(f64(pkg.sdtw_position_bias_backward(g, buckets, scale=scale, **more)), want_dt)


def test_bias_keeps_masked_scores_masked():
    for dtype, low in ((torch.float32, LOW), (torch.float16, -65504.0), (torch.bfloat16, -3.3895313892515355e38)):
        plane = torch.tensor([[[[low, -INF, 0.0, INF, NAN, low, 1.0, -INF, 2.0, low]]]], device="cuda").to(dtype)
        out = pkg.sdtw_position_bias_forward(torch.full((1, 32), 0.5, device="cuda"), plane)
        want = (plane.float() + 0.5).to(dtype)
        assert torch.equal(out.nan_to_num(9.0, posinf=8.0, neginf=-8.0), want.nan_to_num(9.0, posinf=8.0, neginf=-8.0))
        assert torch.equal(torch.isnan(out), torch.isnan(want))


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_bias_on_planes_of_other_strides(kind):
    B, H, N, M = 3, 4, 37, 61
    gen = torch.Generator(device="cuda").manual_seed(2)
    table = torch.randn((H, 16), generator=gen, device="cuda")
    base = torch.randn((B, N, H, M + 3), generator=gen, device="cuda").to(TYPES[kind])
    plane = base.permute(0, 2, 1, 3)[..., 1:M + 1]  # rows between heads, odd starts
    contiguous = plane.contiguous()
    want = pkg.sdtw_position_bias_forward(table, contiguous, max_distance=40)
    assert torch.equal(pkg.sdtw_position_bias_forward(table, plane, max_distance=40), want)
    # one plane shared by all heads and sequences, and its gradient's counterpart: a broadcast gradient
    one = plane[:1, :1].expand(B, H, N, M)
    assert torch.equal(pkg.sdtw_position_bias_forward(table, one, max_distance=40), pkg.sdtw_position_bias_forward(table, one.contiguous(), max_distance=40))
    g = whole_numbers((1, 1, N, M), kind, 3).expand(B, H, N, M)
    assert torch.equal(pkg.sdtw_position_bias_backward(g, 16, max_distance=40), pkg.sdtw_position_bias_backward(g.contiguous(), 16, max_distance=40))
    assert torch.equal(pkg.sdtw_position_bias_backward(base.permute(0, 2, 1, 3)[..., 1:M + 1].float().to(TYPES[kind]), 16, max_distance=40),
                       pkg.sdtw_position_bias_backward(contiguous, 16, max_distance=40))
    # in place, into a strided output, and without a plane
    room = base.clone().permute(0, 2, 1, 3)[..., 1:M + 1]
    assert pkg.sdtw_position_bias_forward(table, room, max_distance=40, out=room) is room and torch.equal(room, want)
    out = torch.empty((B, H, N, M), dtype=TYPES[kind], device="cuda")
    pkg.sdtw_position_bias_forward(table, None, max_distance=40, out=out)
    assert torch.equal(out, pkg.sdtw_position_bias_forward(table, torch.zeros_like(out), max_distance=40))


def test_bias_gradient_is_that_of_the_bias():
    """The bias is linear in its table: <g, out(table + e) - out(table)> = <dtable, e>, on whole numbers exactly."""
    g = whole_numbers((2, 3, 50, 81), "f32", 1)
    plane = whole_numbers((2, 3, 50, 81), "f32", 2)
    dt = pkg.sdtw_position_bias_backward(g, 24, max_distance=60, offset=7)
    e = whole_numbers((3, 24), "f32", 5)
    table = whole_numbers((3, 24), "f32", 6)
    diff = pkg.sdtw_position_bias_forward(table + e, plane, max_distance=60, offset=7) - pkg.sdtw_position_bias_forward(table, plane, max_distance=60, offset=7)
    assert float((g.double() * diff.double()).sum()) == float((dt.double() * e.double()).sum())


def test_bias_of_empty_planes():
    for shape in ((0, 2, 3, 4), (2, 2, 0, 4), (2, 2, 3, 0)):
        plane = torch.zeros(shape, device="cuda")
        assert pkg.sdtw_position_bias_forward(torch.zeros((2, 32), device="cuda"), plane).shape == shape
        assert torch.equal(pkg.sdtw_position_bias_backward(plane, 32), torch.zeros((2, 32), device="cuda"))
    z = torch.zeros((0, 10), device="cuda")
    loss, _ = pkg.sdtw_distill_forward(z, torch.zeros((1, 2), device="cuda"), torch.zeros((1, 2), dtype=torch.int64, device="cuda"))
    assert loss.shape == (0,)


def test_bias_beyond_32_bit_offsets():
    """More than 2^31 cells, far from position 0 by more than 2^32."""
    H, N, M, far = 3, 32768, 32768, 5 * 2 ** 32
    plane = torch.ones((1, H, N, M), dtype=torch.bfloat16, device="cuda")
    dt = pkg.sdtw_position_bias_backward(plane, 32, max_distance=128)
    at = bucket_matrix(1, 2 * N - 1, 32, 128, True, N - 1)[0]  # by diagonal j - i = -(N - 1) .. N - 1
    count = np.bincount(at, weights=N - np.abs(np.arange(-(N - 1), N)), minlength=32).astype(np.float32)
    np.testing.assert_array_equal(dt.cpu().numpy(), np.tile(count, (H, 1)))
    table = torch.arange(H * 32, device="cuda").reshape(H, 32).float()
    pkg.sdtw_position_bias_forward(table, plane, out=plane)
    rows = bucket_matrix(N, 4, 32, 128, True, 0)
    assert torch.equal(plane[0, -1, :, :4].float(), (1 + table[-1][torch.from_numpy(rows).cuda()]).to(torch.bfloat16).float())
    assert float(plane[0, -1, -1, -1]) == float((1 + table[-1, 0]).to(torch.bfloat16))
    small = torch.zeros((1, 1, 2, 3), device="cuda")
    ramp = torch.arange(32.0, device="cuda")[None]
    assert float(pkg.sdtw_position_bias_forward(ramp, small, offset=far).min()) == 15.0    # far to the left: the last of the first half
    assert float(pkg.sdtw_position_bias_forward(ramp, small, offset=-far).max()) == 31.0
    dt = pkg.sdtw_position_bias_backward(small + 1, 32, offset=-far)
    assert float(dt[0, 31]) == 6.0 and float(dt.sum()) == 6.0


# ---------------------------------------------------------------- streams, graphs, repetition

def test_operators_run_on_the_stream_they_are_given():
    s = problem(64, 5000, 20, "f32", True, 1.0, 3)
    plane = torch.randn((2, 2, 100, 120), device="cuda")
    table = torch.randn((2, 32), device="cuda")
    want = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], teacher_lse=s["lse"])
    want_b = pkg.sdtw_position_bias_forward(table, plane)
    want_t = pkg.sdtw_position_bias_backward(plane, 32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], teacher_lse=s["lse"])
        got_b = pkg.sdtw_position_bias_forward(table, plane)
        got_t = pkg.sdtw_position_bias_backward(plane, 32)
    side.synchronize()
    # the same inputs give the same bits, whatever the stream
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got_b, want_b) and torch.equal(got_t, want_t)


def test_memory_of_a_call_on_another_stream_is_not_given_away():
    """A busy stream gets the calls by its handle; meanwhile the current one fills whatever memory it is given."""
    s = problem(600, 70001, 20, "f32", True, 1.0, 3)
    plane = torch.randn((8, 2, 300, 320), device="cuda")
    want = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], teacher_lse=s["lse"])
    want_f = pkg.sdtw_distill_forward(s["z"], s["t"], s["ids"], teacher_lse=s["lse"])
    want_b, want_t = pkg.sdtw_position_bias_forward(plane[0, :, 0, :32], plane), pkg.sdtw_position_bias_backward(plane, 32)
    busy = torch.randn((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(4):
                busy @ busy
        h = side.cuda_stream
        got = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], teacher_lse=s["lse"], stream=h)
        got_f = pkg.sdtw_distill_forward(s["z"], s["t"], s["ids"], teacher_lse=s["lse"], stream=h)
        got_b, got_t = pkg.sdtw_position_bias_forward(plane[0, :, 0, :32], plane, stream=h), pkg.sdtw_position_bias_backward(plane, 32, stream=h)
        kept = [torch.full((n,), 7.0, device="cuda") for n in (600, 600 * 8, 4096, 2 * 32, 1 << 14, 1 << 16, 1 << 20) for _ in range(4)]
        torch.cuda.synchronize()
        pairs = [*zip(got, want), *zip(got_f, want_f), (got_b, want_b), (got_t, want_t)]
        assert all(torch.equal(a.view(torch.int32), b.view(torch.int32)) for a, b in pairs)
        assert all((k == 7.0).all() for k in kept)
    # the default stream by its handle
    assert torch.equal(pkg.sdtw_position_bias_backward(plane, 32, stream=0), want_t)


@pytest.mark.parametrize("T", [2, 400])
def test_operators_in_a_graph(T):
    s = problem(T, 9000, 20, "bf16", True, 1.0, 3)
    plane = torch.randn((2, 2, 100, 120), device="cuda")
    table = torch.randn((2, 32), device="cuda")
    more = {"teacher_lse": s["lse"], "grad_loss": s["g"]}
    loss, dz = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], **more)
    out, dt = pkg.sdtw_position_bias_forward(table, plane), pkg.sdtw_position_bias_backward(plane, 32)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], loss=loss, dlogits=dz, **more)
        pkg.sdtw_position_bias_forward(table, plane, out=out)
        pkg.sdtw_position_bias_backward(plane, 32, dtable=dt)
    for i in range(4):
        s["z"].copy_(torch.randn(s["z"].shape, device="cuda"))
        plane.copy_(torch.randn(plane.shape, device="cuda"))
        want = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], **more)
        want_b, want_t = pkg.sdtw_position_bias_forward(table, plane), pkg.sdtw_position_bias_backward(plane, 32)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(dz, want[1]) and torch.equal(out, want_b) and torch.equal(dt, want_t), i


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_bias_in_place_where_rows_end_inside_a_vector(kind):
    """Every thread writes the cells that are its own, whatever it reads of its neighbours' for the row's end."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    table = torch.randn((2, 32), generator=gen, device="cuda")
    for M in (3, 9, 257, 513, 937, 1026, 2049):
        plane = torch.randn((3, 2, 67, M), generator=gen, device="cuda").to(TYPES[kind])
        at = torch.from_numpy(bucket_matrix(67, M, 32, 128, True, 0)).cuda()
        want = (plane.float() + table[:, at]).to(plane.dtype)
        for _ in range(3):
            room = plane.clone()
            pkg.sdtw_position_bias_forward(table, room, out=room)
            assert torch.equal(room, want), M


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_the_same_inputs_give_the_same_bits(kind):
    gen = torch.Generator(device="cuda").manual_seed(9)
    plane = torch.randn((2, 2, 777, 2051), generator=gen, device="cuda").to(TYPES[kind])
    s = problem(300, 20011, 40, kind, True, 1.3, 5)
    first = None
    for _ in range(5):
        loss, dz = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], teacher_lse=s["lse"])
        loss_f, stats = pkg.sdtw_distill_forward(s["z"], s["t"], s["ids"], teacher_lse=s["lse"])
        dz_f = pkg.sdtw_distill_backward(s["z"], s["t"], s["ids"], stats, teacher_lse=s["lse"])
        got = [loss, dz, loss_f, dz_f, pkg.sdtw_position_bias_backward(plane, 32)]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


def test_refusals_of_the_binding():
    s = problem(4, 50, 5, "f32", False, 1.0, 1)
    z, t, ids = s["z"], s["t"], s["ids"]
    for bad in (lambda: pkg.sdtw_distill_forward(z.double(), t, ids), lambda: pkg.sdtw_distill_forward(z, t, ids.float()),
                lambda: pkg.sdtw_distill_forward(z, t, ids[:, :4]), lambda: pkg.sdtw_distill_forward(z.t().contiguous().t(), t, ids),
                lambda: pkg.sdtw_distill_forward(z, t.cpu(), ids), lambda: pkg.sdtw_distill_forward(z, t, ids, teacher_row=torch.zeros(4, device="cuda")),
                lambda: pkg.sdtw_distill_forward(z, t, ids, teacher_lse=torch.zeros(3, device="cuda")),
                lambda: pkg.sdtw_distill_step(z, t, ids, dlogits=torch.empty((4, 50), dtype=torch.float16, device="cuda")),
                lambda: pkg.sdtw_position_bias_forward(torch.zeros((3, 32), device="cuda"), torch.zeros((1, 2, 4, 4), device="cuda")),
                lambda: pkg.sdtw_position_bias_forward(torch.zeros((2, 32), device="cuda"), torch.zeros((1, 2, 4, 4), device="cuda").transpose(2, 3)),
                lambda: pkg.sdtw_position_bias_forward(torch.zeros((2, 32), device="cuda")),
                lambda: pkg.sdtw_position_bias_backward(torch.zeros((1, 2, 4, 4), dtype=torch.int32, device="cuda"), 32)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: pkg.sdtw_distill_forward(z, t, ids, temperature=0.0), lambda: pkg.sdtw_distill_forward(z, t[:3], ids[:3]),
                lambda: pkg.sdtw_position_bias_forward(torch.zeros((2, 31), device="cuda"), torch.zeros((1, 2, 4, 4), device="cuda")),
                lambda: pkg.sdtw_position_bias_forward(torch.zeros((2, 32), device="cuda"), torch.zeros((1, 2, 4, 4), device="cuda"), max_distance=8),
                lambda: pkg.sdtw_position_bias_backward(torch.zeros((1, 2, 4, 4), device="cuda"), 300)):
        with pytest.raises(pkg.SdtwError):
            bad()


# ---------------------------------------------------------------- masks of every size

def definition(z, t, ids, tau, lse, g):
    """As `reference`, for rows whose masked columns hold any finite number: a share of the tokens outside the kept ones is
    taken among those tokens, not as the quotient of two probabilities that are both 0."""
    T, V = z.shape
    loss, grad, scale = np.zeros(T), np.zeros((T, V)), np.zeros((T, V))
    for i in range(T):
        own, b = z[i] / tau, t[i] / tau
        a = own - own.max()
        log_sum = np.log(np.exp(a).sum())
        p = np.exp(a - log_sum)
        log_q = b - (b.max() + np.log(np.exp(b - b.max()).sum()) if lse is None else lse[i])
        q = np.exp(log_q)
        loss[i] = (q * (log_q - a[ids[i]] + log_sum)).sum()
        kept = np.zeros(V, bool)
        kept[ids[i]] = True
        Q, share = 1.0, np.zeros(V)
        if lse is not None:
            rest = max(0.0, 1.0 - q.sum())
            Q = q.sum() + rest
            out = own[~kept]
            w = np.exp(out - out.max())  # (each maximum is taken off by itself: beside 1e20 the rest would vanish even in 64 bits)
            loss[i] += rest * (math.log(rest) - (out.max() - own.max()) - math.log(w.sum()) + log_sum)
            share[~kept] = rest * w / w.sum()
        d, size = Q * p - share, Q * p + share
        d[ids[i]] -= q
        size[ids[i]] += q
        grad[i], scale[i] = g[i] / tau * d, g[i] / tau * size
    with np.errstate(over="ignore"):
        loss = np.where(np.isinf(loss.astype(np.float32)), np.inf * np.sign(loss), loss)  # (beyond float32)
    return loss, grad, scale


MASKS = [-1e4, -1e9, -1e10, -1e20, -1e30, -2e30, LOW, 1e10, 1e30]


@pytest.mark.parametrize("tau", [1e-6, 0.1, 0.7, 1.0, 2.0, 1e4])
@pytest.mark.parametrize("V,copies,kind", [(700, 1, "f32"), (700, 20, "bf16"), (5000, 20, "f32"), (9001, 1, "bf16"), (9001, 20, "bf16"), (33001, 1, "f32"),
                                           (33001, 20, "f32"), (70001, 1, "f32"), (70001, 12, "bf16")])
def test_masks_of_every_size(V, copies, kind, tau):
    """Rows in which a thread, a wavefront, a slice, the kept tokens, those outside them or all tokens hold one finite mask."""
    gen = np.random.default_rng(V)
    K, rows, spread = 5, [], min(1.0, tau)
    for mask in [max(m, torch.finfo(TYPES[kind]).min) for m in MASKS]:
        for form in range(6):
            z = spread * gen.standard_normal(V)
            ids = V - 1 - gen.permutation(V // 20)[:K]
            if form == 0:    # most of the row, from the front
                z[:V - V // 20] = mask
            elif form == 1:  # most of the row, anywhere
                hide = gen.random(V) < 0.95
                hide[ids] = False
                z[hide] = mask
            elif form == 2:  # the kept tokens
                z[ids] = mask
            elif form == 3:  # everything
                z[:] = mask
            elif form == 4:  # everything outside the kept tokens
                z[:] = mask
                z[ids] = spread * gen.standard_normal(K)
            else:            # everything but one token that is not kept
                z[:] = mask
                z[V // 2] = 0.5 * spread
            rows.append((z, ids, spread * gen.standard_normal(K)))
    n = len(rows)
    z = torch.from_numpy(np.stack([r[0] for r in rows])).to(TYPES[kind]).cuda()
    ids, t = (torch.from_numpy(np.stack([r[k] for r in rows])).cuda() for k in (1, 2))
    t = t.float()
    g = torch.from_numpy(gen.uniform(0.5, 2.0, n).astype(np.float32)).cuda()
    for tail in (False, True):
        lse = (torch.logsumexp(t.double() / float(np.float32(tau)), 1) + 0.3).float() if tail else None
        want = definition(f64(z), f64(t), ids.cpu().numpy(), float(np.float32(tau)), None if lse is None else f64(lse), f64(g))
        many = [None if x is None else x.repeat(copies, *[1] * (x.dim() - 1)) for x in (z, t, ids, lse, g)]
        more = {"temperature": tau, "teacher_lse": many[3]}
        loss, stats = pkg.sdtw_distill_forward(*many[:3], **more)
        dz = pkg.sdtw_distill_backward(*many[:3], stats, grad_loss=many[4], **more)
        for lo, d in ((loss, dz), pkg.sdtw_distill_step(*many[:3], grad_loss=many[4], **more)):
            assert not torch.isnan(lo).any() and not torch.isnan(d).any()
            for c in {0, copies // 2, copies - 1}:
                check_loss(lo[n * c:n * c + n], want[0])
                check_grad(d[n * c:n * c + n], want[1], want[2], kind)


@pytest.mark.parametrize("V", [6, 3001, 9001, 70001])
@pytest.mark.parametrize("copies", [1, 1500])
def test_a_nan_among_the_kept_tokens_with_no_mass_outside(V, copies):
    """The whole gradient of such a row is NaN, that of the tokens outside too, although they have no mass."""
    z = torch.full((2, V), -INF, device="cuda")
    z[:, [1, V - 1]] = torch.tensor([[NAN, 1.0], [0.5, 1.0]], device="cuda")
    more = {"teacher_lse": torch.full((2 * copies,), 2.0, device="cuda")}
    z, t = z.repeat(copies, 1), torch.tensor([[1.0, 0.0]], device="cuda").repeat(2 * copies, 1)
    ids = torch.tensor([[1, V - 1]], device="cuda").repeat(2 * copies, 1)
    loss, stats = pkg.sdtw_distill_forward(z, t, ids, **more)
    dz = pkg.sdtw_distill_backward(z, t, ids, stats, **more)
    for lo, d in ((loss, dz), pkg.sdtw_distill_step(z, t, ids, **more)):
        assert torch.isnan(lo[::2]).all() and torch.isnan(d[::2]).all()
        assert (lo[1::2] == INF).all() and torch.isfinite(d[1::2]).all()


@pytest.mark.parametrize("tau", [0.5, 1.0, 2.0])
@pytest.mark.parametrize("V", [50, 9001, 70001])
def test_teacher_rows_at_the_ends_of_the_type(V, tau):
    """The logarithm of such a row's normaliser is nothing beside its largest logit, and over a temperature below 1 that is beyond
    float32; the shares of the kept tokens are those of the differences all the same."""
    gen = np.random.default_rng(4)
    z = torch.from_numpy(gen.standard_normal((5, V)).astype(np.float32)).cuda()
    t = [[LOW, LOW, LOW], [LOW, LOW, 0.0], [3e38, 3e38, LOW], [-1e38, -1e38, -1e38], [1e12, 1e12, -1e12]]
    same = [[0.0, 0.0, 0.0], [-INF, -INF, 0.0], [0.0, 0.0, -INF], [0.0, 0.0, 0.0], [0.0, 0.0, -INF]]
    t, ids = torch.tensor(t, device="cuda"), torch.tensor([[3, 40, 7]] * 5, device="cuda")
    loss, stats = pkg.sdtw_distill_forward(z, t, ids, temperature=tau)
    dz = pkg.sdtw_distill_backward(z, t, ids, stats, temperature=tau)
    want = reference(f64(z), np.array(same), ids.cpu().numpy(), tau)
    for lo, d in ((loss, dz), pkg.sdtw_distill_step(z, t, ids, temperature=tau)):
        check_loss(lo, want[0])
        check_grad(d, want[1], want[2], "f32")


@pytest.mark.parametrize("offset", [0, "own"])
@pytest.mark.parametrize("kind", sorted(TYPES))
def test_what_has_no_cell_takes_no_part_whatever_its_weight(kind, offset):
    """A mean over a sequence's cells has the weight 1 / 0 where there are none; and a weight is not looked at in buckets of which the
    sequence has no cell."""
    B, H, N, M, buckets = 6, 2, 150, 1100, 32
    g = whole_numbers((B, H, N, M), kind, 11)
    g[4] = 1.0
    rlen = torch.tensor([N, 0, 7, N, 2, 0], dtype=torch.int32, device="cuda")
    clen = torch.tensor([M, M, 0, 600, 1, 0], dtype=torch.int32, device="cuda")
    scale = torch.tensor([1.0, INF, NAN, 0.5, INF, -INF], device="cuda")
    at_d = 0 if offset == 0 else torch.tensor([0, 3, 5, -40, 0, 9], dtype=torch.int32, device="cuda")
    want = np.zeros((H, buckets))
    for b in (0, 3, 4):
        r, c = int(rlen[b]), int(clen[b])
        at = bucket_matrix(N, M, buckets, 128, True, 0 if offset == 0 else int(at_d[b]))[:r, :c].ravel()
        for h in range(H):
            np.add.at(want[h], at, float(scale[b]) * f64(g[b, h, :r, :c]).ravel())
    assert np.isinf(want[:, :2]).all() and np.isfinite(want[:, 2:]).all()  # (rows 0 and 1 of a column: distances 0 and 1)
    got = pkg.sdtw_position_bias_backward(g, buckets, offset=at_d, row_len=rlen, col_len=clen, scale=scale)
    np.testing.assert_array_equal(f64(got), want)
    got = pkg.sdtw_position_bias_backward(g[1:3], buckets, row_len=rlen[1:3].contiguous(), col_len=clen[1:3].contiguous(), scale=scale[1:3].contiguous())
    np.testing.assert_array_equal(f64(got), 0.0)


@pytest.mark.parametrize("two_sided", [True, False])
@pytest.mark.parametrize("offset", [(1 << 62) - 1, 1 - (1 << 62), (1 << 62) - 700, 700 - (1 << 62), 1 << 40, -(1 << 31), 1 << 31, 1 << 30])
def test_bias_at_offsets_up_to_the_limit(offset, two_sided):
    """Every distance is in one last bucket: forward and gradient agree on which."""
    N, M, buckets = 300, 1300, 32
    plane = torch.zeros((2, 1, N, M), device="cuda")
    table = torch.arange(float(buckets), device="cuda")[None]
    last = {(True, True): 15, (True, False): 31, (False, True): 31, (False, False): 0}[two_sided, offset > 0]
    out = pkg.sdtw_position_bias_forward(table, plane, two_sided=two_sided, offset=offset)
    assert (out == last).all()
    want = torch.zeros((1, buckets), device="cuda")
    want[0, last] = 2 * N * M
    assert torch.equal(pkg.sdtw_position_bias_backward(plane + 1, buckets, two_sided=two_sided, offset=offset), want)


# ---------------------------------------------------------------- several rows of a workgroup, sums beyond float32

@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("T,V,kind,pad", [(2300, 5003, "bf16", 0), (2300, 5003, "f16", 2), (1300, 9001, "f32", 0), (800, 33001, "f32", 0), (800, 33001, "f32", 3),
                                          (700, 50021, "bf16", 0)])
def test_rows_that_a_workgroup_takes_one_after_the_other(T, V, kind, pad, tail):
    """Rows that begin anywhere in a vector, more of them than workgroups: vectors shared by two rows, which other workgroups may hold, and
    the ring of slots.  In place as well: a row's gradient is written while the next rows are read."""
    s = problem(T, V, 30, kind, tail, 1.0, V, mapped=True, pad=pad)
    more = {"teacher_lse": s["lse"], "teacher_row": s["at"], "grad_loss": s["g"]}
    loss, dz = pkg.sdtw_distill_step(s["z"], s["t"], s["ids"], **more)
    rows = torch.unique(torch.cat([torch.arange(0, T, 97), torch.arange(T - 5, T)])).cuda()
    pick = lambda x: None if x is None else f64(x[rows])  # noqa: E731
    want = reference(pick(s["z"]), f64(s["t"]), s["ids"].cpu().numpy(), 1.0, None if s["lse"] is None else f64(s["lse"]),
                     s["at"][rows].cpu().numpy(), pick(s["g"]))
    check_loss(loss[rows], want[0])
    check_grad(dz[rows], want[1], want[2], kind)
    # Every row's gradient sums to 0: to a rounding of its type for each element, and 4e-6 of Q p, of q and of the tail's share, 1 each in sum.
    free = (s["at"] < 0)
    assert (loss[free] == 0).all() and (dz[free] == 0).all()
    size = dz.double().abs().sum(1)
    assert (dz.double().sum(1).abs() <= HALF_ULP[kind] * size + 12e-6 * s["g"].double() + V * LEAST[kind]).all()
    room = torch.empty((T, V + pad), dtype=TYPES[kind], device="cuda").fill_(7.0)
    room[:, :V] = s["z"]
    loss_in, _ = pkg.sdtw_distill_step(room[:, :V], s["t"], s["ids"], dlogits=room[:, :V], **more)
    assert torch.equal(room[:, :V], dz) and torch.equal(loss_in, loss) and (room[:, V:] == 7.0).all()


@pytest.mark.parametrize("scaled", [False, True])
@pytest.mark.parametrize("kind,most", [("f32", 1 << 16), ("f16", 1 << 11), ("bf16", 1 << 8)])
@pytest.mark.parametrize("B,H,N,M", [(3, 2, 2048, 2050), (40, 1, 600, 700), (2, 3, 65, 9000)])
def test_bias_gradient_of_sums_beyond_float32(B, H, N, M, kind, most, scaled):
    """Whole numbers whose sums over 64 rows of a diagonal are below 2^24, and over a bucket far above: carried in 64 bits they are exact, and
    the table's entry is the sum rounded once.  (Weights of a few bits leave them exact.)"""
    gen = torch.Generator(device="cuda").manual_seed(M)
    g = torch.randint(most // 2, most + 1, (B, H, N, M), generator=gen, device="cuda")
    g = (g * 2 - 1 if kind == "f32" else g).to(TYPES[kind])
    scale = (torch.randint(32, 64, (B,), generator=gen, device="cuda") * 2 + 1).float() / 128 if scaled else None
    dt = pkg.sdtw_position_bias_backward(g, 32, scale=scale)
    at = torch.from_numpy(bucket_matrix(N, M, 32, 128, True, 0)).cuda()
    total = (g.double() * (1.0 if scale is None else scale.double()[:, None, None, None])).sum(0)
    want = torch.stack([torch.stack([(total[h] * (at == u)).sum() for u in range(32)]) for h in range(H)])
    assert float(want.abs().max()) > 2 ** 25
    assert torch.equal(dt, want.float())


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("B,H,N,M,lengths", [(4, 2, 900, 1100, True), (2, 1, 3000, 500, False), (1, 4, 130, 4100, True)])
def test_bias_gradient_of_real_numbers(B, H, N, M, lengths, kind):
    """Up to 64 terms of a diagonal are added in float32, the rest in 64 bits: an entry is off by (1 + 2^-24)^63 - 1 < 64 * 2^-24 of the sum of what
    it adds up in magnitude at most, and by one rounding."""
    gen = torch.Generator(device="cuda").manual_seed(N)
    g = torch.randn((B, H, N, M), generator=gen, device="cuda").to(TYPES[kind])
    scale = torch.rand(B, generator=gen, device="cuda") + 0.1
    rlen = torch.randint(N // 2, N + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if lengths else None
    clen = torch.randint(M // 2, M + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if lengths else None
    dt = pkg.sdtw_position_bias_backward(g, 64, max_distance=700, two_sided=False, row_len=rlen, col_len=clen, scale=scale).double()
    w = g.double() * scale.double()[:, None, None, None]
    if lengths:
        inside = (torch.arange(N, device="cuda")[:, None] < rlen[:, None, None]) & (torch.arange(M, device="cuda") < clen[:, None, None])
        w = w * inside[:, None]
    at = torch.from_numpy(bucket_matrix(N, M, 64, 700, False, 0)).cuda()
    for h in range(H):
        for u in range(64):
            part = w[:, h][:, at == u]
            want, size = float(part.sum()), float(part.abs().sum())
            assert abs(float(dt[h, u]) - want) <= 64 * 2.0 ** -24 * size + 2.0 ** -24 * abs(want) + 1e-12 * size, (h, u)


def test_bias_refuses_numbers_that_a_descriptor_does_not_hold():
    plane, table = torch.zeros((1, 1, 4, 4), device="cuda"), torch.zeros((1, 32), device="cuda")
    for bad in (dict(offset=1 << 64), dict(offset=0.5), dict(offset=(1 << 63) + 7), dict(max_distance=(1 << 32) + 128), dict(max_distance=64.5)):
        with pytest.raises(ValueError):
            pkg.sdtw_position_bias_forward(table, plane, **bad)
        with pytest.raises(ValueError):
            pkg.sdtw_position_bias_backward(plane, 32, **bad)
        with pytest.raises(ValueError):
            pkg.sdtw_forward_biased(plane[0], plane[0], table, 1.0, **bad)
    with pytest.raises(ValueError):
        pkg.sdtw_position_bias_backward(plane, (1 << 32) + 32)


def test_distillation_of_an_empty_batch():
    z, t = torch.zeros((0, 10), device="cuda", dtype=torch.bfloat16), torch.zeros((0, 3), device="cuda")
    ids = torch.zeros((0, 3), dtype=torch.int32, device="cuda")
    for more in ({}, {"teacher_lse": torch.zeros(0, device="cuda")}, {"teacher_row": torch.zeros(0, dtype=torch.int32, device="cuda")}):
        loss, stats = pkg.sdtw_distill_forward(z, t, ids, **more)
        assert loss.shape == (0,) and pkg.sdtw_distill_backward(z, t, ids, stats, **more).shape == (0, 10)
        loss, dz = pkg.sdtw_distill_step(z, t, ids, **more)
        assert loss.shape == (0,) and dz.shape == (0, 10)
