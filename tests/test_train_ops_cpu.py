"""Host-side checks of the distillation and position-bias entry points that need no GPU: what is refused, before any
device work; sizes of workspaces; the buckets' first distances against whole-number arithmetic."""
import ctypes

import pytest
import torch

import paper_2602_17206_amd as pkg
from paper_2602_17206_amd import binding

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced


def distill_desc(**kw):
    a = dict(rows=4, vocab=100, top=8, teacher_rows=4, temperature=1.0, target=0, logit_type=0, teacher_type=0, id_type=1, flags=0,
             logit_stride=100, grad_stride=100, teacher_stride=8, id_stride=8)
    a.update(kw)
    return binding.DistillDesc(**a)


def bias_desc(**kw):
    a = dict(B=2, H=3, N=8, M=9, buckets=32, max_distance=128, two_sided=1, plane_type=0, table_type=0, flags=0, offset=0,
             in_stride=(216, 72, 9), out_stride=(216, 72, 9), table_stride=(32, 1))
    a.update(kw)
    d = binding.BiasDesc()
    for k, v in a.items():
        if isinstance(v, tuple):
            getattr(d, k)[:] = list(v)
        else:
            setattr(d, k, v)
    return d


def test_struct_sizes_match_the_header_layout():
    assert ctypes.sizeof(binding.DistillDesc) == 72
    assert ctypes.sizeof(binding.BiasDesc) == 112


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(vocab=0), dict(vocab=1 << 30, logit_stride=1 << 30, grad_stride=1 << 30), dict(top=0), dict(top=1025, teacher_stride=2000, id_stride=2000),
    dict(teacher_rows=0), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")),
    dict(temperature=float("inf")), dict(temperature=1e-45), dict(target=2), dict(logit_type=3), dict(teacher_type=-1), dict(id_type=2), dict(flags=1),
    dict(logit_stride=99), dict(grad_stride=99), dict(teacher_stride=7), dict(id_stride=7), dict(logit_stride=1 << 62),
])
def test_invalid_distillation_descriptors_are_refused(kw):
    lib = pkg.load_library()
    d = distill_desc(**kw)
    assert lib.sdtw_distill_workspace_bytes(ctypes.byref(d)) == 0
    tail = FAKE if kw.get("target", 0) else None
    assert lib.sdtw_distill_forward(ctypes.byref(d), FAKE, FAKE, FAKE, tail, None, FAKE, FAKE, FAKE, 1 << 30, None) == 1
    assert lib.sdtw_distill_backward(ctypes.byref(d), FAKE, FAKE, FAKE, tail, None, None, FAKE, FAKE, None) == 1
    assert lib.sdtw_distill_step(ctypes.byref(d), FAKE, FAKE, FAKE, tail, None, None, FAKE, FAKE, FAKE, 1 << 30, None) == 1


def test_distillation_pointers_and_workspace():
    lib = pkg.load_library()
    d = distill_desc()
    need = lib.sdtw_distill_workspace_bytes(ctypes.byref(d))
    assert need > 0 and need % 256 == 0
    ok = [FAKE, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, need, None]

    def forward(desc=d, **at):
        a = list(ok)
        for i, v in at.items():
            a[int(i[1:])] = v
        return lib.sdtw_distill_forward(ctypes.byref(desc), *a)

    for i in (0, 1, 2, 5, 6):
        assert forward(**{"a%d" % i: None}) == binding.STATUS_INVALID_ARG, i
    assert forward(a3=FAKE) == binding.STATUS_INVALID_ARG                         # renormalised targets take no teacher_lse
    assert forward(distill_desc(target=1)) == binding.STATUS_INVALID_ARG          # a tail needs it
    assert forward(distill_desc(teacher_rows=3)) == binding.STATUS_INVALID_ARG    # fewer rows than the student, and no map
    assert forward(a7=None) == binding.STATUS_WORKSPACE
    assert forward(a7=ctypes.c_void_p(0x10010)) == binding.STATUS_WORKSPACE
    assert forward(a8=need - 1) == binding.STATUS_WORKSPACE
    other = ctypes.c_void_p(0x20000)
    bad = distill_desc(logit_stride=128)  # in place needs one stride
    assert lib.sdtw_distill_backward(ctypes.byref(bad), FAKE, other, other, None, None, None, other, FAKE, None) == binding.STATUS_INVALID_ARG
    assert lib.sdtw_distill_backward(ctypes.byref(d), FAKE, other, other, None, None, None, None, other, None) == binding.STATUS_INVALID_ARG
    assert lib.sdtw_distill_step(ctypes.byref(d), FAKE, other, other, None, None, None, other, None, FAKE, need, None) == binding.STATUS_INVALID_ARG
    assert lib.sdtw_distill_forward(None, *ok) == binding.STATUS_INVALID_ARG


def test_no_rows_is_nothing_to_do():
    lib = pkg.load_library()
    d = distill_desc(rows=0)
    assert lib.sdtw_distill_workspace_bytes(ctypes.byref(d)) > 0
    assert lib.sdtw_distill_forward(ctypes.byref(d), *[None] * 8, 0, None) == binding.STATUS_OK
    assert lib.sdtw_distill_backward(ctypes.byref(d), *[None] * 9) == binding.STATUS_OK
    assert lib.sdtw_distill_step(ctypes.byref(d), *[None] * 9, 0, None) == binding.STATUS_OK
    for kw in (dict(B=0), dict(H=0), dict(N=0), dict(M=0)):
        assert lib.sdtw_position_bias_forward(ctypes.byref(bias_desc(**kw)), *[None] * 7) == binding.STATUS_OK
    assert lib.sdtw_position_bias_backward(ctypes.byref(bias_desc(H=0)), *[None] * 7, 0, None) == binding.STATUS_OK


@pytest.mark.parametrize("kw", [
    dict(B=-1), dict(H=-1), dict(N=-1), dict(M=-1), dict(N=1 << 30), dict(buckets=2), dict(buckets=33), dict(buckets=258), dict(buckets=1, two_sided=0),
    dict(buckets=257, two_sided=0), dict(max_distance=8), dict(max_distance=(1 << 24) + 1), dict(two_sided=2), dict(plane_type=3),
    dict(table_type=-1), dict(flags=2), dict(offset=1 << 62), dict(offset=-(1 << 62)), dict(in_stride=(-1, 72, 9)),
    dict(in_stride=(1 << 60, 72, 9)),
])
def test_invalid_bias_descriptors_are_refused(kw):
    lib = pkg.load_library()
    d = bias_desc(**kw)
    assert lib.sdtw_position_bias_workspace_bytes(ctypes.byref(d)) == 0
    assert lib.sdtw_position_bias_starts(ctypes.byref(d), FAKE) == binding.STATUS_INVALID_ARG
    assert lib.sdtw_position_bias_forward(ctypes.byref(d), FAKE, FAKE, None, None, None, FAKE, None) == binding.STATUS_INVALID_ARG
    assert lib.sdtw_position_bias_backward(ctypes.byref(d), FAKE, None, None, None, None, FAKE, FAKE, 1 << 30, None) == binding.STATUS_INVALID_ARG


def test_bias_pointers_strides_and_workspace():
    lib = pkg.load_library()
    other = ctypes.c_void_p(0x20000)

    def forward(d, table=FAKE, inp=FAKE, out=other):
        return lib.sdtw_position_bias_forward(ctypes.byref(d), table, inp, None, None, None, out, None)

    assert forward(bias_desc(), table=None) == binding.STATUS_INVALID_ARG
    assert forward(bias_desc(), out=None) == binding.STATUS_INVALID_ARG
    for strides in ((0, 72, 9), (216, 72, 8), (72, 72, 9), (216, 71, 9)):  # cells of `out` that share memory
        assert forward(bias_desc(out_stride=strides)) == binding.STATUS_INVALID_ARG, strides
    assert forward(bias_desc(in_stride=(0, 72, 9)), inp=FAKE, out=FAKE) == binding.STATUS_INVALID_ARG  # in place: the same strides
    d = bias_desc()
    need = lib.sdtw_position_bias_workspace_bytes(ctypes.byref(d))
    assert need > 0

    def backward(grad=FAKE, dtable=FAKE, ws=FAKE, nbytes=need):
        return lib.sdtw_position_bias_backward(ctypes.byref(d), grad, None, None, None, None, dtable, ws, nbytes, None)

    assert backward(grad=None) == binding.STATUS_INVALID_ARG
    assert backward(dtable=None) == binding.STATUS_INVALID_ARG
    assert backward(ws=None) == binding.STATUS_WORKSPACE
    assert backward(ws=ctypes.c_void_p(0x10010)) == binding.STATUS_WORKSPACE
    assert backward(nbytes=need - 1) == binding.STATUS_WORKSPACE


def test_planes_that_need_more_workgroups_than_there_are():
    lib = pkg.load_library()
    most = (1 << 31) - 1
    for kw in (dict(B=1, H=1 << 20, N=(1 << 30) - 1, M=(1 << 30) - 1), dict(B=most, H=most, N=1 << 20, M=1 << 20), dict(B=1, H=1, N=(1 << 30) - 1, M=(1 << 30) - 1)):
        d = bias_desc(in_stride=(0, 0, 0), out_stride=(0, 0, 0), **kw)
        assert lib.sdtw_position_bias_workspace_bytes(ctypes.byref(d)) == 0
        assert lib.sdtw_position_bias_backward(ctypes.byref(d), FAKE, None, None, None, None, FAKE, FAKE, 1 << 40, None) == binding.STATUS_INVALID_ARG


def starts_in_whole_numbers(n, D):
    e = n // 2
    m = n - e
    out = list(range(e))
    for k in range(m):
        lo, hi = 0, D  # the smallest d with d^m >= e^(m-k) D^k
        while lo < hi:
            mid = (lo + hi) // 2
            if mid ** m >= e ** (m - k) * D ** k:
                hi = mid
            else:
                lo = mid + 1
        out.append(lo)
    return out


@pytest.mark.parametrize("n,D", [(2, 2), (2, 1 << 24), (3, 5), (8, 50), (16, 128), (16, 256), (32, 128), (32, 1024), (33, 1000), (64, 1024), (64, 1 << 20),
                                 (128, 65), (128, 4096), (127, 16777213), (6, 24), (4, 2 * 3 ** 10), (10, 5 * 7 ** 5)])
@pytest.mark.parametrize("two_sided", [False, True])
def test_bucket_starts_are_whole_number_roots(n, D, two_sided):
    assert pkg.sdtw_position_bias_starts(2 * n if two_sided else n, D, two_sided) == starts_in_whole_numbers(n, D)


def test_the_binding_checks_its_tensors():
    z, t, ids = torch.zeros(4, 10), torch.zeros(4, 2), torch.zeros(4, 2, dtype=torch.int64)
    with pytest.raises(ValueError):
        pkg.sdtw_distill_forward(z, t, ids)  # host tensors
    with pytest.raises(ValueError):
        pkg.sdtw_position_bias_forward(torch.zeros(2, 32), torch.zeros(1, 2, 3, 3))
    with pytest.raises(ValueError):
        pkg.sdtw_position_bias_backward(torch.zeros(1, 2, 3, 3), 32)
    with pytest.raises(pkg.SdtwError):
        pkg.sdtw_position_bias_starts(33, 128, True)


def test_position_penalty_entry_points_refuse():
    lib = pkg.load_library()
    d = binding.make_desc(6, 8, 9, 4, 1.0, pkg.UNFUSED)
    b = bias_desc()
    need = lib.sdtw_biased_workspace_bytes(ctypes.byref(d), ctypes.byref(b))
    assert need > pkg.sdtw_workspace_bytes(d) + 4 * 6 * 8 * 9

    def both(d, b, ws=FAKE, nbytes=need, x=FAKE, table=FAKE):
        f = lib.sdtw_forward_biased(ctypes.byref(d), ctypes.byref(b), x, FAKE, table, None, None, FAKE, ws, nbytes, None)
        r = lib.sdtw_backward_biased(ctypes.byref(d), ctypes.byref(b), x, FAKE, table, None, None, None, FAKE, FAKE, FAKE, None, ws, nbytes, None)
        return {f, r}

    for kw in (dict(B=3), dict(H=1), dict(N=9), dict(M=8), dict(plane_type=1), dict(buckets=31), dict(B=0, H=0), dict(table_type=5)):
        assert lib.sdtw_biased_workspace_bytes(ctypes.byref(d), ctypes.byref(bias_desc(**kw))) == 0, kw
        assert both(d, bias_desc(**kw)) == {binding.STATUS_INVALID_ARG}, kw
    assert both(binding.make_desc(6, 8, 9, 4, 1.0, pkg.FUSED), b) == {binding.STATUS_UNSUPPORTED}
    assert both(binding.make_desc(6, 8, 9, 4, -1.0, pkg.UNFUSED), b) == {binding.STATUS_INVALID_ARG}
    assert both(d, b, x=None) == {binding.STATUS_INVALID_ARG}
    assert both(d, b, table=None) == {binding.STATUS_INVALID_ARG}
    assert both(d, b, ws=None) == {binding.STATUS_WORKSPACE}
    assert both(d, b, nbytes=need - 1) == {binding.STATUS_WORKSPACE}


@pytest.mark.parametrize("B,N,M,D", [(6, 8, 9, 4), (32, 1024, 1024, 128), (32, 8192, 8192, 128)])
def test_values_alone_need_no_more_workspace_than_without_a_penalty(B, N, M, D):
    lib = pkg.load_library()
    b = bias_desc(B=B // 2, H=2, N=N, M=M)
    for flags in (binding.FLAG_VALUE_ONLY, binding.FLAG_VALUE_ONLY | binding.FLAG_MIN_MEMORY):
        d = binding.make_desc(B, N, M, D, 1.0, pkg.UNFUSED, flags=flags)
        need = lib.sdtw_biased_workspace_bytes(ctypes.byref(d), ctypes.byref(b))
        assert pkg.sdtw_workspace_bytes(d) <= need < pkg.sdtw_workspace_bytes(d) + 256
        args = [FAKE, FAKE, FAKE, None, None, FAKE, FAKE]
        assert lib.sdtw_forward_biased(ctypes.byref(d), ctypes.byref(b), *args, need - 256, None) == binding.STATUS_WORKSPACE
        assert lib.sdtw_biased_workspace_bytes(ctypes.byref(d), ctypes.byref(bias_desc(B=B // 2, H=2, N=N, M=M, buckets=31))) == 0


def test_grids_of_2_to_the_32_threads_are_refused():
    """Short rows take a quarter of a workgroup of 256 threads each, rows with many slots a workgroup, planes one at least."""
    lib = pkg.load_library()
    other = ctypes.c_void_p(0x20000)
    for kw in (dict(rows=1 << 26, teacher_rows=1 << 26), dict(rows=1 << 25, teacher_rows=1 << 25, top=200, teacher_stride=200, id_stride=200),
               dict(rows=(1 << 31) - 1, teacher_rows=(1 << 31) - 1), dict(rows=1 << 25, teacher_rows=1 << 25, vocab=1 << 20, logit_stride=1 << 20, grad_stride=1 << 20)):
        d = distill_desc(**kw)
        ref = ctypes.byref(d)
        assert lib.sdtw_distill_forward(ref, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, FAKE, 1 << 50, None) == binding.STATUS_INVALID_ARG, kw
        assert lib.sdtw_distill_backward(ref, FAKE, FAKE, FAKE, None, None, None, FAKE, other, None) == binding.STATUS_INVALID_ARG, kw
        assert lib.sdtw_distill_step(ref, FAKE, FAKE, FAKE, None, None, None, FAKE, other, FAKE, 1 << 50, None) == binding.STATUS_INVALID_ARG, kw
    for kw in (dict(B=1, H=1 << 19, N=1, M=1), dict(B=1, H=1, N=1 << 29, M=1 << 29), dict(B=(1 << 31) - 1, H=(1 << 31) - 1, N=1, M=1)):
        d = bias_desc(in_stride=(0, 0, 0), **kw)
        assert lib.sdtw_position_bias_workspace_bytes(ctypes.byref(d)) == 0, kw
        assert lib.sdtw_position_bias_backward(ctypes.byref(d), FAKE, None, None, None, None, other, FAKE, 1 << 50, None) == binding.STATUS_INVALID_ARG, kw
    for kw in (dict(B=1 << 22, H=4, N=1, M=1, out_stride=(4, 1, 1)), dict(B=1, H=1, N=1 << 29, M=1 << 29, out_stride=(1, 1, 1 << 29))):
        d = bias_desc(in_stride=(0, 0, 0), **kw)
        assert lib.sdtw_position_bias_forward(ctypes.byref(d), FAKE, FAKE, None, None, None, other, None) == binding.STATUS_INVALID_ARG, kw
    # what just fits is still planned for
    d = bias_desc(B=1, H=(1 << 19) - 1, N=1, M=1)
    assert lib.sdtw_position_bias_workspace_bytes(ctypes.byref(d)) >= 8 * 32 * ((1 << 19) - 1)


def test_temperatures_whose_scale_is_beyond_float32_are_refused():
    lib = pkg.load_library()
    for temperature, fine in ((3e-39, False), (4.2e-39, False), (4.3e-39, True), (1e-30, True), (3e38, True)):
        d = distill_desc(temperature=temperature)
        assert (lib.sdtw_distill_workspace_bytes(ctypes.byref(d)) > 0) == fine, temperature
        if not fine:
            assert lib.sdtw_distill_step(ctypes.byref(d), FAKE, FAKE, FAKE, None, None, None, FAKE, FAKE, FAKE, 1 << 30, None) == binding.STATUS_INVALID_ARG


def test_numbers_that_a_descriptor_does_not_hold_are_refused():
    for buckets, far in ((32, (1 << 32) + 128), (32, 128.5), ((1 << 32) + 32, 128), (32.5, 128), (32, float("nan")), (32, float("inf"))):
        with pytest.raises((ValueError, OverflowError)):
            pkg.sdtw_position_bias_starts(buckets, far)
    assert pkg.sdtw_position_bias_starts(32.0, 128.0) == pkg.sdtw_position_bias_starts(32, 128)


def test_no_rows_of_the_teacher_either():
    lib = pkg.load_library()
    d = distill_desc(rows=0, teacher_rows=0)
    assert lib.sdtw_distill_workspace_bytes(ctypes.byref(d)) > 0
    assert lib.sdtw_distill_forward(ctypes.byref(d), *[None] * 8, 0, None) == binding.STATUS_OK
    assert lib.sdtw_distill_backward(ctypes.byref(d), *[None] * 9) == binding.STATUS_OK
    assert lib.sdtw_distill_step(ctypes.byref(d), *[None] * 9, 0, None) == binding.STATUS_OK
    for bad in (dict(rows=0, teacher_rows=-1), dict(rows=1, teacher_rows=0)):
        assert lib.sdtw_distill_workspace_bytes(ctypes.byref(distill_desc(**bad))) == 0
