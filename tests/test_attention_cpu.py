"""Host-side checks of the attention and clipping entry points that need no GPU: what is refused, before any device work; sizes of
workspaces."""
import ctypes

import pytest

import paper_2602_17206_amd as pkg
from paper_2602_17206_amd import binding

FAKE, OTHER, THIRD, FOURTH = (ctypes.c_void_p(0x10000 * n) for n in (1, 2, 3, 4))  # never dereferenced
INVALID, UNSUPPORTED, WORKSPACE, OK = binding.STATUS_INVALID_ARG, binding.STATUS_UNSUPPORTED, binding.STATUS_WORKSPACE, binding.STATUS_OK


def desc(**kw):
    q, k = (384, 64, 16, 1), (448, 64, 16, 1)
    a = dict(B=2, H=4, Hk=2, N=6, M=7, D=16, type=2, table_type=0, buckets=32, max_distance=128, two_sided=1, causal=0, scale=0.25, cap=0.0, flags=0,
             offset=0, prefix=0, q_stride=q, k_stride=(224, 32, 16, 1), v_stride=(224, 112, 16, 1), out_stride=(384, 96, 16, 1), dout_stride=q,
             dq_stride=(384, 16, 64, 1), dk_stride=(224, 112, 16, 1), dv_stride=(224, 16, 32, 1), table_stride=(32, 1))
    a.update(kw)
    d = binding.AttentionDesc()
    for name, v in a.items():
        if isinstance(v, tuple):
            getattr(d, name)[:] = list(v)
        else:
            setattr(d, name, v)
    return d


def forward(d, q=FAKE, k=FAKE, v=FAKE, table=FAKE, lists=None, out=OTHER, lse=OTHER, ws=FAKE, nbytes=1 << 40):
    return pkg.load_library().sdtw_attention_forward(ctypes.byref(d) if d else None, q, k, v, table, lists, out, lse, ws, nbytes, None)


def backward(d, q=FAKE, k=FAKE, v=FAKE, table=FAKE, lists=None, out=FAKE, lse=FAKE, dout=FAKE, dq=OTHER, dk=THIRD, dv=FOURTH, dtable=OTHER, ws=FAKE,
             nbytes=1 << 40):
    return pkg.load_library().sdtw_attention_backward(ctypes.byref(d) if d else None, q, k, v, table, lists, out, lse, dout, dq, dk, dv, dtable, ws,
                                                      nbytes, None)


def sizes(d):
    lib = pkg.load_library()
    return lib.sdtw_attention_forward_workspace_bytes(ctypes.byref(d)), lib.sdtw_attention_backward_workspace_bytes(ctypes.byref(d))


def test_struct_sizes_match_the_header_layout():
    assert ctypes.sizeof(binding.AttentionDesc) == 64 + 16 + 8 * 32 + 16
    assert ctypes.sizeof(binding.AttentionLists) == 48


@pytest.mark.parametrize("kw", [
    dict(B=-1), dict(H=-1), dict(Hk=0), dict(Hk=3), dict(N=-1), dict(M=-1), dict(N=(1 << 28) + 1), dict(M=(1 << 28) + 1), dict(D=0), dict(type=3),
    dict(type=-1), dict(flags=1), dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(scale=2.0 ** -27), dict(scale=2.0 ** 27),
    dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(cap=1e-45), dict(offset=1 << 62), dict(offset=-(1 << 62)), dict(prefix=-1, causal=1),
    dict(prefix=1), dict(buckets=-1), dict(buckets=3), dict(buckets=258), dict(buckets=1, two_sided=0), dict(max_distance=8), dict(max_distance=1 << 25),
    dict(two_sided=2), dict(table_type=5), dict(table_stride=(-1, 1)), dict(q_stride=(-1, 64, 16, 1)), dict(k_stride=(224, 112, 16, -1)),
    dict(v_stride=(1 << 60, 112, 16, 1)),
])
def test_invalid_attention_descriptors_are_refused(kw):
    d = desc(**kw)
    assert sizes(d) == (0, 0)
    assert forward(d) == INVALID and backward(d) == INVALID


def test_more_features_than_there_are_kernels_for():
    d = desc(D=129, q_stride=(3096, 774, 129, 1), out_stride=(3096, 774, 129, 1))
    assert sizes(d) == (0, 0) and forward(d) == UNSUPPORTED and backward(d) == UNSUPPORTED


def test_attention_pointers_strides_and_workspace():
    assert forward(None) == INVALID and backward(None) == INVALID
    d = desc()
    f, b = sizes(d)
    assert f > 0 and b > 0 and f % 256 == 0 and b % 256 == 0
    for name in ("q", "k", "v", "table", "out", "lse"):
        assert forward(d, **{name: None}) == INVALID, name
    for name in ("q", "k", "v", "table", "out", "lse", "dout", "dq", "dk", "dv"):
        assert backward(d, **{name: None}) == INVALID, name
    plain = desc(buckets=0)
    assert forward(plain) == INVALID                       # a table without buckets
    assert backward(plain, table=None) == INVALID          # ... or its gradient
    for ws, nbytes in ((None, f), (ctypes.c_void_p(0x10010), f), (FAKE, f - 1)):
        assert forward(d, ws=ws, nbytes=nbytes) == WORKSPACE
    for ws, nbytes in ((None, b), (ctypes.c_void_p(0x10010), b), (FAKE, b - 1)):
        assert backward(d, ws=ws, nbytes=nbytes) == WORKSPACE
    # elements of an output that share memory, or features apart
    for stride in ((0, 96, 16, 1), (384, 64, 16, 1), (384, 96, 15, 1), (384, 96, 16, 2), (384, 16, 16, 1)):
        assert forward(desc(out_stride=stride)) == INVALID, stride
        assert backward(desc(dq_stride=stride)) == INVALID, stride
    for stride in ((0, 112, 16, 1), (224, 112, 15, 1), (111, 112, 16, 1), (224, 112, 16, 0)):
        assert backward(desc(dk_stride=stride)) == INVALID, stride
        assert backward(desc(dv_stride=stride)) == INVALID, stride


def test_outputs_in_the_place_of_inputs_are_refused():
    fifth = ctypes.c_void_p(0x50000)
    for name in ("q", "k", "v", "table"):
        assert forward(desc(), **{name: OTHER}) == INVALID, name
    for out in ("dq", "dk", "dv"):
        for name in ("q", "k", "v", "table", "out", "dout"):
            assert backward(desc(), **{name: fifth, out: fifth}) == INVALID, (out, name)
    for a, b in (("dq", "dk"), ("dq", "dv"), ("dk", "dv")):
        assert backward(desc(), **{a: fifth, b: fifth}) == INVALID, (a, b)


def test_attention_lists():
    lists = binding.AttentionLists()
    d, ref = desc(), ctypes.byref(lists)
    lists.prefixes = 0x10000
    assert forward(d, lists=ref) == INVALID and backward(d, lists=ref) == INVALID  # a prefix belongs to a causal mask
    lists.prefixes, lists.row_document = None, 0x10000
    assert forward(d, lists=ref) == INVALID and backward(d, lists=ref) == INVALID  # documents of rows and of keys go together
    lists.row_document, lists.col_document = None, 0x10000
    assert forward(d, lists=ref) == INVALID and backward(d, lists=ref) == INVALID


def test_an_empty_list_of_documents_has_no_place():
    lists = binding.AttentionLists()
    lists.col_document = FAKE
    assert forward(desc(), lists=ctypes.byref(lists)) == INVALID and backward(desc(), lists=ctypes.byref(lists)) == INVALID
    assert forward(desc(N=0), lists=ctypes.byref(lists)) == OK and backward(desc(N=0, M=0), lists=ctypes.byref(lists), dtable=None) == OK


def test_nothing_to_do():
    for kw in (dict(B=0), dict(H=0), dict(N=0)):
        assert forward(desc(**kw), q=None, k=None, v=None, table=None, out=None, lse=None, ws=None, nbytes=0) == OK
    for kw in (dict(B=0), dict(N=0, M=0), dict(H=0, M=0)):
        none = dict.fromkeys(("q", "k", "v", "table", "out", "lse", "dout", "dq", "dk", "dv", "dtable", "ws"))
        assert backward(desc(**kw), **none, nbytes=0) == OK


def test_problems_that_need_more_workgroups_than_there_are():
    most = (1 << 31) - 1
    for kw in (dict(B=1 << 20, H=1 << 20, Hk=1 << 20), dict(B=most, H=most, Hk=most, N=1 << 28, M=1 << 28),
               dict(B=1 << 20, H=1, Hk=1, M=1 << 28, N=1 << 28), dict(B=most, H=most, Hk=1, N=1 << 28, M=1 << 28), dict(B=1 << 12, H=1 << 12, Hk=1, N=1 << 20)):
        d = desc(**{**kw, **{s: (0, 0, 0, 1) for s in ("q_stride", "k_stride", "v_stride", "dout_stride")}})
        assert sizes(d)[0] == 0 or sizes(d)[1] == 0
        assert forward(d) == INVALID and backward(d) == INVALID


# ---------------------------------------------------------------- clipping

def gradients(*entries):
    words = (ctypes.c_int64 * (4 * max(1, len(entries))))()
    for i, (data, out, count, kind, out_kind) in enumerate(entries):
        words[4 * i:4 * i + 4] = [data, out, count, kind | out_kind << 32]
    return words, len(entries)


def clip(entries, max_norm=1.0, norm=OTHER, ws=FAKE, nbytes=1 << 30):
    words, n = gradients(*entries)
    return pkg.load_library().sdtw_gradient_clip(words if n else None, n, max_norm, norm, ws, nbytes, None)


@pytest.mark.parametrize("entry", [(0x1000, 0x1000, -1, 0, 0), (0x1000, 0x1000, 1 << 48, 0, 0), (0x1000, 0x1000, 5, 3, 0), (0x1000, 0x1000, 5, 0, 7), (0, 0x1000, 5, 0, 0),
                                   (0x1000, 0, 5, 0, 0), (0x1000, 0x1000, 5, 0, 1)])
def test_invalid_gradients_are_refused(entry):
    words, n = gradients(entry)
    assert pkg.load_library().sdtw_gradient_clip_workspace_bytes(words, n) == 0
    assert clip([entry]) == INVALID


def test_clip_arguments():
    fine = (0x1000, 0x1000, 100, 0, 0)
    lib = pkg.load_library()
    need = lib.sdtw_gradient_clip_workspace_bytes(*gradients(fine))
    assert need > 0 and need % 256 == 0
    assert lib.sdtw_gradient_clip_workspace_bytes(None, 0) > 0
    assert lib.sdtw_gradient_clip_workspace_bytes(None, 1) == 0 and lib.sdtw_gradient_clip_workspace_bytes(None, -1) == 0
    for bad in (-1.0, float("nan"), -float("inf")):
        assert clip([fine], max_norm=bad) == INVALID
    assert clip([fine], norm=None) == INVALID
    for ws, nbytes in ((None, need), (ctypes.c_void_p(0x10010), need), (FAKE, need - 256)):
        assert clip([fine], ws=ws, nbytes=nbytes) == WORKSPACE


@pytest.mark.parametrize("entries", [
    [(0x1000, 0x1000, 100, 0, 0), (0x1000, 0x1000, 100, 0, 0)],     # the same tensor twice
    [(0x1000, 0x1000, 100, 0, 0), (0x118c, 0x118c, 100, 0, 0)],     # the last element is another's first
    [(0x1000, 0x2000, 100, 0, 0), (0x2004, 0x2004, 1, 0, 0)],       # written into a gradient
    [(0x1000, 0x3000, 100, 0, 0), (0x2000, 0x3100, 100, 0, 0)],     # two outputs
    [(0x1000, 0x1004, 100, 0, 0)],                                  # into its own memory, elsewhere
    [(0x1000, 0x0f00, 100, 1, 0)],
    [(0x1000, 0x2000, 100, 0, 0), (0x1f00, 0x4000, 1000, 2, 2), (0x9000, 0x9000, 3, 0, 0)],
])
def test_outputs_that_overlap_are_refused(entries):
    assert clip(entries) == INVALID
    assert clip(entries[::-1]) == INVALID


@pytest.mark.filterwarnings("ignore::UserWarning")
def test_tensors_on_another_device_are_refused():
    """What a call is given beside its inputs lies on their device too.  (Tensors without memory, so that this needs no device.)"""
    torch = pytest.importorskip("torch")
    from torch._subclasses.fake_tensor import FakeTensorMode

    with FakeTensorMode():
        make = lambda *s, at=0: torch.empty(s, device="cuda:%d" % at)  # noqa: E731
        q, out, lse, table = make(1, 2, 3, 16), make(1, 2, 3, 16), make(1, 2, 3), make(2, 16)
        workspace = pkg.Workspace.__new__(pkg.Workspace)
        workspace.nbytes, workspace.buffer = 1 << 20, torch.empty(1 << 20, dtype=torch.uint8, device="cuda:1")
        for kw in (dict(lse=make(1, 2, 3, at=1)), dict(workspace=workspace)):
            with pytest.raises(ValueError, match="must be on cuda:0"):
                pkg.sdtw_attention_forward(q, q, q, table, **kw)
        for kw in (dict(lse=make(1, 2, 3, at=1)), dict(dtable=make(2, 16, at=1)), dict(workspace=workspace)):
            a = {"lse": lse, **kw}
            with pytest.raises(ValueError, match="must be on cuda:0"):
                pkg.sdtw_attention_backward(q, q, q, out, a.pop("lse"), out, table, **a)
        for kw in (dict(norm=make(at=1)), dict(workspace=workspace)):
            with pytest.raises(ValueError, match="must be on cuda:0"):
                pkg.sdtw_gradient_clip([make(0)], 1.0, **kw)


def test_statistics_in_the_place_of_inputs_and_outputs_are_refused():
    fifth = ctypes.c_void_p(0x50000)
    for name in ("q", "k", "v", "table"):
        assert forward(desc(), **{name: fifth, "lse": fifth}) == INVALID, name
    assert forward(desc(), out=fifth, lse=fifth) == INVALID
    for out in ("dq", "dk", "dv"):
        assert backward(desc(), **{"lse": fifth, out: fifth}) == INVALID, out
        assert backward(desc(), **{"dtable": fifth, out: fifth}) == INVALID, out


def test_a_norm_within_a_gradient_is_refused():
    for at in (0x1000, 0x118c, 0x2000, 0x218c):
        assert clip([(0x1000, 0x2000, 100, 0, 0)], norm=ctypes.c_void_p(at)) == INVALID, hex(at)
        assert clip([(0x9000, 0x9000, 3, 0, 0), (0x1000, 0x2000, 100, 0, 0)], max_norm=float("inf"), norm=ctypes.c_void_p(at)) == INVALID, hex(at)
    for at in (0x0ffc, 0x1190, 0x1ffc, 0x2190):
        assert clip([(0x1000, 0x2000, 100, 0, 0)], norm=ctypes.c_void_p(at), ws=None) == WORKSPACE, hex(at)


@pytest.mark.parametrize("scale,cap,fine", [
    (2.0 ** -26, 2e38, False), (0.25, 2e38, False), (0.25, 2.0 ** 124, True), (0.25, 2.0 ** 125, False), (2.0 ** 26, 2.0 ** 127, True), (2.0 ** -26, 1e-40, False),
    (2.0 ** -26, 2.0 ** -126, True), (0.25, 2.0 ** -126, True), (2.0, 2.0 ** -126, True), (4.0, 2.0 ** -126, False),
])
def test_caps_that_float32_cannot_divide_by_or_into(scale, cap, fine):
    # scale / cap would be a subnormal number or 0 (scores lose their digits, or are all 0), or 1 / cap infinite (gradients NaN)
    d = desc(scale=scale, cap=cap)
    assert (sizes(d)[0] > 0) == (sizes(d)[1] > 0) == fine
    assert forward(d, ws=None) == backward(d, ws=None) == (WORKSPACE if fine else INVALID)


@pytest.mark.parametrize("kind,M,read", [(0, 300, True), (1, 300, False), (2, 512, False), (1, 513, True)])
def test_workspaces_hold_no_copy_that_nothing_reads(kind, M, read):
    # outputs whose rows are far apart are packed where delta comes from them; 16-bit gradients over few keys take it from the keys
    B, H, N, D = 2, 4, 64, 24
    rows, keys = (N * H * D, N * D, D, 1), (M * 2 * D, M * D, D, 1)
    near, far = (sizes(desc(N=N, M=M, D=D, type=kind, buckets=0, q_stride=rows, dout_stride=rows, dq_stride=rows, k_stride=keys, v_stride=keys, dk_stride=keys,
                            dv_stride=keys, out_stride=out))[1] for out in (rows, (N * H << 22, N << 22, 1 << 22, 1)))
    assert far - near == (B * H * N * D * (4 if kind == 0 else 2) if read else 0)
