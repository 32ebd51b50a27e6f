"""Attention where there are rows enough for the kernel of long ones - 1024 wavefronts of 32 rows - and keys for many of its tiles, in every type:
tiles that are filled while others are read, a running reference that rises from tile to tile, tiles near the diagonal and far from it.
Bars as in test_attention_gpu.py."""
import pytest
import torch

import paper_2602_17206_amd as pkg
from paper_2602_17206_amd import binding
from test_attention_gpu import TYPES, check, problem, some_table

pytestmark = pytest.mark.gpu


def own(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def kernels_of(call):
    """The names of the kernels that a call launches"""
    torch.cuda.synchronize()
    binding.debug_profile(True)
    try:
        call()
        torch.cuda.synchronize()
        return [name for name, _ in binding.debug_profile_read()]
    finally:
        binding.debug_profile(False)


def long_check(B, H, Hk, N, M, D, kind, **more):
    (q, k, v, _), _ = problem(B, H, Hk, N, M, D, kind)
    assert "attention_forward" in kernels_of(lambda: pkg.sdtw_attention_forward(q, k, v))
    check(B, H, Hk, N, M, D, kind, **more)


def masks(name, N, M):
    gen = torch.Generator().manual_seed(N)
    strewn = lambda n: torch.randint(-1, 3, (2, n), generator=gen, dtype=torch.int32).cuda()  # noqa: E731
    packed = lambda n: torch.sort(torch.randint(0, 4, (2, n), generator=gen, dtype=torch.int32), 1)[0].cuda()  # noqa: E731
    near, wide = dict(table=some_table(16, 16), max_distance=20, two_sided=False), dict(table=some_table(16, 128), max_distance=4096, two_sided=False)
    both = dict(table=some_table(16, 32), two_sided=True)
    return {
        "none": dict(),
        "causal near": dict(causal=True, **near),
        "causal wide": dict(causal=True, offset=own(M - N, 5), **wide),
        "both sides": dict(**both),
        "lengths": dict(row_len=own(N - 300, N), col_len=own(M, M // 3), **both),
        "prefix": dict(causal=True, prefix=own(M // 2, 70), offset=own(-200, 3), **near),
        "packed": dict(causal=True, row_document=packed(N), col_document=packed(M), **near),
        "strewn": dict(row_document=strewn(N), col_document=strewn(M)),
        "cap": dict(causal=True, cap=4.0, **near),
        "cap alone": dict(cap=3.0),
        "cap and all": dict(causal=True, cap=5.0, prefix=own(0, 333), row_len=own(N, N - 77), col_len=own(M - 1, M), row_document=packed(N),
                            col_document=packed(M), **both),
    }[name]


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("name", ["none", "causal near", "causal wide", "both sides", "lengths", "prefix", "packed", "strewn", "cap", "cap alone",
                                  "cap and all"])
def test_many_tiles(name, D, kind):
    long_check(2, 16, 4, 1030, 700, D, kind, **masks(name, 1030, 700))


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("H,Hk,N,M,D", [(32, 32, 1025, 257, 24), (32, 8, 1024, 1111, 80), (128, 128, 257, 513, 33), (16, 16, 2048, 321, 100)])
def test_other_shapes(H, Hk, N, M, D, kind):
    long_check(1, H, Hk, N, M, D, kind, causal=True, offset=M - N, table=some_table(H, 32), two_sided=False)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("size", [0.01, 6.0, 40.0])
def test_references_that_rise(size, kind):
    long_check(1, 32, 32, 1024, 700, 64, kind, size=size)


@pytest.mark.parametrize("kind", sorted(TYPES))
def test_a_training_step_of_2048_positions(kind):
    long_check(1, 16, 16, 2048, 2048, 64, kind, causal=True, table=some_table(16, 32), two_sided=False)


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("M", [300, 600])
def test_outputs_are_packed_where_they_are_read(M, kind):
    (q, k, v, dout), _ = problem(2, 4, 2, 70, M, 21, kind)
    out, lse = pkg.sdtw_attention_forward(q, k, v)
    few = M <= 512 and kind != "f32"
    assert kernels_of(lambda: pkg.sdtw_attention_backward(q, k, v, out, lse, dout)).count("attention_pack") == (4 if few else 5)
    check(2, 4, 2, 70, M, 21, kind)
