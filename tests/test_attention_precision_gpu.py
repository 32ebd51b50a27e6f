"""How far attention and its gradients are from 64 bits, in the 2-norm of each result, beside a plain chain in 32 bits that rounds once at the end.

The bars elsewhere are sums of worst cases: they say that a result is right, and do not notice a lost digit.  Here a result may be off by at most
  2 times what the chain is, in a 16-bit type: the chain rounds a result once.  The kernels also round the weights of p or ds once for the matrix
    cores (out, dv, dk), and take delta from a rounded `out` (dq, dk): at most three errors of that size that know nothing of each other, 1.73 of
    one of them;
  4 times, where the result has 32 bits: chain and kernels round a score and its exponent two to four times each, in other places and orders, the
    kernels' exponential is a step of the hardware's and lse is rounded to 32 bits in between.
(Where the chain is exact to the last bit, one step of the result's type is allowed all the same.)"""
import pytest
import torch

import paper_2602_17206_amd as pkg
from test_attention_gpu import HALF_ULP, INF, TYPES, bucket_matrix, problem, some_table, visible

pytestmark = pytest.mark.gpu


def chain(q, k, v, dout, table, dtype, causal=False, cap=0.0, offset=0, two_sided=True):
    (B, H, N, D), (_, Hk, M, _) = q.shape, k.shape
    found = {x: [] for x in ("out", "lse", "dq", "dk", "dv")}
    dtable = torch.zeros((H, table.shape[1] if table is not None else 1), dtype=dtype, device="cuda")
    seen = visible(N, M, 0, causal=causal, offset=offset)
    at = None if table is None else bucket_matrix(N, M, table.shape[1], 128, two_sided, offset)
    for b in range(B):
        rows, keys = {x: [] for x in ("out", "lse", "dq")}, {x: [0] * Hk for x in ("dk", "dv")}
        for h in range(H):
            g = h // (H // Hk)
            Q, K, V, G = (x.to(dtype) for x in (q[b, h], k[b, g], v[b, g], dout[b, h]))
            z = Q @ K.t() * D ** -0.5
            if cap:
                t = torch.tanh(z / cap)
                z = cap * t
            if at is not None:
                z = z + table[h].to(dtype)[at]
            z = z.masked_fill(~seen, -INF)
            p = torch.softmax(z, 1)
            rows["out"].append(p @ V)
            rows["lse"].append(torch.logsumexp(z, 1))
            p = torch.exp(z - rows["lse"][-1][:, None])
            dp = G @ V.t()
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            if at is not None:
                dtable[h] += torch.stack([ds[at == u].sum() for u in range(table.shape[1])])
            if cap:
                ds = ds * (1 - t * t)
            ds = ds * D ** -0.5
            rows["dq"].append(ds @ K)
            keys["dk"][g] = keys["dk"][g] + ds.t() @ Q
            keys["dv"][g] = keys["dv"][g] + p.t() @ G
        for x, y in (*rows.items(), *keys.items()):
            found[x].append(torch.stack(y))
    found = {x: torch.stack(y) for x, y in found.items()}
    if table is not None:
        found["dtable"] = dtable
    return found


@pytest.mark.parametrize("kind", sorted(TYPES))
@pytest.mark.parametrize("B,H,Hk,N,M,D,buckets,options", [
    (4, 2, 2, 96, 96, 16, 16, dict()),
    (1, 8, 2, 600, 600, 64, 32, dict(causal=True, two_sided=False)),
    (1, 8, 8, 600, 700, 64, 0, dict(causal=True, offset=100)),
    (1, 32, 8, 1030, 700, 128, 0, dict(cap=20.0)),
    (1, 16, 16, 2048, 2048, 64, 32, dict(causal=True, two_sided=False)),
    (2, 8, 2, 2, 9000, 128, 32, dict(two_sided=False, causal=True, offset=8998)),
])
def test_errors_beside_a_plain_chain(B, H, Hk, N, M, D, buckets, options, kind):
    (q, k, v, dout), _ = problem(B, H, Hk, N, M, D, kind)
    table = some_table(H, buckets) if buckets else None
    out, lse = pkg.sdtw_attention_forward(q, k, v, table, **options)
    got = dict(zip(("out", "lse", "dq", "dk", "dv", "dtable"), (out, lse, *pkg.sdtw_attention_backward(q, k, v, out, lse, dout, table, **options))))
    plain, exact = chain(q, k, v, dout, table, torch.float32, **options), chain(q, k, v, dout, table, torch.float64, **options)
    for name, x in exact.items():
        y = got[name]
        own, theirs = (float((a.to(y.dtype).double() - x).norm() / x.norm()) for a in (y, plain[name]))
        step = 2 * HALF_ULP["f32" if y.dtype == torch.float32 else kind]
        assert own <= max((4 if y.dtype == torch.float32 else 2) * theirs, step), (name, own, theirs)
