"""The operators that a model trained beside Soft-DTW calls, as cases that can be timed.

``op`` of a case:
  distill_forward  a loss per row: the student's logits against the top logits that a teacher left behind
  distill_grad     the same loss, and its gradient in a second call, as an autograd function makes them
  distill_step     loss and gradient in one call, where the weight of every row is known beforehand
  bias_forward     a learned relative position bias added to planes of scores or costs
  bias_backward    the gradient of that bias's table, from the gradient of the planes

Where ``own`` is false everything is computed in the plain form: elementary operations in 32 bits, rounded at the end.
"""
import functools
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def _distill(op, T, V, K, type, tail, temperature=1.0, **more):
    c = {"op": op, "T": T, "V": V, "K": K, "type": type, "tail": tail, "temperature": temperature,
         "mapped": False,   # the student's rows name the teacher's rows they go with; some go with none
         "ragged": False,   # fewer than K logits in some of the teacher's rows, none in a few
         "masked": 0,       # columns at the end of the vocabulary that are padding (-inf)
         "stride": V}       # elements from one row of logits to the next
    c.update(more)
    return c


def _bias(op, B, H, N, M, type, buckets=32, max_distance=128, two_sided=True, **more):
    c = {"op": op, "B": B, "H": H, "N": N, "M": M, "type": type, "buckets": buckets, "max_distance": max_distance,
         "two_sided": two_sided,
         "cached": False,   # every sequence has a past of its own length: the rows' positions start behind it
         "ragged": False,   # every sequence has its own numbers of rows and columns; what lies beyond holds NaN
         "scaled": False}   # a weight per sequence that multiplies the planes' gradient
    c.update(more)
    return c


def listed():
    return [
        # one answer scored against what the teacher would have said: latency
        dict(_distill("distill_forward", 1, 32768, 20, "bf16", False), name="distill_forward_row"),
        # a small batch of short sequences over a small vocabulary (4 sequences of 64, speech units)
        dict(_distill("distill_grad", 256, 1000, 10, "f32", False, 2.0), name="distill_grad_units"),
        # the ordinary training step: 4096 tokens, 16-bit logits
        dict(_distill("distill_step", 4096, 32768, 64, "bf16", False), name="distill_step_4k"),
        # an odd vocabulary with padding, rows aligned to another sequence's, teacher rows of several lengths
        dict(_distill("distill_step", 1037, 50021, 50, "f16", True, 1.5, mapped=True, ragged=True, masked=27, stride=50048),
             name="distill_step_aligned"),
        # logits kept in 32 bits, odd and long rows, forward and backward as separate calls
        dict(_distill("distill_grad", 1024, 100003, 100, "f32", True), name="distill_grad_f32_wide"),
        # a long evaluation batch over a large vocabulary
        dict(_distill("distill_forward", 8192, 131072, 128, "bf16", True), name="distill_forward_eval"),
        # one new token per sequence against a cache, every sequence with a past of its own
        dict(_bias("bias_forward", 32, 16, 1, 4097, "bf16", two_sided=False, cached=True), name="bias_forward_token"),
        # a learned prior on the cost planes of a batch of alignments
        dict(_bias("bias_forward", 32, 1, 1024, 1024, "f32"), name="bias_forward_costs"),
        # attention scores of a padded batch, odd lengths
        dict(_bias("bias_forward", 8, 16, 1100, 937, "f16", ragged=True), name="bias_forward_heads"),
        # the table's gradient for a handful of short pairs: latency
        dict(_bias("bias_backward", 4, 1, 64, 64, "f32", scaled=True), name="bias_backward_tiny"),
        # the same for attention scores in 16 bits
        dict(_bias("bias_backward", 4, 16, 2048, 2048, "bf16", two_sided=False), name="bias_backward_heads"),
        # the largest: alignment matrices of long sequences, one weight per pair
        dict(_bias("bias_backward", 32, 1, 8192, 8192, "f32", buckets=64, max_distance=1024, scaled=True),
             name="bias_backward_long"),
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n + 1 if n == 3 * 1024 else n


def draw(rng):
    op = rng.choice(["distill_forward", "distill_grad", "distill_step", "bias_forward", "bias_backward"])
    type = rng.choice(sorted(TYPES))
    if op.startswith("distill"):
        V = _log_int(rng, 500, 131072)
        T = max(1, min(_log_int(rng, 1, 8192), (1 << 28) // V))
        masked = rng.choice([0, 0, rng.randint(1, 100)])
        return _distill(op, T, V, _log_int(rng, 1, 128), type, rng.random() < 0.5, rng.choice([1.0, 1.0, 0.7, 2.0]),
                        mapped=rng.random() < 0.3, ragged=rng.random() < 0.3, masked=masked,
                        stride=V if rng.random() < 0.6 else (V + 63) // 64 * 64)
    H = rng.choice([1, 1, 4, 8, 12, 16, 32])
    buckets, max_distance = rng.choice([(32, 128), (32, 128), (64, 1024), (16, 50), (128, 4096)])
    two_sided = rng.random() < 0.6
    if op == "bias_forward" and rng.random() < 0.3:
        B, N, M, cached = _log_int(rng, 1, 64), rng.choice([1, 1, 1, 4]), _log_int(rng, 16, 16384), True
    else:
        N = _log_int(rng, 16, 4096)
        M = max(1, int(N * rng.uniform(0.6, 1.5)))
        M += M == 3 * 1024
        B, cached = max(1, min(_log_int(rng, 1, 64), (1 << 28) // (H * N * M))), rng.random() < 0.2
    return _bias(op, B, H, N, M, type, buckets, max_distance, two_sided, cached=cached, ragged=rng.random() < 0.3,
                 scaled=op == "bias_backward" and rng.random() < 0.5)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    return (_prepare_distill if case["op"].startswith("distill") else _prepare_bias)(s, case, gen)


def _prepare_distill(s, case, gen):
    T, V, K, dtype = case["T"], case["V"], case["K"], TYPES[case["type"]]
    real = V - case["masked"]
    rows = max(1, 3 * T // 4) if case["mapped"] else T
    z = torch.empty((T, case["stride"]), dtype=dtype, device="cuda")
    for a in range(0, T, 1024):  # in pieces: a long batch in 32 bits would be several times its own size
        z[a:a + 1024] = 2.0 * torch.randn((min(1024, T - a), case["stride"]), generator=gen, device="cuda")
    # K different tokens for each of the teacher's rows, the most likely first
    step = torch.randint(1, max(2, real // K), (rows, 1), generator=gen, device="cuda")
    first = torch.randint(0, real, (rows, 1), generator=gen, device="cuda")
    ids = (first + step * torch.arange(K, device="cuda")) % real
    t = torch.randn((rows, K), generator=gen, device="cuda") + 12.0 - 1.5 * torch.log1p(torch.arange(K, device="cuda"))
    at = None
    if case["mapped"]:  # an alignment: rising, several rows on one, some on none
        at = (torch.arange(T, device="cuda") * rows // T).to(torch.int32)
        at[torch.rand(T, generator=gen, device="cuda") < 0.1] = -1
    # a student that has learnt some of it
    own_rows = torch.arange(T, device="cuda") if at is None else at.long().clamp(min=0)
    lift = 0.5 * t[own_rows] + torch.randn((T, K), generator=gen, device="cuda")
    z.scatter_(1, ids[own_rows], lift.to(dtype))
    z[:, real:V] = -math.inf
    s["logits"] = z[:, :V]
    if case["ragged"]:
        kept = torch.randint(0, K + 1, (rows, 1), generator=gen, device="cuda")
        kept[torch.rand((rows, 1), generator=gen, device="cuda") < 0.5] = K
        ids = torch.where(torch.arange(K, device="cuda") < kept, ids, -1)
    s["teacher_logits"], s["teacher_ids"], s["teacher_row"] = t.to(dtype), ids, at
    s["teacher_lse"] = None
    if case["tail"]:  # over the teacher's whole vocabulary, at this temperature: a few per cent lie outside its top
        lse = torch.logsumexp(s["teacher_logits"].double() / case["temperature"], 1)
        s["teacher_lse"] = (lse + 0.02 + 0.1 * torch.rand(rows, generator=gen, device="cuda")).float()
    # the weight of each row in the mean; with the loss scaled up where float16 gradients would vanish otherwise
    s["weight"] = (torch.rand(T, generator=gen, device="cuda") + 0.5) * ((4096.0 if case["type"] == "f16" else 1.0) / T)
    return s


def _prepare_bias(s, case, gen):
    B, H, N, M, dtype = case["B"], case["H"], case["N"], case["M"], TYPES[case["type"]]
    plane = torch.empty((B, H, N, M), dtype=dtype, device="cuda")
    for b in range(B):
        plane[b] = torch.randn((H, N, M), generator=gen, device="cuda")
    s["row_len"] = s["col_len"] = None
    if case["ragged"]:
        for name, full in (("row_len", N), ("col_len", M)):
            s[name] = torch.randint(full // 4, full + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
        for b in range(B):
            plane[b, :, int(s["row_len"][b]):] = math.nan
            plane[b, :, :, int(s["col_len"][b]):] = math.nan
    s["offset"] = 0
    if case["cached"]:
        s["offset"] = torch.randint(0, max(1, M - N) + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    s["plane"] = plane
    if case["op"] == "bias_forward":
        s["table"] = 0.5 * torch.randn((case["buckets"], H), generator=gen, device="cuda").t()
    s["scale"] = (torch.rand(B, generator=gen, device="cuda") + 0.5) / B if case["scaled"] else None
    return s


# ------------------------------------------------------------------ the calls

def run(s):
    case = s["case"]
    if not own:
        return {"distill_forward": _plain_distill, "distill_grad": _plain_distill, "distill_step": _plain_distill,
                "bias_forward": _plain_bias_forward, "bias_backward": _plain_bias_backward}[case["op"]](s)
    from paper_2602_17206_amd import binding as sdtw

    if case["op"].startswith("distill"):
        teacher = (s["teacher_logits"], s["teacher_ids"])
        more = {"temperature": case["temperature"], "teacher_lse": s["teacher_lse"], "teacher_row": s["teacher_row"]}
        if case["op"] == "distill_step":
            loss, dlogits = sdtw.sdtw_distill_step(s["logits"], *teacher, grad_loss=s["weight"], **more)
            return {"loss": loss, "dlogits": dlogits}
        loss, stats = sdtw.sdtw_distill_forward(s["logits"], *teacher, **more)
        if case["op"] == "distill_forward":
            return {"loss": loss}
        return {"loss": loss, "dlogits": sdtw.sdtw_distill_backward(s["logits"], *teacher, stats, grad_loss=s["weight"], **more)}
    more = {"max_distance": case["max_distance"], "two_sided": case["two_sided"], "offset": s["offset"],
            "row_len": s["row_len"], "col_len": s["col_len"]}
    if case["op"] == "bias_forward":
        return {"out": sdtw.sdtw_position_bias_forward(s["table"], s["plane"], **more)}
    return {"dtable": sdtw.sdtw_position_bias_backward(s["plane"], case["buckets"], scale=s["scale"], **more)}


# ------------------------------------------------------------------ the plain forms

def _plain_distill(s):
    case = s["case"]
    tau = case["temperature"]
    z = s["logits"].float() / tau
    t, ids, teacher_lse, at = s["teacher_logits"].float() / tau, s["teacher_ids"], s["teacher_lse"], s["teacher_row"]
    if at is not None:
        rows = at.long().clamp(min=0)
        t, ids = t[rows], torch.where((at >= 0)[:, None], ids[rows], -1)
        teacher_lse = None if teacher_lse is None else teacher_lse[rows]
    used = ids >= 0
    col = ids.clamp(min=0)
    t = torch.where(used, t, -math.inf)
    if case["tail"]:
        q = torch.exp(t - teacher_lse[:, None])
    else:
        w = torch.exp(t - t.amax(1, keepdim=True).clamp(min=-1e30))
        q = w / w.sum(1, keepdim=True).clamp(min=1e-30)
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - m)
    total = e.sum(1, keepdim=True)
    log_total = m + torch.log(total)
    log_p = torch.gather(z, 1, col) - log_total
    zero = torch.zeros((), device=z.device)
    loss = torch.where(q > 0, q * (torch.log(q) - log_p), zero).sum(1)
    if case["tail"]:
        rest = (1.0 - q.sum(1)).clamp(min=0.0)
        top = torch.zeros((z.shape[0], z.shape[1] + 1), dtype=torch.bool, device=z.device)
        top = top.scatter_(1, torch.where(used, ids, z.shape[1]), True)[:, :-1]
        outside = torch.where(top, zero, e).sum(1)
        log_rest = torch.log(outside) - torch.log(total[:, 0])
        loss = loss + torch.where(rest > 0, rest * (torch.log(rest) - log_rest), zero)
    if case["op"] == "distill_forward":
        return {"loss": loss}
    mass = q.sum(1, keepdim=True)
    p = e / total
    if case["tail"]:
        mass = mass + rest[:, None]
        d = torch.where(top, mass * p, (mass * outside[:, None] / total - rest[:, None]) * (e / outside[:, None]))
    else:
        d = mass * p
    d = d.scatter_add_(1, col, torch.where(used, -q, zero))
    return {"loss": loss, "dlogits": (d * (s["weight"] / tau)[:, None]).to(s["logits"].dtype)}


def _diagonal_buckets(case, device, offset):
    """The bucket on each of the N + M - 1 diagonals j - i, lowest first, for one offset or one of each sequence."""
    N, M, n = case["N"], case["M"], case["buckets"] // (2 if case["two_sided"] else 1)
    e = n // 2  # one distance for each of the first half of the buckets, equal steps of the logarithm after them
    rel = torch.arange(-(N - 1), M, device=device)[None] - (offset if isinstance(offset, int) else offset[:, None])
    d = rel.abs() if case["two_sided"] else (-rel).clamp(min=0)
    # the logarithm in 64 bits; what is added keeps the distances that begin a bucket exactly on its side of the floor
    steps = torch.log(d.clamp(min=e).double() / e) * ((n - e) / math.log(case["max_distance"] / e)) + 1e-9
    bucket = torch.where(d < e, d, (e + steps.floor().long()).clamp(max=n - 1))
    return bucket + n * (rel > 0) if case["two_sided"] else bucket


def _inside(s):
    case, dev = s["case"], s["plane"].device
    i, j = torch.arange(case["N"], device=dev), torch.arange(case["M"], device=dev)
    return ((i[:, None] < s["row_len"][:, None, None]) & (j < s["col_len"][:, None, None]))[:, None]


def _plain_bias_forward(s):
    case, plane = s["case"], s["plane"]
    N, M = case["N"], case["M"]
    diagonal = s["table"][:, _diagonal_buckets(case, plane.device, s["offset"])].transpose(0, 1)  # [1 or B, H, N+M-1]
    at = torch.arange(M, device=plane.device) - torch.arange(N, device=plane.device)[:, None] + (N - 1)
    x = plane.float()
    y = x + diagonal[:, :, at]
    if s["row_len"] is not None:
        y = torch.where(_inside(s), y, x)
    return {"out": y.to(plane.dtype)}


def _plain_bias_backward(s):
    case = s["case"]
    B, H, N, M = case["B"], case["H"], case["N"], case["M"]
    g = s["plane"].float()
    if s["row_len"] is not None:
        g = torch.where(_inside(s), g, torch.zeros((), device=g.device))
    if s["scale"] is not None:
        g = g * s["scale"][:, None, None, None]
    bucket = _diagonal_buckets(case, g.device, s["offset"])  # [1 or B, N+M-1]
    if bucket.shape[0] == 1:
        g = g.sum(0, keepdim=True)
    # the last row first and every row one place further right than the one before: a diagonal becomes a column
    g = torch.nn.functional.pad(g.flip(2), (0, N)).flatten(2)[:, :, :N * (N + M - 1)].reshape(g.shape[0], H, N, N + M - 1)
    hot = (bucket[..., None] == torch.arange(case["buckets"], device=g.device)).float()  # [1 or B, N+M-1, buckets]
    return {"dtable": torch.matmul(g.sum(2), hot).sum(0)}


# ------------------------------------------------------------------ in 64 bits, from the definitions

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("distill"):
        return _exact_distill(case, s)
    first = _exact_buckets(case)
    B, H, N, M = case["B"], case["H"], case["N"], case["M"]
    lowest = -(N - 1) - M  # an offset is at most M - N + 1 or 0
    lookup = torch.tensor([first(r) for r in range(lowest, M + N + 1)], device="cuda")
    apart = torch.arange(M, device="cuda") - torch.arange(N, device="cuda")[:, None]
    forward = case["op"] == "bias_forward"
    out = torch.empty((B, H, N, M), dtype=torch.float64, device="cuda") if forward else None
    dtable = torch.zeros((H, case["buckets"]), dtype=torch.float64, device="cuda")
    total = torch.zeros((H, N, M), dtype=torch.float64, device="cuda")
    for b in range(B):
        r = int(s["row_len"][b]) if case["ragged"] else N
        c = int(s["col_len"][b]) if case["ragged"] else M
        offset = int(s["offset"][b]) if case["cached"] else 0
        x = s["plane"][b].double()
        if forward:
            x[:, :r, :c] += s["table"].double()[:, lookup[apart[:r, :c] - offset - lowest]]
            out[b] = x
            continue
        weight = float(s["scale"][b]) if case["scaled"] else 1.0
        if case["cached"]:
            bucket = lookup[apart[:r, :c] - offset - lowest]
            dtable += weight * torch.stack([(x[:, :r, :c] * (bucket == k)).sum((1, 2)) for k in range(case["buckets"])], 1)
        else:
            total[:, :r, :c] += weight * x[:, :r, :c]
    if forward:
        return {"out": out}
    if not case["cached"]:
        bucket = lookup[apart - lowest]
        dtable = torch.stack([(total * (bucket == k)).sum((1, 2)) for k in range(case["buckets"])], 1)
    return {"dtable": dtable}


def _exact_buckets(case):
    n = case["buckets"] // (2 if case["two_sided"] else 1)
    e, D = n // 2, case["max_distance"]

    @functools.lru_cache(None)
    def side_to(d):
        if d < e:
            return d
        k = 0  # in whole numbers: d^(n-e) against e^(n-e-k) D^k
        while k + 1 < n - e and d ** (n - e) >= e ** (n - e - k - 1) * D ** (k + 1):
            k += 1
        return e + k

    def side(d):
        return side_to(min(d, D))  # from D on everything is in the last bucket

    if case["two_sided"]:
        return lambda r: side(abs(r)) + (n if r > 0 else 0)
    return lambda r: side(max(0, -r))


def _exact_distill(case, s):
    T, V, tau = case["T"], case["V"], case["temperature"]
    losses, grads = [], []
    rows_at_once = max(1, (1 << 27) // V)
    for a in range(0, T, rows_at_once):
        z = s["logits"][a:a + rows_at_once].double().requires_grad_()
        n = z.shape[0]
        at = torch.arange(a, a + n, device="cuda") if s["teacher_row"] is None else s["teacher_row"][a:a + n].long()
        ids = s["teacher_ids"][at.clamp(min=0)].clone()
        ids[at < 0] = -1
        # the teacher's probabilities laid out over the vocabulary, with one more place for unused slots
        slot = torch.where(ids < 0, V, ids)
        t = s["teacher_logits"][at.clamp(min=0)].double() / tau
        t[ids < 0] = -math.inf
        norm = s["teacher_lse"][at.clamp(min=0)].double() if case["tail"] else torch.logsumexp(t, 1)
        prob = torch.exp(t - norm[:, None])
        prob[ids < 0] = 0.0
        q = torch.zeros((n, V + 1), dtype=torch.float64, device="cuda").scatter_(1, slot, prob)[:, :V]
        log_p = z / tau - torch.logsumexp(z / tau, 1, keepdim=True)
        loss = torch.special.xlogy(q, q).sum(1) - torch.where(q > 0, q * log_p, 0.0).sum(1)
        if case["tail"]:
            rest = (1.0 - q.sum(1)).clamp(min=0.0)
            top = torch.zeros((n, V + 1), dtype=torch.bool, device="cuda").scatter_(1, slot, True)[:, :V]
            log_rest = torch.logsumexp(log_p.masked_fill(top, -math.inf), 1)
            loss = loss + torch.special.xlogy(rest, rest) - rest * log_rest
        losses.append(loss.detach())
        if case["op"] != "distill_forward":
            (d,) = torch.autograd.grad((loss * s["weight"][a:a + n].double()).sum(), z)
            grads.append(d)
    found = {"loss": torch.cat(losses)}
    if grads:
        found["dlogits"] = torch.cat(grads)
    return found


def work(case):
    size = TYPES[case["type"]].itemsize
    if case["op"].startswith("distill"):
        T, V, K = float(case["T"]), case["V"], case["K"]
        teacher = T * K * (size + 8) + T * 8
        # a maximum, a difference, a scaling, an exponential and a sum per logit; a scaling and a product more for its gradient
        if case["op"] == "distill_forward":
            return {"bytes": T * V * size + teacher, "flops": 5 * T * V}
        return {"bytes": 2 * T * V * size + teacher, "flops": 7 * T * V}
    cells = float(case["B"]) * case["H"] * case["N"] * case["M"]
    table = 4.0 * case["H"] * case["buckets"]
    inside = cells * (0.625 ** 2 if case["ragged"] else 1.0)  # lengths uniform in [1/4, 1] of the full ones
    if case["op"] == "bias_forward":
        return {"bytes": 2 * cells * size + table, "flops": inside}
    return {"bytes": inside * size + table, "flops": inside}
