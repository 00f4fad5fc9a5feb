"""The operators on rows of logits at the sizes where they go other ways: rows that a workgroup keeps, inputs larger than the caches, rows that fill a part of a
workgroup, lists longer than the entries that threads keep, rows off the grid of vectors.  References in 64 bits, for whole batches on the GPU as well.
"""
import math

import pytest

torch = pytest.importorskip("torch")

from .test_gpu_operators import HALF_ULP, SMALLEST, TYPES, U, _check_distill, _check_logprobs, _check_logprobs_grad, _check_route, _logits, _ops, _sum_tol, _teacher

pytestmark = pytest.mark.gpu


def _rows(batch, n, dtype, seed, lead=0, apart=0):
    """Rows made on the GPU that start `lead` elements into rooms of n + lead + apart."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    room = torch.randn((batch, n + lead + apart), generator=g, device="cuda") * 3.0
    room[:, lead::max(n // 3, 1)] += 9.0
    return room.to(dtype)[:, lead:lead + n]


def _within(got, want, bound, what):
    got = got.double()
    bad = ~((got == want) | ((got - want).abs() <= bound))
    assert not bad.any(), "%s: %d of %d out of bounds, first at %s" % (what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist())


def _log_softmax(x, temperature):
    return torch.log_softmax(x.double() / temperature, 1)


def _check_step(student, k, tail, temperature, value_dtype=torch.float32, teacher_seed=3):
    """Forward, gradient and step over a whole batch; lists without repetitions, some cut short, some empty."""
    ops = _ops()
    batch, n = student.shape
    g = torch.Generator(device="cuda").manual_seed(teacher_seed)
    t = student.float() * 1.1 + torch.randn((batch, n), generator=g, device="cuda")
    values, indices = torch.topk(t, k, dim=1)
    values = values.to(value_dtype)
    length = torch.randint(0, k + 1, (batch,), generator=g, device="cuda")
    length[::2] = k
    given = torch.arange(k, device="cuda") < length[:, None]
    indices = torch.where(given, indices, -1)
    z = torch.where(given, values.double() / temperature, -math.inf)
    norm = torch.logsumexp(z, 1)
    lse = None
    if tail:
        lse = torch.where(norm == -math.inf, 0.0, norm + torch.rand((batch,), generator=g, device="cuda")).float()
    logq = z - (lse.double() if tail else torch.where(norm == -math.inf, 0.0, norm))[:, None]
    q = logq.exp()
    logp = _log_softmax(student, temperature)
    p = logp.exp()
    lp = logp.gather(1, indices.clamp(min=0))
    loss = torch.where(q == 0, 0.0, q * (logq - lp)).sum(1)
    size = torch.where(q == 0, 0.0, q * (1 + logq.abs() + lp.abs())).sum(1)
    dense = torch.zeros_like(p).scatter_add_(1, indices.clamp(min=0), q)
    grad = p * q.sum(1, keepdim=True) - dense
    grad_size = p * q.sum(1, keepdim=True) + dense
    if tail:
        # (padding points at column 0 here, which may be listed as well: what is listed is counted)
        listed = torch.zeros_like(p).scatter_add_(1, indices.clamp(min=0), given.double()) > 0
        rest = (1 - q.sum(1)).clamp(min=0)
        other = torch.logsumexp(logp.masked_fill(listed, -math.inf), 1)
        loss = loss + torch.where(rest > 0, rest * (rest.log() - other), 0.0)
        size = size + torch.where(rest > 0, (rest + 1) * (1 + rest.log().abs() + other.abs()), 0.0)
        # (a row that is listed whole has no rest to share: the loss is infinite, and there is nothing to push down)
        share = (logp.masked_fill(listed, -math.inf) - torch.where(other == -math.inf, 0.0, other)[:, None]).exp()
        grad = grad + rest[:, None] * (p - share)
        grad_size = grad_size + p + share
    w = torch.rand((batch,), generator=g, device="cuda") + 0.5
    w[batch // 3] = 0.0
    grad, grad_size = w[:, None] * grad / temperature, w[:, None] * grad_size / temperature
    tol = _sum_tol(n) + U * (k / 256 + 64)
    bound = 8 * tol * grad_size + HALF_ULP[student.dtype] * 1.01 * grad.abs() + 2 * SMALLEST[student.dtype]
    got, stats = ops.distill(student, values, indices, lse, temperature)
    _within(got, loss, tol * (1 + size), "loss")
    _within(ops.distill_backward(student, values, indices, stats, w, lse, temperature), grad, bound, "gradient")
    out = torch.full((batch, n + 5), 7.0, dtype=student.dtype, device="cuda")[:, 3:3 + n] if student.stride(0) != n else None
    got, dx = ops.distill_step(student, values, indices, w, lse, temperature, out=out)
    _within(got, loss, tol * (1 + size), "loss of the step")
    _within(dx, grad, bound, "gradient of the step")
    if out is not None:
        assert (out._base[:, :3] == 7).all() and (out._base[:, 3 + n:] == 7).all()


# (vectors of 16 bytes in a row: up to 1024, 2048, 4096, 8192, 16384, 20480, and a row too long to be kept)
@pytest.mark.parametrize("tail", [False, True], ids=["list", "rest"])
@pytest.mark.parametrize("batch,vectors,dtype,odd", [
    (300, 1000, torch.bfloat16, 0), (300, 1500, torch.float32, 0), (140, 3999, torch.float16, 3), (600, 4096, torch.bfloat16, 0), (530, 8000, torch.bfloat16, 0),
    (140, 8191, torch.float32, 1), (130, 16384, torch.bfloat16, 0), (400, 16000, torch.float16, 0), (129, 16383, torch.bfloat16, 5), (270, 20480, torch.float32, 0),
    (128, 20479, torch.float16, 7), (130, 21000, torch.float32, 0)])
def test_distill_rows_that_a_workgroup_keeps(batch, vectors, dtype, odd, tail):
    n = vectors * (4 if dtype is torch.float32 else 8)
    _check_step(_rows(batch, n - odd, dtype, batch + n, lead=odd, apart=odd), 33, tail, 1.3)


@pytest.mark.parametrize("tail", [False, True], ids=["list", "rest"])
@pytest.mark.parametrize("batch,vectors,dtype,odd", [
    (256, 16384, torch.bfloat16, 0), (505, 10000, torch.float16, 0), (250, 16383, torch.bfloat16, 5), (480, 20480, torch.float32, 0), (236, 20479, torch.float16, 7),
    (768, 8200, torch.float32, 0), (257, 16384, torch.bfloat16, 0)])
def test_distill_rows_that_fill_the_compute_units(batch, vectors, dtype, odd, tail):
    n = vectors * (4 if dtype is torch.float32 else 8)
    _check_step(_rows(batch, n - odd, dtype, batch + n, lead=odd, apart=odd), 70, tail, 0.8)


@pytest.mark.parametrize("tail", [False, True], ids=["list", "rest"])
@pytest.mark.parametrize("batch,n,k", [(260, 9000, 1025), (130, 70000, 2500), (3, 30000, 5000), (2, 200000, 2049), (500, 2600, 2600)])
def test_distill_lists_longer_than_the_entries_that_threads_keep(batch, n, k, tail):
    _check_step(_rows(batch, n, torch.bfloat16, k), k, tail, 1.0, torch.float16)
    if batch * n < 200000:
        x = _logits(batch, n, torch.float32, k)
        values, indices, lse = _teacher(x, k, 5, 1.0, torch.float32, tail)
        if tail:
            lse += 1.0
        indices[:, k // 2:k // 2 + 200] = indices[:, :200]              # listed twice
        _check_distill(x, values, indices, lse, 1.0)


@pytest.mark.parametrize("batch,n,dtype", [(1100, 50001, torch.bfloat16), (520, 100003, torch.float16), (260, 120000, torch.float32)])
def test_operators_on_inputs_larger_than_the_caches(batch, n, dtype):
    ops = _ops()
    x = _rows(batch, n, dtype, n)
    assert batch * n * x.element_size() > 96 << 20
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens = torch.randint(0, n, (batch, 1), generator=g, device="cuda")
    r = ops.logprobs(x, tokens, k=3, entropy=True)
    logp = _log_softmax(x, 1.0)
    tol = _sum_tol(n)
    want = logp.gather(1, tokens)
    _within(r.logprobs, want, tol + 8 * U * want.abs(), "logprobs")
    entropy = -(logp.exp() * logp).sum(1)
    _within(r.entropy, entropy, tol * (1 + math.log(n)) + 8 * U * entropy.abs(), "entropy")
    top, at = torch.topk(x.float(), 3, dim=1)
    assert torch.equal(x.float().gather(1, r.top_indices), top)
    _within(r.top_logprobs, logp.gather(1, at), tol + 8 * U * logp.gather(1, at).abs(), "top_logprobs")
    weight = torch.randn((batch, 1), generator=g, device="cuda")
    got = ops.logprobs_backward(x, tokens, r.row_stats, weight)
    p = logp.exp_()
    want = torch.zeros_like(p).scatter_(1, tokens, weight.double()) - p * weight
    listed = torch.zeros_like(p).scatter_(1, tokens, 1.0)
    _within(got, want, tol * weight.abs() * torch.maximum(p, listed) + (HALF_ULP[dtype] * 1.01 + 16 * U) * want.abs() + 2 * SMALLEST[dtype], "gradient")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("batch", [1, 6, 300, 700])
def test_logprobs_of_rows_that_fill_a_part_of_a_workgroup(batch, dtype):
    for i, (n, k) in enumerate([(63, 63), (256, 1), (511, 40), (513, 2), (1212, 1), (1500, 64), (2047, 7), (2049, 64), (2900, 3)]):
        x = _logits(batch, n + 3, dtype, n + batch)[:, i % 4:]
        tokens = torch.randint(0, x.shape[1], (batch, 1), generator=torch.Generator().manual_seed(i))
        x[0] = x[0].abs().neg() if i % 2 else 0.0                        # a row of equals
        r, logp = _check_logprobs(x, tokens, k, 0.7)
        if i % 3 == 0:
            _check_logprobs_grad(x, tokens, r, logp, 0.7, i)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("batch,n", [(130, 9001), (300, 20003), (600, 6001), (135, 40000), (129, 60001)])
def test_logprobs_of_batches_by_size(batch, n, dtype):
    x = _logits(batch, n, dtype, n)
    x[1, 5:] = -math.inf
    x[2] = torch.sort(x[2].float())[0].to(dtype)                         # every vector has a new largest
    tokens = torch.randint(0, n, (batch, 2), generator=torch.Generator().manual_seed(1))
    _check_logprobs(x, tokens, 5, 1.0, entropy=True)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tokens,experts,k", [(70, 15, 3), (70, 63, 6), (4200, 99, 4), (5000, 198, 5), (9, 301, 8), (66, 257, 40), (5, 999, 16)])
def test_route_of_rows_off_the_grid_of_vectors(tokens, experts, k, dtype):
    g = torch.Generator().manual_seed(experts)
    room = (torch.randn((tokens, experts + 2), generator=g) * 1.5).to(dtype).cuda()
    bias = (torch.randn((experts + 1,), generator=g) * 0.1).cuda()[1:]
    for x in (room[:, 1:-1], room[:, 2:], room[:, 1:-1].contiguous()):
        _check_route(x, k, "sigmoid", bias, groups=3 if experts % 3 == 0 else 1, topk_groups=2 if experts % 3 == 0 else 1, renormalize=True, scale=2.0)
        _check_route(x, k, "softmax", renormalize=False)
    w, at = _ops().route(x, k)
    out = torch.full((tokens, experts + 3), 7.0, dtype=dtype, device="cuda")
    into = out[:, 1:1 + experts]
    _ops().route_backward(x, at, w, out=into)
    assert torch.equal(into, _ops().route_backward(x, at, w)) and (out[:, 0] == 7).all() and (out[:, 1 + experts:] == 7).all()


@pytest.mark.parametrize("tail", [False, True], ids=["list", "rest"])
@pytest.mark.parametrize("batch,n,k", [(2, 150001, 900), (200, 3001, 700), (700, 2003, 300), (260, 9000, 1500)])
def test_distill_columns_listed_more_than_once_give_the_same_bits_every_time(batch, n, k, tail):
    ops = _ops()
    x = _rows(batch, n, torch.float32, n)
    g = torch.Generator(device="cuda").manual_seed(k)
    indices = torch.randint(0, n, (batch, k), generator=g, device="cuda")
    indices[:, k // 3:2 * (k // 3)] = indices[:, :k // 3].flip(1)
    values = x.gather(1, indices) + torch.randn((batch, k), generator=g, device="cuda")
    lse = torch.logsumexp(values.double(), 1).float() + 0.5 if tail else None
    w = torch.rand((batch,), generator=g, device="cuda")

    def all_of_it():
        loss, stats = ops.distill(x, values, indices, lse)
        return [loss, stats, ops.distill_backward(x, values, indices, stats, w, lse), *ops.distill_step(x, values, indices, w, lse)]

    first = [t.clone() for t in all_of_it()]
    for _ in range(4):
        assert all(torch.equal(p, q) for p, q in zip(first, all_of_it()))
    rows = slice(0, 4)
    _check_distill(x[rows], values[rows], indices[rows], None if lse is None else lse[rows], 1.0)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tokens,experts,groups,topk_groups,k", [
    (40, 400, 8, 3, 10), (33, 512, 32, 9, 4), (5000, 384, 12, 5, 6), (3, 257, 1, 1, 16), (50, 272, 17, 4, 3), (20, 160, 8, 3, 6), (4500, 240, 8, 4, 12), (6, 1024, 8, 4, 13),
    (10, 960, 64, 20, 8), (7, 512, 8, 8, 33)])
def test_route_groups_of_whole_lanes_and_others(tokens, experts, groups, topk_groups, k, dtype):
    g = torch.Generator().manual_seed(experts + k)
    x = (torch.randn((tokens, experts), generator=g) * 1.5).to(dtype).cuda()
    bias = (torch.randn((experts,), generator=g) * 0.1).cuda()
    kw = dict(groups=groups, topk_groups=topk_groups, scale=1.5)
    _check_route(x, k, "softmax", **kw)
    _check_route(x, k, "sigmoid", bias, group_score="top2" if experts // groups > 1 else "max", **kw)


def test_route_scores_at_the_ends_of_the_range():
    ops = _ops()
    x = torch.full((6, 200), -math.inf, device="cuda")
    x[0, 3], x[0, 9] = 200.0, -200.0                   # sigmoids of 1 and of less than any number
    x[1, :50] = -87.5                                  # ... that are no ordinary numbers
    x[2, 7] = math.inf
    x[3] = 0.0
    x[3, 5] = -88.0
    x[4, :4] = torch.tensor([1e30, -1e30, 1e30, 0.0], device="cuda")
    w, at = ops.route(x, 4, score="sigmoid", renormalize=False)
    want = torch.sigmoid(x).gather(1, at)
    assert torch.allclose(w, want, rtol=2e-6, atol=1e-44)
    assert at[0, :2].tolist() == [3, 9] and at[1].tolist() == [0, 1, 2, 3] and at[5].tolist() == [0, 1, 2, 3] and not w[5].any()
    w, at = ops.route(x, 4, score="softmax", renormalize=False)
    assert w[2].isnan().any() and torch.allclose(w[[0, 1, 3, 4]], torch.softmax(x.double(), 1).gather(1, at)[[0, 1, 3, 4]].float(), rtol=2e-6, atol=1e-44)
    assert not w[5].any()


def test_route_counted_in_a_graph():
    ops = _ops()
    x = torch.randn((8200, 256), device="cuda").bfloat16()
    bias = torch.randn((256,), device="cuda") * 0.1
    counts = torch.zeros(256, dtype=torch.int64, device="cuda")
    run = lambda c: ops.route(x, 8, score="sigmoid", bias=bias, groups=8, topk_groups=4, group_score="top2", counts=c)  # noqa: E731
    eager = torch.zeros_like(counts)
    w, at = run(eager)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run(counts)
    for i in range(1, 4):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], w) and torch.equal(held[1], at) and torch.equal(counts, i * eager)
        assert torch.equal(run(None)[1], at)
