"""The operators on rows of logits (log probabilities, distillation, routing) on the GPU, against their definitions in 64 bits.

Tolerances follow from the arithmetic, in units of u = 2^-24: a lane adds up a few hundred terms and lanes are joined pairwise (at most n / 256 + 64 roundings of
positive terms), an exponent's argument of up to 24 is rounded three times and 2^x once, and a gradient is rounded once to the logits' type.
"""
import math

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TYPES = [torch.float32, torch.float16, torch.bfloat16]
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
SMALLEST = {torch.float32: 0.0, torch.float16: 2.0 ** -25, torch.bfloat16: 0.0}
SHAPES = [(1, 1), (3, 2), (2, 7), (5, 64), (3, 257), (4, 1000), (2, 8193), (1, 20000), (300, 1025), (1, 131072), (7, 50257), (3, 262147)]


def _ops():
    from paper_2501_14336_amd import operators
    return operators


def _sum_tol(n):
    return U * (n / 256 + 64 + 72)


def _logits(batch, n, dtype, seed, sigma=3.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((batch, n), generator=g) * sigma
    x[:, torch.randint(0, n, (min(n, 3),), generator=g)] += 9.0
    return x.to(dtype).cuda()


def _near(got, want, atol, rtol, what):
    got, want = got.cpu(), want.double().cpu()
    most = want.to(got.dtype).double()
    got, want = got.double(), torch.where(most.isinf(), most, want)     # (beyond the type's range there is only infinity)
    assert got.shape == want.shape, what
    same = (got == want) | (got.isnan() & want.isnan())
    off = (got - want).abs()
    bound = atol + rtol * want.abs()
    bad = ~same & ~(off <= bound)
    assert not bad.any(), "%s: %d of %d out of bounds, worst %g (bound there %g), first at %s" % (
        what, int(bad.sum()), bad.numel(), float(off[bad].max()), float(bound.expand_as(off)[bad].max()) if torch.is_tensor(bound) else bound, bad.nonzero()[0].tolist())


def _ref_logp(x, temperature):
    """64-bit log probabilities; a row without anything but -inf has p = 0 everywhere."""
    y = x.double().cpu() / temperature
    m = y.amax(1, keepdim=True)
    empty = m == -math.inf
    y = y - torch.where(empty, 0.0, m)
    s = y.exp().sum(1, keepdim=True)
    return torch.where(empty, -math.inf, y - s.log())


def _ref_entropy(logp):
    p = logp.exp()
    return -torch.where(p == 0, 0.0, p * logp).sum(1)


def _ref_logprobs_grad(logp, tokens, g, gh, temperature):
    n = logp.shape[1]
    p = logp.exp()
    ok = (tokens >= 0) & (tokens < n)
    g = torch.where(ok, g.double().cpu(), 0.0)
    dx = -p * g.sum(1, keepdim=True)
    dx.scatter_add_(1, torch.where(ok, tokens, 0), g)
    if gh is not None:
        dx -= gh.double().cpu()[:, None] * torch.where(p == 0, 0.0, p * (logp + _ref_entropy(logp)[:, None]))
    return dx / temperature


def _top(x, k):
    """Positions of the k largest, lowest first among equals (no NaN, no zeros of both signs in these rows)."""
    return torch.sort(x.float().cpu(), dim=1, descending=True, stable=True)[1][:, :k]


def _check_logprobs(x, tokens, k, temperature, entropy=True):
    ops = _ops()
    n = x.shape[1]
    r = ops.logprobs(x, None if tokens is None else tokens.cuda(), k=k, temperature=temperature, entropy=entropy)
    logp = _ref_logp(x, temperature)
    tol = _sum_tol(n)
    if tokens is not None:
        want = torch.where(tokens < 0, 0.0, logp.gather(1, tokens.clamp(0, n - 1)))
        want = torch.where(tokens >= n, math.nan, want)
        _near(r.logprobs, want, tol, 8 * U, "logprobs")
    if entropy:
        _near(r.entropy, _ref_entropy(logp), tol * (1 + math.log(n)), 8 * U, "entropy")
    if k:
        at = _top(x, k)
        assert torch.equal(r.top_indices.cpu(), at)
        _near(r.top_logprobs, logp.gather(1, at), tol, 8 * U, "top_logprobs")
    return r, logp


def _check_logprobs_grad(x, tokens, r, logp, temperature, seed, out=None):
    ops = _ops()
    batch, n = x.shape
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(tokens.shape, generator=gen)
    gh = torch.randn((batch,), generator=gen)
    for with_entropy in (False, True):
        got = ops.logprobs_backward(x, tokens.cuda(), r.row_stats, g.cuda(), r.entropy if with_entropy else None, gh.cuda() if with_entropy else None,
                                    temperature, out=out)
        want = _ref_logprobs_grad(logp, tokens, g, gh if with_entropy else None, temperature)
        scale = (g.abs().sum(1, keepdim=True).double() + (gh.abs()[:, None].double() * (1 + math.log(n)) ** 2 if with_entropy else 0.0)) / temperature
        # (p itself is off by the sum's tolerance; where the terms cancel, what is left is off by theirs)
        p = logp.exp()
        listed = torch.zeros_like(p).scatter_(1, tokens.clamp(0, n - 1), 1.0)
        atol = _sum_tol(n) * scale * torch.maximum(p, listed) + 2 * SMALLEST[x.dtype]
        _near(got, want, atol, HALF_ULP[x.dtype] * 1.01 + 16 * U, "gradient (entropy: %s)" % with_entropy)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("batch,n", SHAPES)
def test_logprobs_and_their_gradient(batch, n, dtype):
    for i, (m, k, temperature) in enumerate([(1, 0, 1.0), (3, 5, 0.7), (0, 64, 2.0), (2, 20, 1.0), (1, 200, 1.0)]):
        x = _logits(batch, n, dtype, 100 * i + n)
        tokens = torch.randint(0, n, (batch, m), generator=torch.Generator().manual_seed(i))
        r, logp = _check_logprobs(x, tokens, min(k, n), temperature)
        if m:
            _check_logprobs_grad(x, tokens, r, logp, temperature, i)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_logprobs_masks_and_rows_that_they_leave_empty(dtype):
    low = torch.finfo(dtype).min
    batch, n = 9, 3001
    x = _logits(batch, n, dtype, 7)
    keep = torch.rand((batch, n), generator=torch.Generator().manual_seed(8)) < 0.3
    keep[:, 17] = True
    keep = keep.cuda()
    for mask in (-math.inf, low):
        y = x.masked_fill(~keep, mask)
        y[2] = mask                                   # nothing is left (the lowest value: all alike)
        y[3] = mask
        y[3, 1234] = 5.0                              # one is left
        y[4, 1:] = mask                               # the first alone, in the row's first vector
        y[5, :-1] = mask                              # the last alone
        y[6] = 0.0                                    # all alike
        tokens = torch.tensor([[17, 0], [17, 5], [3, 4], [1234, 7], [0, n - 1], [n - 1, 0], [1, 2], [17, 17], [-1, 17]])
        for k in (1, 10, 70):
            r, logp = _check_logprobs(y, tokens, k, 0.9)
        _check_logprobs_grad(y, tokens, r, logp, 0.9, 3)
        if mask == -math.inf:
            assert r.entropy[2] == 0 and r.logprobs[2, 0] == -math.inf and r.row_stats[2, 1] == 0


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_logprobs_of_values_that_are_no_numbers(dtype):
    ops = _ops()
    n = 5003
    x = _logits(5, n, dtype, 9)
    x[1, 4000] = math.nan
    x[2, 77] = math.inf
    x[3] = math.nan
    tokens = torch.tensor([[5], [5], [5], [5], [n]]).cuda()
    r = ops.logprobs(x, tokens, k=6, entropy=True)
    assert r.logprobs[1:, 0].isnan().all() and not r.logprobs[0].isnan().any()
    assert r.entropy[1:4].isnan().all() and not r.entropy[[0, 4]].isnan().any()
    assert r.top_logprobs[1:4].isnan().all() and not r.top_logprobs[[0, 4]].isnan().any()
    assert r.top_indices[1, 0] == 4000 and r.top_indices[2, 0] == 77 and r.top_indices[3].tolist() == list(range(6))
    assert torch.equal(r.top_indices[[0, 4]].cpu(), _top(x[[0, 4]], 6))
    grad = ops.logprobs_backward(x, tokens, r.row_stats, torch.ones((5, 1), device="cuda"), r.entropy, torch.ones(5, device="cuda"))
    assert grad[1:4].isnan().any(1).all() and not grad[0].isnan().any()
    # a token that is none has no gradient
    alone = ops.logprobs_backward(x, tokens, r.row_stats, torch.ones((5, 1), device="cuda"))
    assert not alone[4].any()


def _orders(n):
    ramp = torch.linspace(-9.0, 9.0, n)
    return {
        "ascending": ramp, "descending": ramp.flip(0), "equal": torch.full((n,), 1.5),
        "two values": torch.where(torch.arange(n) % 3 == 0, 2.0, 1.0), "blocks": ramp[:: max(1, n // 40)].repeat_interleave(64)[:n] if n >= 64 * 40 else ramp,
        "best in one lane": torch.where(torch.arange(n) % 2048 < 8, 3.0 + torch.rand(n, generator=torch.Generator().manual_seed(1)), torch.zeros(n)),
        "best at the end": torch.cat([torch.zeros(n - n // 50), torch.rand(n // 50, generator=torch.Generator().manual_seed(2))]) + 1.0,
        "saw": (torch.arange(n) % 100).float() / 7.0,
    }


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("n", [5000, 100003])
def test_logprobs_alternatives_of_rows_in_order_and_of_equal_logits(n, dtype):
    rows = _orders(n)
    x = torch.stack([v if v.numel() == n else torch.nn.functional.pad(v, (0, n - v.numel()), value=-3.0) for v in rows.values()]).to(dtype).cuda()
    for batch_of in (x, x[1:2], x.repeat(40, 1)):
        for k in (1, 7, 50, 64):
            r = _ops().logprobs(batch_of, k=k)
            want = _top(batch_of, k)
            got = r.top_indices.cpu()
            for i in range(min(len(rows), batch_of.shape[0])):
                assert torch.equal(got[i], want[i]), (list(rows)[i], k)
            assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
def test_logprobs_of_strided_and_misaligned_rows(dtype):
    base = _logits(6, 4999, dtype, 21)
    for x in (base[:, 3:], base[::2, 1:-2], base[1:3, 5:2222], base[:, :1]):
        assert not x.is_contiguous()
        batch, n = x.shape
        tokens = torch.randint(0, n, (batch, 2), generator=torch.Generator().manual_seed(5))
        r, logp = _check_logprobs(x, tokens, min(5, n), 1.0)
        _check_logprobs_grad(x, tokens, r, logp, 1.0, 2)
        room = torch.full((batch, n + 9), 7.0, dtype=dtype, device="cuda")
        for shift in (0, 1, 3):                        # the gradient starts elsewhere than the logits
            room.fill_(7.0)
            _check_logprobs_grad(x, tokens, r, logp, 1.0, 2, out=room[:, shift:shift + n])
            assert (room[:, :shift] == 7).all() and (room[:, shift + n:] == 7).all()


def test_logprobs_tokens_listed_more_than_once_add_up():
    x = _logits(4, 30011, torch.float32, 31)
    tokens = torch.randint(0, 30011, (4, 300), generator=torch.Generator().manual_seed(6))
    tokens[:, 100:200] = tokens[:, :100]
    tokens[0, 200:] = 5
    tokens[1, 7] = -100
    tokens[2, 9] = 30011
    r, logp = _check_logprobs(x, tokens, 0, 1.0)
    _check_logprobs_grad(x, tokens, r, logp, 1.0, 4)


def test_logprobs_of_rows_beyond_four_gigabytes():
    n, apart = 70001, (1 << 31) + 24
    big = torch.empty((2 * apart,), dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((3, n), (apart // 2 + 1000, 1))
    x.copy_(_logits(3, n, torch.bfloat16, 41))
    tokens = torch.randint(0, n, (3, 1), generator=torch.Generator().manual_seed(7))
    r, logp = _check_logprobs(x, tokens, 4, 1.0)
    _check_logprobs_grad(x, tokens, r, logp, 1.0, 1)


# ---------------------------------------------------------------------------
# distillation
# ---------------------------------------------------------------------------

def _ref_distill(student, values, indices, lse, temperature):
    """64-bit loss, d loss / d student, and the magnitudes of what is added up in them."""
    n = student.shape[1]
    logp = _ref_logp(student, temperature)
    z, at, given = values.double().cpu() / temperature, indices.cpu(), indices.cpu() >= 0
    z = torch.where(given, z, -math.inf)
    if lse is None:
        norm = torch.logsumexp(z, 1, keepdim=True)
        logq = torch.where(norm == -math.inf, -math.inf, z - norm)
    else:
        logq = z - lse.double().cpu()[:, None]
    q = logq.exp()
    lp = logp.gather(1, at.clamp(0, n - 1))
    terms = torch.where(q == 0, 0.0, q * (logq - lp))
    loss, size = terms.sum(1), torch.where(q == 0, 0.0, q * (1 + logq.abs() + lp.abs())).sum(1)
    dense = torch.zeros_like(logp)
    for j in range(q.shape[1]):                       # (an entry at a time: columns may be listed twice)
        dense.scatter_add_(1, at[:, j:j + 1].clamp(min=0), q[:, j:j + 1])
    grad = logp.exp() * q.sum(1, keepdim=True) - dense
    grad_size = logp.exp() * q.sum(1, keepdim=True) + dense
    if lse is not None:
        listed = torch.zeros_like(logp, dtype=torch.bool)
        for j in range(q.shape[1]):
            listed.scatter_(1, at[:, j:j + 1].clamp(min=0), listed.gather(1, at[:, j:j + 1].clamp(min=0)) | given[:, j:j + 1])
        rest = (1 - q.sum(1)).clamp(min=0)
        other = torch.logsumexp(logp.masked_fill(listed, -math.inf), 1)
        loss = loss + torch.where(rest > 0, rest * (rest.log() - other), 0.0)
        # q is off by a few units of its exponent's argument, the rest by as much as all of them
        size = size + torch.where(rest > 0, (rest + 1) * (1 + rest.log().abs() + other.abs()), 0.0)
        y = (student.double().cpu() / temperature).masked_fill(listed, -math.inf)
        m = y.amax(1, keepdim=True)                   # (not from logp: logits far below all others would lose their sum's digits there)
        e = (y - torch.where(m == -math.inf, 0.0, m)).exp()
        share = e / torch.where(m == -math.inf, 1.0, e.sum(1, keepdim=True))
        grad = grad + rest[:, None] * (logp.exp() - share)
        grad_size = grad_size + logp.exp() + share
    return loss, grad / temperature, size, grad_size / temperature


def _teacher(student, k, seed, temperature, value_dtype, tail):
    g = torch.Generator().manual_seed(seed)
    t = student.double().cpu() * 1.1 + torch.randn(student.shape, generator=g).double()
    values, indices = torch.topk(t, k, dim=1)
    values = values.to(value_dtype)
    lse = None
    if tail:
        chosen = torch.logsumexp(values.double() / temperature, 1)
        lse = torch.logaddexp(chosen, torch.logsumexp(t.scatter(1, indices, -math.inf) / temperature, 1) if k < student.shape[1] else chosen - 9.0).float().cuda()
    return values.cuda(), indices.cuda(), lse


def _check_distill(student, values, indices, lse, temperature, seed=0):
    ops = _ops()
    batch, n = student.shape
    k = indices.shape[1]
    want, grad, size, grad_size = _ref_distill(student, values, indices, lse, temperature)
    tol = _sum_tol(n) + U * (k / 256 + 64)
    loss, stats = ops.distill(student, values, indices, lse, temperature)
    _near(loss, want, tol * (1 + size), 0.0, "loss")
    w = torch.rand((batch,), generator=torch.Generator().manual_seed(seed)) + 0.5
    w[batch // 2] = 0.0
    got = ops.distill_backward(student, values, indices, stats, w.cuda(), lse, temperature)
    bound = w[:, None].double() * tol * 8 * grad_size + 2 * SMALLEST[student.dtype]
    wanted = torch.where(w[:, None] == 0, 0.0, w[:, None].double() * grad)
    _near(got, wanted, bound, HALF_ULP[student.dtype] * 1.01, "gradient")
    l2, g2 = ops.distill_step(student, values, indices, w.cuda(), lse, temperature)
    _near(l2, want, tol * (1 + size), 0.0, "loss of the step")
    _near(g2, wanted, bound, HALF_ULP[student.dtype] * 1.01, "gradient of the step")
    return loss, got


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tail", [False, True], ids=["list", "rest"])
@pytest.mark.parametrize("batch,n,k", [(1, 1, 1), (3, 2, 1), (2, 7, 7), (5, 64, 9), (3, 257, 50), (4, 1000, 300), (2, 8193, 1024), (1, 30011, 100), (300, 1025, 5), (2, 131072, 1024),
                                       (7, 50257, 50), (2, 262147, 33), (2, 600001, 20)])
def test_distill_and_its_gradient(batch, n, k, tail, dtype):
    for i, (temperature, value_dtype) in enumerate([(1.0, torch.float32), (2.0, dtype), (0.7, torch.float16)]):
        if i and n > 100000:
            continue
        student = _logits(batch, n, dtype, 10 * i + n)
        values, indices, lse = _teacher(student, k, i, temperature, value_dtype, tail)
        _check_distill(student, values, indices, lse, temperature, i)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tail", [False, True], ids=["list", "rest"])
def test_distill_lists_of_any_length_and_masked_rows(tail, dtype):
    batch, n, k = 8, 3001, 40
    student = _logits(batch, n, dtype, 5)
    values, indices, lse = _teacher(student, k, 6, 1.0, torch.float32, tail)
    indices[1, 20:] = -1
    indices[2] = -1                                    # an empty list
    indices[3, ::2] = -7
    values[4, 10:] = -math.inf                         # a teacher that gives the rest nothing
    values[indices < 0] = math.nan                     # what padding holds is not looked at
    student[5].masked_fill_(torch.ones(n, dtype=torch.bool, device="cuda").index_fill_(0, indices[5], False), -math.inf if not tail else torch.finfo(dtype).min / 4)
    student[6, ::3] = torch.finfo(dtype).min
    student[6, indices[6]] = 2.0
    if tail:
        lse[7] -= 3.0                                  # sums to more than 1: the rest is 0
    loss, grad = _check_distill(student, values, indices, lse, 1.0)
    assert loss.isfinite().all()
    if not tail:
        assert loss[2] == 0 and not grad[2].any()


def test_distill_rows_that_have_no_finite_loss():
    ops = _ops()
    n = 2000
    student = _logits(5, n, torch.bfloat16, 15)
    values, indices, lse = _teacher(student, 10, 3, 1.0, torch.float32, True)
    student[1, indices[1, 0]] = -math.inf              # the student rules out what the teacher holds
    indices[2, 4] = n                                  # no such column
    student[3] = math.nan
    w = torch.ones(5, device="cuda")
    w[3] = 0.0
    for l in (None, lse):
        loss, stats = ops.distill(student, values, indices, l)
        assert loss[0].isfinite() and loss[4].isfinite() and loss[1] == math.inf and loss[2].isnan() and loss[3].isnan()
        grad = ops.distill_backward(student, values, indices, stats, w, l)
        assert grad[[0, 1, 4]].isfinite().all() and not grad[3].any()    # a row of weight 0 gets zeros whatever it holds


@pytest.mark.parametrize("tail", [False, True], ids=["list", "rest"])
def test_distill_columns_listed_twice_and_strided_students(tail):
    base = _logits(6, 5003, torch.float32, 25)
    student = base[::2, 2:]
    values, indices, lse = _teacher(student, 90, 3, 1.0, torch.float32, tail)
    if tail:
        lse += 1.0
    indices[:, 60:] = indices[:, :30]
    indices[0, 3:40] = 11
    _check_distill(student, values, indices, lse, 1.0)


# ---------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------

def _ref_route(x, k, score, bias, groups, topk_groups, top2, renormalize, scale):
    """64-bit weights and choice, and how near any decision of a row came to a tie that 32 bits could see otherwise."""
    x = x.double().cpu()
    t, e = x.shape
    empty = (x == -math.inf).all(1, keepdim=True)
    s = x.sigmoid() if score == "sigmoid" else torch.where(empty, 0.0, torch.softmax(torch.where(empty, 0.0, x), 1))
    c = s + bias.double().cpu() if bias is not None else s if top2 else x
    c = torch.where(x == -math.inf, -math.inf, c)
    by_score = bias is not None or top2
    allowed = torch.ones_like(c, dtype=torch.bool)
    gap = torch.full((t,), math.inf, dtype=torch.float64)
    if topk_groups < groups:
        parts = torch.sort(c.view(t, groups, -1), dim=2, descending=True)[0]
        value = parts[:, :, :2 if top2 else 1].sum(2)
        ordered, order = torch.sort(value, dim=1, descending=True, stable=True)
        stays = torch.zeros_like(value, dtype=torch.bool).scatter_(1, order[:, :topk_groups], True)
        allowed = stays[:, :, None].expand(-1, -1, e // groups).reshape(t, e)
        if by_score:
            d = ordered[:, topk_groups - 1] - ordered[:, topk_groups]
            gap = torch.minimum(gap, torch.where(d.isnan(), math.inf, d))
    ordered, order = torch.sort(c, dim=1, descending=True, stable=True)
    first = torch.sort(allowed.gather(1, order).to(torch.int8), dim=1, descending=True, stable=True)[1]
    order, ordered = order.gather(1, first), ordered.gather(1, first)
    if by_score:
        d = ordered[:, :k] - torch.nn.functional.pad(ordered, (0, 1), value=-math.inf)[:, 1:k + 1]
        d = torch.where(d.isnan(), math.inf, d)        # (-inf beside -inf: the order is by index)
        gap = torch.minimum(gap, d.min(1)[0])
    at = order[:, :k]
    w = s.gather(1, at)
    total = w.sum(1, keepdim=True)
    if renormalize:
        w = torch.where(total == 0, 0.0, w / torch.where(total == 0, 1.0, total))
    return scale * w, at, gap


def _ref_route_grad(x, at, g, score, renormalize, scale):
    y = x.double().cpu().requires_grad_()
    s = y.sigmoid() if score == "sigmoid" else torch.softmax(y, 1)
    w = s.gather(1, at)
    if renormalize:
        w = w / w.sum(1, keepdim=True)
    return torch.autograd.grad((scale * w * g.double()).sum(), y)[0]


def _check_route(x, k, score="softmax", bias=None, groups=1, topk_groups=1, group_score="max", renormalize=True, scale=1.0, seed=0):
    ops = _ops()
    t, e = x.shape
    counts = torch.ones(e, dtype=torch.int64, device="cuda")
    kw = dict(score=score, renormalize=renormalize, scale=scale)
    w, at = ops.route(x, k, bias=bias, groups=groups, topk_groups=topk_groups, group_score=group_score, counts=counts, **kw)
    want, want_at, gap = _ref_route(x, k, score, bias, groups, topk_groups, group_score == "top2", renormalize, scale)
    assert torch.equal(counts.cpu(), 1 + torch.bincount(at.cpu().reshape(-1), minlength=e))
    clear = gap > 32 * U                               # scores are off by a few units, sums of two and a bias by a few more
    assert clear.double().mean() > 0.9 or t < 20
    assert torch.equal(at.cpu()[clear], want_at[clear])
    _near(w[clear.cuda()], want[clear], 0.0, U * (40 + e / 64), "weights")
    g = torch.randn((t, k), generator=torch.Generator().manual_seed(seed))
    grad = ops.route_backward(x, at, g.cuda(), **kw)
    want = _ref_route_grad(x, at.cpu(), g, score, renormalize, scale)
    # terms of g times a weight, which may cancel
    size = abs(scale) * g.abs().max(1, keepdim=True)[0].double() * k
    _near(grad, want, U * (64 + e / 32) * size * torch.ones_like(want) + 2 * SMALLEST[x.dtype], HALF_ULP[x.dtype] * 1.01, "gradient")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("tokens,experts,groups,topk_groups,k", [
    (1, 1, 1, 1, 1), (3, 2, 1, 1, 2), (17, 8, 1, 1, 2), (5, 60, 1, 1, 4), (100, 64, 8, 3, 6), (33, 60, 6, 2, 7), (16, 256, 8, 4, 8), (1000, 256, 8, 4, 8), (9, 160, 8, 3, 6),
    (50, 128, 1, 1, 8), (7, 512, 16, 5, 16), (4, 1024, 64, 7, 64), (3, 1000, 1, 1, 64), (2, 65, 13, 13, 5), (12, 12, 12, 5, 5)])
def test_route_and_its_gradient(tokens, experts, groups, topk_groups, k, dtype):
    g = torch.Generator().manual_seed(tokens + experts)
    x = (torch.randn((tokens, experts), generator=g) * 1.5).to(dtype).cuda()
    bias = (torch.randn((experts,), generator=g) * 0.1).cuda()
    for renormalize, scale in ((True, 2.5), (False, 1.0)):
        kw = dict(groups=groups, topk_groups=topk_groups, renormalize=renormalize, scale=scale)
        _check_route(x, k, "softmax", **kw)
        _check_route(x, k, "softmax", bias, **kw)
        _check_route(x, k, "sigmoid", **kw)
        _check_route(x, k, "sigmoid", bias, group_score="top2", **kw)


def test_route_equal_scores_masks_and_values_that_are_no_numbers():
    ops = _ops()
    x = torch.zeros((6, 96), device="cuda")
    x[1, 40:] = 1.0
    x[2] = -math.inf                                   # nothing is left
    x[3] = -math.inf
    x[3, [90, 5, 50]] = torch.tensor([1.0, 2.0, 3.0], device="cuda")
    x[4, 70] = math.nan
    x[5, 64:] = -math.inf
    for score in ("softmax", "sigmoid"):
        w, at = ops.route(x, 4, score=score)
        assert at[:4].tolist() == [[0, 1, 2, 3], [40, 41, 42, 43], [0, 1, 2, 3], [50, 5, 90, 0]], at
        assert at[4, 0] == 70 and w[4].isnan().all() and at[5].tolist() == [0, 1, 2, 3]
        assert torch.equal(w[0], torch.full((4,), 0.25, device="cuda")) and not w[2].any() and w[3, 3] == 0
        bias = torch.zeros(96, device="cuda")
        bias[[7, 80]] = 3.0
        assert ops.route(x, 4, score=score, bias=bias)[1][[0, 2, 3, 5]].tolist() == [[7, 80, 0, 1], [0, 1, 2, 3], [50, 5, 90, 0], [7, 0, 1, 2]]
        # experts of other groups are not chosen, even where masks leave too few
        w, at = ops.route(x, 4, score=score, groups=3, topk_groups=1)
        assert at[5].tolist() == [0, 1, 2, 3] and set(at[3].tolist()) == {50, 32, 33, 34} and at[1].tolist() == [40, 41, 42, 43]
        grad = ops.route_backward(x, at, torch.ones((6, 4), device="cuda"), score=score)
        assert not grad[2].isnan().any() and not grad[[0, 1, 2, 3, 5]].isnan().any()


def test_route_of_strided_rows_and_counts_that_are_added_to():
    ops = _ops()
    base = torch.randn((41, 200), generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()
    x = base[1::2, 7:135]
    _check_route(x, 5, "sigmoid")
    counts = torch.full((128,), 5, dtype=torch.int64, device="cuda")
    _, at = ops.route(x, 5, counts=counts)
    ops.route(x, 5, counts=counts)
    assert torch.equal(counts.cpu(), 5 + 2 * torch.bincount(at.cpu().reshape(-1), minlength=128))
    out = torch.full((20, 131), 9.0, dtype=torch.bfloat16, device="cuda")
    g = torch.randn((20, 5), device="cuda")
    ops.route_backward(x, at, g, out=out[:, 1:129])
    assert torch.equal(out[:, 1:129], ops.route_backward(x, at, g)) and (out[:, 129:] == 9).all() and (out[:, 0] == 9).all()


# ---------------------------------------------------------------------------
# all of them
# ---------------------------------------------------------------------------

def _differences(f, x, seed, h=1.0 / 64):
    """d f / d x along a direction, from f itself, and the direction."""
    d = torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)).cuda()
    with torch.no_grad():
        a, b = (float(f(x + t).double()) for t in (h * d, -h * d))
        c, e = (float(f(x + t).double()) for t in (2 * h * d, -2 * h * d))
    return (8 * (a - b) - (c - e)) / (12 * h), d


@pytest.mark.parametrize("seed", range(4))
def test_gradients_against_differences(seed):
    # (central differences of fourth order, h = 1/64: what they leave out is below 1e-5 of the derivative's scale for logits of a few units, and forward values
    # are good to a few units of 2^-24 of theirs: 1e-5 again)
    ops = _ops()
    x = _logits(3, 211, torch.float32, seed, 1.0)
    tokens = torch.randint(0, 211, (3, 2), generator=torch.Generator().manual_seed(seed)).cuda()
    values, indices, lse = _teacher(x, 12, seed, 1.3, torch.float32, True)
    routed = torch.randn((5, 24), generator=torch.Generator().manual_seed(seed)).cuda()
    bias = torch.zeros(24, device="cuda")
    bias[:6] = 100.0                                   # the choice stays while the logits move

    def lp(v):
        r = ops.logprobs(v, tokens, entropy=True, temperature=0.8)
        return r.logprobs.sum() + 0.5 * r.entropy.sum()

    functions = [(lp, x), (lambda v: ops.distill(v, values, indices, None, 1.3)[0].sum(), x), (lambda v: ops.distill(v, values, indices, lse, 1.3)[0].sum(), x)]
    for score in ("softmax", "sigmoid"):
        for renormalize in (False, True):
            def rt(v, score=score, renormalize=renormalize):
                w, at = ops.route(v, 6, score=score, bias=bias, renormalize=renormalize, scale=1.5)
                return (w * (at % 5 + 1)).sum()
            functions.append((rt, routed))
    for i, (f, at) in enumerate(functions):
        y = at.clone().requires_grad_()
        grad, = torch.autograd.grad(f(y), y)
        want, d = _differences(f, at, seed + 10 * i)
        got = float((grad.double() * d.double()).sum())
        scale = float((grad.double().abs() * d.double().abs()).sum()) + 1.0
        assert abs(got - want) <= 2e-3 * scale, (i, got, want)


def _program(ops, x, tokens, values, indices, weights, routed, bias, counts):
    r = ops.logprobs(x, tokens, k=5, entropy=True)
    g = ops.logprobs_backward(x, tokens, r.row_stats, torch.ones_like(r.logprobs), r.entropy, weights)
    loss, stats = ops.distill(x, values, indices)
    dg = ops.distill_backward(x, values, indices, stats, weights)
    l2, g2 = ops.distill_step(x, values, indices, weights, stats[:, 0].contiguous() + 9.0)
    w, at = ops.route(routed, 4, score="sigmoid", bias=bias, groups=4, topk_groups=2, group_score="top2", counts=counts)
    rg = ops.route_backward(routed, at, w, score="sigmoid")
    return [t for t in (*r, g, loss, stats, dg, l2, g2, w, at, rg) if t is not None]


def _program_inputs(batch, n, dtype, seed):
    x = _logits(batch, n, dtype, seed)
    values, indices, _ = _teacher(x, 30, seed, 1.0, torch.bfloat16, False)
    gen = torch.Generator().manual_seed(seed)
    return (x, torch.randint(0, n, (batch, 2), generator=gen).cuda(), values, indices, torch.rand((batch,), generator=gen).cuda(),
            torch.randn((batch, 64), generator=gen).to(dtype).cuda(), torch.randn((64,), generator=gen).cuda(), torch.zeros(64, dtype=torch.int64, device="cuda"))


@pytest.mark.parametrize("batch,n,dtype", [(2, 131072, torch.bfloat16), (600, 3001, torch.float16), (9, 70001, torch.float32)])
def test_the_same_call_gives_the_same_bits_on_any_stream(batch, n, dtype):
    ops = _ops()
    a = _program_inputs(batch, n, dtype, 3)
    first = [t.clone() for t in _program(ops, *a)]
    for _ in range(3):
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(first, _program(ops, *a)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = _program(ops, *a)
    side.synchronize()
    assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(first, again))


def test_operators_in_a_graph():
    ops = _ops()
    a = _program_inputs(4, 50257, torch.bfloat16, 5)
    eager = [t.clone() for t in _program(ops, *a)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _program(ops, *a)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _program(ops, *a)
    for seed in (5, 6, 7, 5):
        b = _program_inputs(4, 50257, torch.bfloat16, seed)
        for p, q in zip(a, b):
            p.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        want = _program(ops, *b)
        assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(held, want))
    assert all(torch.equal(p.view(torch.uint8), q.view(torch.uint8)) for p, q in zip(held, eager))


def test_automatic_differentiation_is_the_backward_calls():
    ops = _ops()
    x, tokens, values, indices, weights, routed, bias, _ = _program_inputs(6, 4001, torch.float32, 8)
    y = x.clone().requires_grad_()
    r = ops.logprobs(y, tokens, k=3, entropy=True, temperature=0.9)
    g = torch.randn_like(r.logprobs)
    (torch.sum(r.logprobs * g) + torch.sum(r.entropy * weights)).backward()
    assert torch.equal(y.grad, ops.logprobs_backward(x, tokens, r.row_stats, g, r.entropy.detach(), weights, 0.9))
    y.grad = None
    ops.logprobs(y, tokens[:, 0].contiguous())[0].sum().backward()              # no entropy, tokens as [batch]
    assert torch.equal(y.grad, ops.logprobs_backward(x, tokens[:, 0].contiguous(), r.row_stats * 0 + ops.logprobs(x).row_stats, torch.ones((6, 1), device="cuda")))
    y.grad = None
    loss, stats = ops.distill(y, values, indices, temperature=1.5)
    (loss * weights).sum().backward()
    assert torch.equal(y.grad, ops.distill_backward(x, values, indices, stats, weights, temperature=1.5))
    z = routed.clone().requires_grad_()
    w, at = ops.route(z, 4, bias=bias)
    (w * 2.0).sum().backward()
    assert torch.equal(z.grad, ops.route_backward(routed, at, torch.full_like(w, 2.0)))


def test_refusals_on_the_gpu():
    from paper_2501_14336_amd.binding import RtopkError
    ops = _ops()
    x = torch.zeros((4, 100), device="cuda")
    tokens = torch.zeros((4, 1), dtype=torch.int64, device="cuda")
    stats, ones = torch.ones((4, 2), device="cuda"), torch.ones(4, device="cuda")
    values, indices = torch.zeros((4, 3), device="cuda"), torch.zeros((4, 3), dtype=torch.int64, device="cuda")
    dstats = torch.ones((4, 8), device="cuda")
    bad = [
        lambda: ops.logprobs(x[0], tokens), lambda: ops.logprobs(x.t(), tokens), lambda: ops.logprobs(x.double(), tokens), lambda: ops.logprobs(x, tokens.int()),
        lambda: ops.logprobs(x, tokens[:3]), lambda: ops.logprobs(x, tokens.cpu()), lambda: ops.logprobs(x, tokens, k=101), lambda: ops.logprobs(x, tokens, k=-1),
        lambda: ops.logprobs(x, tokens, temperature=0.0), lambda: ops.logprobs(x, tokens, temperature=float("nan")), lambda: ops.logprobs(x, tokens, temperature=1e-39),
        lambda: ops.logprobs(x[:0], tokens[:0]), lambda: ops.logprobs(x[:, :0], tokens), lambda: ops.logprobs(x.expand(4, 100)[:1].expand(4, 100), tokens),
        lambda: ops.logprobs_backward(x, tokens, stats, None), lambda: ops.logprobs_backward(x, tokens, stats[:3], ones[:, None]),
        lambda: ops.logprobs_backward(x, tokens, stats, ones[:, None], None, ones), lambda: ops.logprobs_backward(x, tokens, stats, ones[:, None], out=x),
        lambda: ops.logprobs_backward(x, tokens, stats, ones[:, None], out=x.half()), lambda: ops.logprobs_backward(x[:2], tokens[:2], stats[:2], ones[:2, None], out=x[1:3]),
        lambda: ops.distill(x, values, indices[:, :2]), lambda: ops.distill(x, values, indices.int()), lambda: ops.distill(x, values.double(), indices),
        lambda: ops.distill(x, values, indices, ones[:3]), lambda: ops.distill(x, values, indices, temperature=-1.0), lambda: ops.distill(x, values[:, :0], indices[:, :0]),
        lambda: ops.distill_backward(x, values, indices, stats, ones), lambda: ops.distill_backward(x, values, indices, dstats, ones, out=x),
        lambda: ops.distill_step(x, values, indices, ones, out=x), lambda: ops.distill_step(x, values, indices, ones.double()),
        lambda: ops.route(x, 0), lambda: ops.route(x, 101), lambda: ops.route(x, 65), lambda: ops.route(x, 2, groups=3), lambda: ops.route(x, 2, groups=4, topk_groups=5),
        lambda: ops.route(x, 26, groups=4, topk_groups=1), lambda: ops.route(x, 2, score="relu"), lambda: ops.route(x, 2, group_score="mean"),
        lambda: ops.route(x, 2, bias=ones), lambda: ops.route(x, 2, counts=torch.zeros(100, device="cuda")), lambda: ops.route(x, 2, groups=100, topk_groups=2),
        lambda: ops.route(torch.zeros((2, 1025), device="cuda"), 2), lambda: ops.route(x, 2, scale=float("nan")),
        lambda: ops.route_backward(x, indices, values[:, :2]), lambda: ops.route_backward(x, indices, values, out=x), lambda: ops.route_backward(x, indices.int(), values),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(RtopkError) as e:
            f()
        assert e.value.status in (1, 3), i
    torch.cuda.synchronize()
