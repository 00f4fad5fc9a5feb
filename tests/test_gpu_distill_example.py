"""The example that runs the selection, routing, distillation and log probabilities together."""
import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def test_the_student_learns_from_the_kept_logits():
    from paper_2501_14336_amd import distill_example
    losses, used, best, scores = distill_example.run(steps=150)
    assert losses[-1] < 0.5 * losses[0]
    assert int(used.sum()) == 512 * 2 and int((used > 0).sum()) == 8
    assert scores.logprobs.shape == (2000, 1) and (scores.logprobs <= 0).all() and scores.entropy.isfinite().all()
    assert (scores.top_logprobs[:, :1] >= scores.logprobs).all()
    hit = scores.top_indices == best
    assert torch.equal(scores.top_logprobs[hit], scores.logprobs.expand(-1, 5)[hit])


def test_the_first_step_is_what_plain_operations_give():
    from paper_2501_14336_amd import binding as B
    from paper_2501_14336_amd import operators as O
    from paper_2501_14336_amd.distill_example import RoutedStudent
    torch.manual_seed(1)
    vocab, kept, batch = 301, 20, 64
    teacher = torch.randn((vocab, vocab), device="cuda") * 3
    values, indices, _ = B.topk(teacher, kept)
    lse = torch.logsumexp(teacher.double(), 1).float()
    student = RoutedStudent(vocab, 32, 8, 2).cuda()
    tokens = torch.randint(0, vocab, (batch,), device="cuda")
    logits = student(tokens)
    loss, grad = O.distill_step(logits.detach(), values[tokens], indices[tokens], torch.full((batch,), 1.0 / batch, device="cuda"), lse[tokens])
    logits.backward(grad)
    got = [p.grad.double().cpu() for p in student.parameters()]

    plain = RoutedStudent(vocab, 32, 8, 2).cuda()
    plain.load_state_dict(student.state_dict())
    plain = plain.double().cpu()
    x = plain.embedding(tokens.cpu())
    s = plain.router(x).sigmoid()
    at = torch.topk(s, 2, dim=1)[1]                   # (the bias is still 0)
    w = s.gather(1, at)
    w = w / w.sum(1, keepdim=True)
    y = x
    for e, expert in enumerate(plain.experts):
        y = y + (w * (at == e)).sum(1, keepdim=True) * expert(x)
    logp = torch.log_softmax(plain.out(y), 1)
    q = torch.exp(values[tokens].double().cpu() - lse[tokens].double().cpu()[:, None])
    rest, listed = 1 - q.sum(1), indices[tokens].cpu()
    other = torch.logsumexp(logp.scatter(1, listed, -float("inf")), 1)
    want = (q * (q.log() - logp.gather(1, listed))).sum(1) + rest * (rest.log() - other)
    assert torch.allclose(loss.double().cpu(), want, rtol=0, atol=2e-5)
    want.mean().backward()
    for g, p in zip(got, plain.parameters()):
        assert (g - p.grad).abs().max() <= 1e-4 * p.grad.abs().max() + 1e-9
