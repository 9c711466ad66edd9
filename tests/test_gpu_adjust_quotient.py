"""GPU: the repetition penalty of positive logits is their quotient, rounded once, whatever the penalty."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("vocab", [50, 8192, 8193, 40000])      # lists counted beside a row's entries, and in a hash table
@pytest.mark.parametrize("repetition", [1.1, 1.7, 0.3, 1e-39, 2.0 ** -149, 3e38, 3.0])
def test_positive_logits_are_divided(repetition, vocab):
    from paper_1906_04585_b200 import sequence as S
    gen = torch.Generator().manual_seed(vocab)
    x = torch.randn(3, vocab, generator=gen)
    x[:, ::7] *= 1e-5
    x[:, 1::7] *= 1e-30
    x[1] *= 1e30
    history = torch.stack([torch.randperm(vocab, generator=gen)[:40] for _ in range(3)])
    rep = torch.full((3,), repetition)
    want = x.clone()
    hit = x.gather(1, history)
    want.scatter_(1, history, torch.where(hit > 0, hit / rep.unsqueeze(1), hit * rep.unsqueeze(1)))
    got = S.adjust_logits(x.cuda(), history=history.to(torch.int32).cuda(), repetition=rep.cuda())
    assert torch.equal(got.cpu(), want)
