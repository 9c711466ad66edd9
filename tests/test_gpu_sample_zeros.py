"""GPU: the filtered draw on rows with zeros of both signs beside the smallest values of the type, where a cut may fall
between zero and the largest negative value (the host walks through the same search in test_sample_search.py).  Bounds as
in test_gpu_sample.py: ranks are exact, masses and the draw within 1e-5."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_sample import compare  # noqa: E402

TYPES = {torch.float32: (torch.int32, 32), torch.bfloat16: (torch.int16, 16), torch.float16: (torch.int16, 16)}


def from_bits(bits, dtype):
    kind, n = TYPES[dtype]
    signed = np.asarray(bits, np.int64)
    signed = np.where(signed >= 1 << (n - 1), signed - (1 << n), signed)
    return torch.from_numpy(signed).to(kind).view(dtype).cuda()


@pytest.mark.parametrize("vocab", [300, 1000, 9000, 40000])
@pytest.mark.parametrize("dtype", list(TYPES))
def test_cuts_beside_zero(vocab, dtype):
    n = TYPES[dtype][1]
    sign, R = 1 << (n - 1), 24
    rng = np.random.default_rng(vocab + n)
    rows, ks, ts = [], [], []
    for r in range(R):
        top = {torch.float16: (7, 0x2c41), torch.bfloat16: (7, 0x3f7f), torch.float32: (0x0007ffff, 0x3f7fffff)}[dtype][r % 2]
        zeros = vocab // 4
        row = np.concatenate([[top], np.where(np.arange(zeros) % 3 == 2, sign, 0), np.full(vocab - zeros - 1, sign + 1)])
        if r % 4 > 1:      # other small values of both signs among them
            at = rng.integers(1, vocab, vocab // 8)
            row[at] = np.where(rng.random(len(at)) < 0.5, sign, 0) + rng.integers(0, 900, len(at))
        rng.shuffle(row)
        rows.append(row)
        ks.append(int(rng.integers(2, vocab)) if r % 3 else zeros + 1 + int(rng.integers(0, 3)))
        ts.append((1.0, 200.0, 1.7)[r % 3])
    logits = from_bits(np.stack(rows), dtype)
    u = rng.random(R, dtype=np.float32)
    compare(logits, u, t=ts, k=ks)
    compare(logits, u, t=ts, p=rng.uniform(0.05, 0.95, R))
    compare(logits, u, t=ts, k=ks, p=rng.uniform(0.05, 0.95, R), m=np.full(R, 0.5))
