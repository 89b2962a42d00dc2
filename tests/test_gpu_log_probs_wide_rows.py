"""isc_log_probs of logits further apart than the largest single-precision number, at factors that bring them near each other."""
import math

import pytest

from test_gpu_log_probs import TYPES, check, some_targets

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,vocab", [(6, 10), (6, 50), (6, 700), (6, 20000), (2, 131072), (2500, 5001), (900, 17000)])
@pytest.mark.parametrize("scale", [2.0**-126, 2.0**-124, 2.0**-118, 2.0**-60])
def test_far_apart(kind, rows, vocab, scale):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = (2.0 * torch.rand(rows, vocab + 1, device="cuda", generator=g) - 1.0) * 3.3e38
    x[1::6] = torch.where(torch.rand(vocab + 1, device="cuda", generator=g) < 0.5, 3.3e38, -3.3e38)
    x[2::6] = x[2::6].sort(1).values
    x[3::6, ::3] = torch.finfo(TYPES[kind]).min
    x[4::6, ::2] = -math.inf
    x[5::6] *= 1e-3
    x = x.to(TYPES[kind])[:, :vocab]
    check(x, some_targets(rows, vocab, g), 4, scale)
