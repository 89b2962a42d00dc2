"""isc_log_probs of masked rows at factors at which no finite number is far enough below the others to stand for a mask."""
import math

import pytest

import paper_2108_09413_b200 as isc
from test_gpu_log_probs import TYPES, check, some_targets

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

KINDS = ["bf16", "fp16", "fp32"]
SCALES = [1e-30, 1e-6, 1e-5, 1e-4, 1e-3, 1e-2, 0.25, 1e9]


def masked_rows(rows, vocab, kind, g):
    """70 % masks around numbers of every sort; the pitch is odd, so that the rows begin at every alignment"""
    pitch = (vocab + 1) | 1
    x = torch.randn(rows, pitch, device="cuda", generator=g) * 3.0
    x[1::9] -= 60000.0
    x[2::9] = -65472.0                                         # fp16's last but one
    x[3::9] = torch.finfo(TYPES[kind]).min
    x[4::9] = x[4::9].abs() + 60000.0
    x.masked_fill_(torch.rand(rows, pitch, device="cuda", generator=g) < 0.7, -math.inf)
    x[5::9, : vocab // 2] = -math.inf
    x[6::9] = -math.inf                                        # nothing left
    x[7::9] = -math.inf
    x[7::9, vocab // 3] = -3.0                                 # one left
    x[8::9] = torch.randn(pitch, device="cuda", generator=g)   # no masks
    return x.to(TYPES[kind])[:, :vocab]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [40, 65, 700, 5000, 20000, 131072])
@pytest.mark.parametrize("scale", SCALES)
def test_masks_weigh_nothing(kind, vocab, scale):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = masked_rows(18, vocab, kind, g)
    check(x, some_targets(18, vocab, g), 3, scale)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,vocab", [(2500, 5001), (900, 17000)])
@pytest.mark.parametrize("scale", [1e-30, 1e-5, 1e-3, 0.25])
def test_masks_of_many_rows_weigh_nothing(kind, rows, vocab, scale):
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = masked_rows(rows, vocab, kind, g)
    check(x, some_targets(rows, vocab, g), 3, scale)


@pytest.mark.parametrize("vocab", [65, 700, 20000, 131072])
def test_result_does_not_depend_on_the_rows_alignment(vocab):
    """The same fp16 row at each of the eight places within 16 bytes."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    row = masked_rows(9, vocab, "fp16", g)[1].float()
    for scale in (1e-5, 1e-4, 1e-3):
        x = torch.zeros(8, vocab + 16, device="cuda", dtype=torch.float16)
        results = []
        for at in range(8):
            x[:, at:at + vocab] = row.half()
            results.append(float(isc.log_probs(x[:1, at:at + vocab], scale=scale)[1][0]))
        # each is within its own roundings: see `check`
        assert max(results) - min(results) <= 2 * 360 * 2.0**-24 * (2 + 2 * max(results))



@pytest.mark.parametrize("vocab", [700, 20000, 131072])
@pytest.mark.parametrize("scale", [1e-5, 1e-3, 1.0])
def test_stretches_with_and_without_masks(vocab, scale):
    """fp16's lowest number is no mask, beside masks and far from them."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = torch.randn(8, vocab + 1, device="cuda", generator=g) * 3.0
    i = torch.arange(vocab + 1, device="cuda")
    x[:, i // 64 % 3 == 1] = -65504.0
    x[:, i // 100 % 4 == 2] = -math.inf
    x[4:, i % 7 == 3] = -65504.0
    x[6:] -= 65000.0
    x[6:].clamp_(min=-65504.0)
    x[6:, i // 200 % 2 == 0] = -math.inf
    x = x.half()[:, :vocab]
    check(x, some_targets(8, vocab, g), 5, scale)
    many = x.repeat(120, 1)
    check(many, some_targets(960, vocab, g), 5, scale)
