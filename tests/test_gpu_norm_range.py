"""isc_rms_norm_quant where the way to a row's scale leaves the range of single precision and the scale does not."""
import pytest

import paper_2108_09413_b200 as isc
from test_gpu_norm_quant import TYPES, check

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LARGEST = float(torch.finfo(torch.float32).max)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,width", [(5, 64), (3, 500), (4, 4096), (2, 9000), (1300, 4096), (2, 20000)])
def test_largest_weights_and_eps(kind, rows, width):
    dtype = TYPES[kind]
    g = torch.Generator(device="cuda").manual_seed(width)
    # one element of 0.01 times a weight of 2e38: the normed value is sqrt(width) times the weight, its 127th part a number again
    x = torch.zeros(rows, width, device="cuda")
    x[:, width // 3] = 0.01
    w = torch.ones(width, device="cuda")
    w[width // 3] = 2e38
    check(isc.rms_norm_quant(x.to(dtype), w, 0.0), x.to(dtype), None, w, 0.0)
    # sums that single precision cannot add eps to
    x = (torch.randn(rows, width, device="cuda", generator=g) * 1e17).to(dtype)
    one = torch.ones(width, device="cuda")
    for eps in (LARGEST, 3.4e38, 1e38):
        check(isc.rms_norm_quant(x, one, eps), x, None, one, float(torch.tensor(eps, dtype=torch.float32)))
    # scales below the smallest normal number
    small = (torch.rand(rows, width, device="cuda", generator=g) * 2.0**-20 + 2.0**-21).to(dtype)
    check(isc.rms_norm_quant(small, one, LARGEST), small, None, one, LARGEST)
    tiny = torch.full((width,), 2.0**-70, device="cuda")
    check(isc.rms_norm_quant(small, tiny, LARGEST), small, None, tiny, LARGEST)
