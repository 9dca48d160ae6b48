"""How near the sines and cosines of rotated fp32 heads are to those in 64 bits."""
import numpy as np
import pytest
import torch

from paper_1705_09864_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("factor", [1.0, 1.2, -0.7])
@pytest.mark.parametrize("interleaved", [False, True])
def test_sines_and_cosines(interleaved, factor):
    """A pair (1, 0) becomes its angle's cosine and sine, computed in 64 bits, times the factor, and rounded to fp32 once: by half a step, 2^-24 of the result, and
    2^-25 at most up to 1.  The series end with a^11 and a^10, a <= pi / 4: a sine's next part is a^13 / 13! < 1e-11 of it, a cosine's a^12 / 12! < 2e-10.  The angles
    themselves, up to 4400, are products in 64 bits on either side, off by 2^-53 of that four times: below 2e-12, which the factor multiplies (f cos t changes by f sin t)."""
    rng = np.random.default_rng(5)
    rows, pairs = 4096, 128
    freq = torch.from_numpy(rng.random(pairs))
    freq[:4] = torch.tensor([np.pi / 2, np.pi / 2 + 1e-3, np.pi / 4, 2 * np.pi / 3], dtype=torch.float64)
    x = torch.zeros((rows, 1, pairs, 2), device="cuda")
    x[..., 0] = 1
    if not interleaved:
        x = x.transpose(2, 3).contiguous()
    positions = torch.arange(rows, dtype=torch.int32, device="cuda") - rows // 2
    got = B.rotary(x.view(rows, 1, 2 * pairs), positions, freq.cuda(), interleaved, factor).double().cpu().numpy()
    got = got.reshape(rows, pairs, 2) if interleaved else got.reshape(rows, 2, pairs).transpose(0, 2, 1)
    angle = positions.cpu().numpy().astype(np.float64)[:, None] * freq.numpy()[None]
    want = factor * np.stack([np.cos(angle), np.sin(angle)], -1)
    off = 2.0**-24 * np.where(np.abs(want) < 1, np.minimum(0.5, np.abs(want)), np.abs(want)) + 2e-10 * np.abs(want) + abs(factor) * 2e-12
    err = np.abs(got - want)
    bad = int((err > off).sum())
    assert bad == 0, (bad, float((err / off).max()), want[err > off][:3].tolist())
