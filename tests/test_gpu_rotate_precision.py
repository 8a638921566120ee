"""How exact the sines and cosines of the rotation are, by pairs (1, 0), which it turns into (cos, sin) without another rounding."""
import numpy as np
import pytest
import torch

from paged_cases import dev, ints
from paper_2503_00540_amd.rekv import Rekv

pytestmark = pytest.mark.gpu

# In units of 2^-24, with |y| <= pi / 4 the angle that is left.  Sine: 0.5 for y, 0.5 for the result (each half a step below 1), 0.34 for
# z y s, |z y| <= 0.485 and |s| <= 0.168 with 4.2 roundings, 0.03 for the series.  Cosine: 0.5 |sin y| <= 0.36 for y, 0.5 for the result, 0.52 for
# z d, z <= 0.617, d within 0.35 and z's own rounding times 0.5.  Either below 1.4; positions below 2^20 add 2^20 * 2^-51 * pi / 2 at most, here 0.01.
BOUND = 1.41 * 2.0 ** -24


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_sines_and_cosines(layout):
    d, n = 256, 20000
    r = Rekv(2, 1, d, 16, "f32")
    pos = np.random.default_rng(1).integers(-(1 << 20), 1 << 20, n).astype(np.int32)
    x = np.zeros((n, 1, d), np.float32)
    first, second = (slice(0, d // 2), slice(d // 2, d)) if layout == "half" else (slice(0, d, 2), slice(1, d, 2))
    x[..., first] = 1
    t = pos[:, None].astype(np.float64) * 1e4 ** (-2.0 * np.arange(d // 2) / d)
    for inverse in (False, True):
        got = r.rotate(dev(x), dev(pos), layout=layout, inverse=inverse).double().cpu().numpy()[:, 0]
        for part, want in ((first, np.cos(t)), (second, np.sin(-t if inverse else t))):
            err = np.abs(got[:, part] - want)
            assert err.max() <= BOUND, err.max() * 2.0 ** 24
            assert np.sqrt((err ** 2).mean()) <= 2.0 ** -25          # (each rounding on its own is 2^-25 / sqrt(3) at most)


def test_appended_keys_are_turned_by_the_same_angles():
    r = Rekv(2, 1, 64, 16, "f32")
    k = torch.zeros((3000, 1, 64), device="cuda:0")
    k[..., :32] = 1
    pages = torch.zeros((3000 // 16 + 1, 16, 1, 64), device="cuda:0")
    r.append_kv(k, k, pages, pages.clone(), ints([0, 3000]), ints([3000]), ints([list(range(3000 // 16 + 1))]))
    assert torch.equal(pages.view(-1, 1, 64)[:3000], r.rotate(k, ints(list(range(3000)))))
