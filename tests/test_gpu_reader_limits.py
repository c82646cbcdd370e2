"""The attention over latent caches and behind shared prefixes at the ends of what its arguments may be."""
import pytest
import torch

import test_gpu_latent as latent
import test_gpu_latent_expanded as expanded
import test_gpu_shared_prefix as shared
from gpu_utils import announce

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def fsr():
    import paper_2604_20503_amd as f
    f.load_library()
    return f


@pytest.mark.parametrize("most", [2 ** 31 - 1, 2 ** 30, 2 ** 30 + 1])
@pytest.mark.parametrize("dtype", [BF, F32])
def test_any_number_of_workgroups_is_a_bound(fsr, dtype, most):
    """A bound beyond the device's units is none, up to the largest number."""
    announce(f"bounds on workgroups: {dtype} {most}")
    a = latent.Batch(51, [70, 3], [2, 1], 16, 512, 64, 16, dtype)
    assert all(torch.equal(x, y) for x, y in zip(latent.run(fsr, a, dtype, max_workgroups=most), latent.run(fsr, a, dtype)))
    b = expanded.Batch(52, [30], [200], 2, expanded.BIG, dtype)
    assert all(torch.equal(x, y) for x, y in zip(b.run(fsr, dtype, max_workgroups=most), b.run(fsr, dtype)))
    c = shared.Batch(53, [(100, [(5, 2), (9, 1)])], 8, 2, 128, 16, dtype)
    assert all(torch.equal(x, y) for x, y in zip(c.run(fsr, dtype, max_workgroups=most), c.run(fsr, dtype)))
