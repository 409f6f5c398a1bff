"""The recurrence on every way that a call is spread over the chip (layer_plans), against the plain 64-bit
reference, with the tolerances of test_gpu_scan."""
import pytest

import layer_plans as plans
import test_gpu_scan as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [s for s, _, _ in plans.SCAN])
def test_recurrence(shape, dtype):
    B, C, L = shape
    S.run_case(B, C, L, dtype, L, packed=B == 2, lengths=B > 2, carry=True)


@pytest.mark.parametrize("shape", [(3, 1400, 1100), (2, 600, 2600)])
def test_recurrence_of_ragged_samples(shape):
    """A sample that ends at once, one that ends at the last position and one between, with starts."""
    S.run_case(*shape, "f32", 3, packed=True, lengths=True, carry=True)
