"""epl_dispatch_backward where the threads of a workgroup change: at 3, 4, 8 and 9 choices, and where a row's 16-byte vectors
need one more wave or one more pass."""
import pytest

from tests.test_gpu_dispatch_weighted import test_backward as check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [3, 4, 8, 9])
@pytest.mark.parametrize("vectors", [448, 511, 512, 513, 768, 769, 832, 1024, 1025, 1344])
def test_backward(vectors, k):
    check((1, 12, k, 11, 8 * vectors, 0))
