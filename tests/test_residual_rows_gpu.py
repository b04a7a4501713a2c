"""The joint's rows of two runs a lane on 256 threads (2056 to 4096 channels), and the widest
ones of each kernel, as its other sizes: against the formula in 64 bits."""
import pytest

from gpu_util import require_gpu
from test_residual_norm_gpu import ALL, TYPES, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", TYPES, ids="-".join)
@pytest.mark.parametrize("sizes", [(2, 3, 2048), (1, 5, 2056), (3, 4, 2304), (2, 3, 4088), (1, 2, 4096), (2, 2, 6144), (1, 3, 8192), (2, 2, 8200)],
                         ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("given", [ALL, ("f", "w", "dro")], ids=["all", "some"])
def test_rows(given, sizes, types):
    require_gpu()
    check(make(*sizes, types, seed=sizes[2]), types, given)
