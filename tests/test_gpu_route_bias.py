"""A bias at an expert that is not there (a logit of -inf) counts for nothing,
whatever its value: selections, weights and places are those of the definition
in float64 (bounds of tests/test_gpu_route.py)."""

import pytest
import torch
from test_gpu_route import _bias, _check, _logits, _opts

pytestmark = pytest.mark.gpu

F32, F64, BF = torch.float32, torch.float64, torch.bfloat16
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def C():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_21137_amd import cardan
    return cardan


@pytest.mark.parametrize("dtype", [F32, BF, F64])
@pytest.mark.parametrize("N", [9, 60, 200])
@pytest.mark.parametrize("o", [_opts(4), _opts(4, "softmax", False), _opts(4, "sigmoid"), _opts(4, "sigmoid", False),
                               _opts(4, "sigmoid", True, 1.0, 4, 2, 2), _opts(4, "softmax", False, 2.0, 4, 2, 1)])
def test_bias_of_an_expert_that_is_not_there(C, o, N, dtype):
    z, bias = _logits(N, 32, dtype, 3), _bias(32)
    z[:, 3] = -INF          # in no row: NaN and +inf there are in no row's way
    z[:, 20] = -INF
    bias[3], bias[20] = NAN, INF
    z[::2, 9] = -INF        # pinned on where it is there
    bias[9] = INF
    z[5] = -INF             # a padding row
    z[7, 2:] = -INF
    idx, w, place, _ = _check(C, z, bias, o)
    assert not torch.isnan(w).any()
    assert (idx[5] == -1).all() and (w[5] == 0).all() and (place[5] == -1).all()
    assert (idx[1] == 9).any() and not (idx[0] == 9).any()
    assert ((idx != 3) & (idx != 20)).all()
