"""The codes with which a workspace's size is refused: those of the call it is for."""
import pytest

import paper_2407_19644_amd as ubp
from layer_util import layer


@pytest.mark.parametrize("size", [ubp.linear_grad_workspace, ubp.weight_grad_workspace])
def test_codes_of_refused_workspaces(size):
    blocks, W, _ = layer(64, 48, 4, 4, 0.3, "f16", 1)
    p = ubp.pack(W, "f16", 4, 4, blocks)
    for N, code in ((-1, 1), (-2**31, 1), (2**31 - 2**16 + 1, 4), (2**31 - 1, 4)):
        with pytest.raises(ubp.UBPError) as e:
            size(p, N)
        assert e.value.code == code
    assert size(p, 2**31 - 2**16) > 0 and size(p, 0) == 0
