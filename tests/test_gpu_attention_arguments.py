"""Arguments that raise while they are looked at."""
import pytest
import torch

import paper_2406_06484_amd as dn

pytestmark = pytest.mark.gpu


class Undecided:
    def __bool__(self):
        raise KeyError("neither")


def test_an_error_of_the_callers_own_comes_back_as_it_is():
    q, k = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, 2, 64, device="cuda")
    with pytest.raises(KeyError, match="neither"):
        dn.deltanet_qk_norm_rope_fwd(q, k, interleaved=Undecided())
    with pytest.raises(RuntimeError):
        dn.deltanet_qk_norm_rope_fwd(q, k, interleaved=torch.zeros(2))
    with pytest.raises(TypeError):
        dn.deltanet_qk_norm_rope_fwd(q, k, eps="small")
    a, b = dn.deltanet_qk_norm_rope_fwd(q, k, interleaved=False)
    assert a.shape == q.shape and not b.any()
