"""Arguments that the binding must not pass over: host tensors, so that nothing is launched."""
import pytest

import __graft_entry__

torch = pytest.importorskip("torch")
__graft_entry__._build_module().build()
import paper_2609_35593_gb300 as ress  # noqa: E402


def test_gradients_of_a_norm_of_k_without_k():
    """Nothing would be written to them."""
    pos, h, g = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, 2, 64), (torch.zeros(64), torch.zeros(64))
    with pytest.raises(ValueError, match="k_norm_grads"):
        ress.rope_bwd(ress.rope_plan((32, 32)), pos, h, h, k_norm_grads=g)
    with pytest.raises(ValueError, match="k_norm_grads"):
        ress.rope_bwd(ress.rope_plan((32, 32)), pos, h, h, q=h, q_norm=(None, None), q_norm_grads=g, k_norm_grads=g)
