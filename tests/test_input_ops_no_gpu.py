"""The operators that form Q, K and V on a machine without a GPU: what their launches make of it."""
import os

import pytest

import __graft_entry__

__graft_entry__._build_module().build()
import paper_2609_35593_gb300 as ress  # noqa: E402
from test_input_ops_cpu import ln, ln_bwd, norm, rope, rope_bwd  # noqa: E402

ECUDA = -4


@pytest.mark.skipif(os.path.exists("/dev/nvidiactl"), reason="the calls would run: needs a machine without a GPU")
def test_a_failed_question_about_the_gpu_is_the_calls_error_and_is_not_kept():
    """Without a GPU the first thing that a call cannot learn ends it, before any launch."""
    torch = pytest.importorskip("torch")
    assert not torch.cuda.is_available()
    before = ress.kernel_launches()
    for _ in range(2):
        assert ln(norm()) == ECUDA and ln_bwd(norm()) == ECUDA and rope() == ECUDA and rope_bwd() == ECUDA
        assert ress.kernel_launches() == before
