"""The projection where a pair of CTAs takes one unit after another: tiles of 1 to 4 heads in turn, every kind of
plan, with and without norm and bias.  (8000 tokens are 32 stripes; a GB300 has 76 pairs.)"""
import pytest

torch = pytest.importorskip("torch")

from test_gpu_input_ops import float32_by_default, qkv_case, ress  # noqa: E402, F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H", [3, 5, 6, 7])
@pytest.mark.parametrize("plan", [((32, 32), "sections"), ((64,), "halves"), ((32, 32), "interleaved"),
                                  ((10, 6, 14), "sections"), ((14,), "interleaved"), None])
@pytest.mark.parametrize("norms,bias", [((True, True), True), ((False, True), False), ((False, False), False)])
def test_pairs_with_several_units(ress, H, plan, norms, bias):  # noqa: F811
    assert 32 * 3 * -(-H // 4) > torch.cuda.get_device_properties(0).multi_processor_count // 2
    qkv_case(ress, 8000, H, 128, plan, norms, bias, seed=4)


def test_many_units_per_pair(ress):  # noqa: F811
    qkv_case(ress, 20011, 13, 192, ((10, 6, 14), "sections"), seed=5)
