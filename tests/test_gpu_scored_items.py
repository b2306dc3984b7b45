"""dk_scored_attend in fp32 with items of 16 and of 32 packed rows, against the oracle with the bounds of test_gpu_scored."""
import pytest

from test_gpu_scored import MASKS, Batch, _masks

pytestmark = pytest.mark.gpu


# 84, 176 and 416 tiles of 32 rows: 16 rows an item; 32 unless rows have starts of their own; 32
@pytest.mark.parametrize("delta", [[90, 75], [200, 150], [430, 400]], ids=["short", "middle", "long"])
@pytest.mark.parametrize("kind", ["cap", "slopes", "window", "prefix", "all", "first"])
@pytest.mark.parametrize("d", [64, 128])
def test_items_of_both_heights(d, kind, delta):
    b = Batch(50, 16, 4, d, "f32", hist=[60, 200], delta=delta)
    b.check(False, **_masks(b, MASKS[kind]))
