"""Long lists of top logits on both sides of the rules by rows and by the list's length."""
import pytest

import test_gpu_distill as distill

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", distill.TYPES)
@pytest.mark.parametrize("kind", ["normal", "ties", "lowest", "up", "nan"])
@pytest.mark.parametrize("rows,classes,k", [(511, 2500, 65), (512, 2500, 65), (512, 2300, 100), (512, 2300, 101), (2047, 2100, 128), (2048, 2100, 128), (2048, 2100, 129)])
def test_top(rows, classes, k, kind, dtype):
    distill.check_top(distill.fill(kind, rows, classes, dtype, 40).cuda(), k)
