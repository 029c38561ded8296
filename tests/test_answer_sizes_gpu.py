"""The example behind a binary layer at sizes that are no multiple of anything."""
import math

import pytest

from paper_1603_05279_amd import answer as ans

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,inputs,width,classes", [(1, 64, 32, 2), (77, 100, 65, 9), (301, 333, 130, 41)])
def test_sizes(rows, inputs, width, classes):
    got = ans.run(rows=rows, inputs=inputs, width=width, classes=classes, steps=2, report=lambda line: None)
    assert abs(got["losses"][0] - math.log(classes)) < 1e-5 and math.isfinite(got["losses"][-1]) and got["same"] > 0.5
