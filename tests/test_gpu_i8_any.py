"""seer_i8_product where rows do not lie at multiples of 16 bytes, in sizes that go to the tiled kernel for any address."""
import numpy as np
import pytest

from tests.gpu_util import announce
from tests.routed_util import TYPES, shifted, spread
from tests.test_gpu_i8_product import check_product, i8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(TYPES))
@pytest.mark.parametrize("columns", [1, 15, 17, 33, 100, 111, 113, 127])
def test_fewer_columns_than_a_step(columns, kind):
    """Pieces behind the end of a row that is shorter than the 128 columns of a step."""
    announce(f"i8 any, {columns} columns, {kind}")
    rng = np.random.default_rng(columns)
    for M, N in ((300, 300), (1000, 1000), (641, 129)):
        check_product(spread(i8(rng, M, columns), columns + 1, 99), spread(i8(rng, N, columns), columns + 2, -77)[None], None, kind, rng)
    lengths = [700, 0, 1, 129, 513, 300, 255, 102]
    a, b = shifted(i8(rng, sum(lengths) + 37, columns), 1), shifted(i8(rng, 8, 256, columns), 3)
    check_product(a, b, np.concatenate([[0], np.cumsum(lengths)]).tolist(), kind, rng)
