"""Pages that are not there, of every size: larger than a step of the attention, as large, smaller."""
import numpy as np
import pytest

from tests.test_gpu_attn_kv4 import Cache, check, env, queries, shuffled  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("T,D", [(1, 64), (1, 128), (5, 64), (20, 128), (40, 64)])
def test_missing_pages_of_every_size(env, P, T, D):  # noqa: F811
    """The first page, the last, neighbours, all of them."""
    each, n_pages = 6, 20
    table = shuffled(P, 3, each, n_pages).astype(np.int64)
    table[0, [0, 3, 5]] = [-1, n_pages, 2 ** 31 - 1]
    table[1, [1, 2]] = -(2 ** 31)
    table[2, :] = -1
    c = Cache(P + T, n_pages, 2, D, P)
    pos = np.array([each * P - T, 3 * P + 5, 2 * P])
    check(env, c, queries(T, 3, T, 4, D), pos, table)
    check(env, c, queries(T, 3, T, 4, D), pos, table, window=P + 20, sinks=3)
