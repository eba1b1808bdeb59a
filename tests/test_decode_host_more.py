"""Host side of the decoding-step calls, continued: pages that leave the tables."""
import numpy as np

from oracle import decode as ref


def test_oracle_pages_that_leave():
    """Two beams of 36 tokens that share a page of 16: the second's full page of its own is in no table afterwards, the
    pages in progress stay."""
    cache = dict(k=np.zeros((5, 1, 16, 8)), v=np.zeros((5, 1, 16, 8)), k_mean=None, lens=np.array([36, 36]),
                 table=np.array([[0, 1, 2], [0, 3, 4]]))
    table, lens, _ = ref.reorder(cache, np.array([[0, 0]]))
    assert table.tolist() == [[0, 1, 2], [0, 1, 4]] and lens.tolist() == [36, 36]
    cache.update(table=np.array([[0, 1], [2, 3]]), lens=np.array([20, 20]))
    assert ref.reorder(cache, np.array([[0, 0]]))[0].tolist() == [[0, 1], [0, 3]]
