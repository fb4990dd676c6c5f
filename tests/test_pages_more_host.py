"""Pages of a pool, as far as it goes without a GPU: what pins the oracle where pages are held."""
from oracle import pages_oracle


def test_a_held_page_that_is_not_full_is_copied():
    # a stored prompt of 20 tokens in pages of 16; who holds pages 0 and 1 may go on from there too
    held = [1, 1, 0, 0]
    assert pages_oracle.fork([[0, 1, -1]], [20], [0], held, 16, 4) == ([[0, 2, -1]], [20], [1], [2], 0)
    assert pages_oracle.fork([[0, 1, -1]], [20], [0, 0], held, 16, 4) == ([[0, 2, -1], [0, 3, -1]], [20, 20], [1, 1], [2, 3], 0)
    assert pages_oracle.fork([[0, 1, -1]], [20], [0, 0], [1, 1, 1, 0], 16, 4) == ([[0, 3, -1], [0, -1, -1]], [20, 20], [1, -1], [3, -1], 1)
    # whole pages are shared, held or not; a page that nobody holds stays with the first
    assert pages_oracle.fork([[0, 1, -1]], [32], [0, 0], held, 16, 4) == ([[0, 1, -1], [0, 1, -1]], [32, 32], [-1, -1], [-1, -1], 0)
    assert pages_oracle.fork([[0, 1, -1]], [20], [0, 0], [1, 0, 0, 0], 16, 4) == ([[0, 1, -1], [0, 2, -1]], [20, 20], [-1, 1], [-1, 2], 0)
