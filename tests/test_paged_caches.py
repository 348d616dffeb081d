"""PagedCaches: which pages a place holds, on the CPU (the pools' addresses are never followed)."""
import pytest

torch = pytest.importorskip("torch")

from paper_2604_21215_amd.paged import PagedCaches  # noqa: E402


def _pages(c, place):
    return [int(p) for p in c.table[place] if int(p) >= 0]


@pytest.mark.parametrize("bits", [0, 8])
def test_pages_are_given_out_once_and_come_back(bits):
    c = PagedCaches(2, 3, 4, 100, 10, page_len=16, bits=bits, device="cpu")
    assert c.layer[0].bits == bits and c.layer[1].pages == 10 and c.layer[0].page_len == 16 and c.layer[0].table_stride == 7
    assert (c.layer[0].K_exp is None) == (bits == 0)
    c.reserve([33, 0, 16, -1])
    assert [len(_pages(c, s)) for s in range(4)] == [3, 0, 1, 0] and len(c.free) == 6
    first = _pages(c, 0)
    c.reserve([20, 17, 16, 0])          # less than place 0 holds: nothing changes there
    assert _pages(c, 0) == first and len(_pages(c, 1)) == 2
    held = sum((_pages(c, s) for s in range(4)), [])
    assert len(set(held)) == len(held) == 6 and not set(held) & set(c.free)
    c.release(0)
    assert _pages(c, 0) == [] and set(first) <= set(c.free)
    c.reserve([0, 0, 0, 100])
    assert len(_pages(c, 3)) == 7 and len(c.free) == 0


def test_refusals_give_nothing_out():
    c = PagedCaches(1, 1, 3, 64, 5, page_len=16, device="cpu")
    with pytest.raises(MemoryError):
        c.reserve([64, 32, 0])
    with pytest.raises(ValueError):
        c.reserve([65, 0, 0])
    assert len(c.free) == 5 and all(_pages(c, s) == [] for s in range(3)) and c.held == [0, 0, 0]
    with pytest.raises(ValueError):
        PagedCaches(1, 1, 1, 64, 4, bits=4, device="cpu")
