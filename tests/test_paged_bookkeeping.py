"""PagedKVCache's pages and lengths (host side; no kernel runs)."""
import pytest
import torch

import paper_2509_15763_amd as u


def make(**kw):
    a = dict(B=3, Hkv=1, n_pages=10, page=4, max_rows=20, D=8, device="cpu", weights=True)
    a.update(kw)
    return u.PagedKVCache(**a)


def taken(c):
    return sorted(p for ps in c.pages for p in ps)


def test_pages_are_dealt_and_given_back():
    c = make()
    c.extend([5, 0, 1])
    assert c.rows == [5, 0, 1] and [len(p) for p in c.pages] == [2, 0, 1]
    assert c.kv_len.tolist() == [5, 0, 1] and c.cu.tolist() == [0, 5, 5, 6]
    assert c.table.shape == (3, 5) and c.table[0, :2].tolist() == c.pages[0] and (c.table[0, 2:] == -1).all() and (c.table[1] == -1).all()
    c.extend([3, 1, 3])  # fills the pages there are, and one more
    assert [len(p) for p in c.pages] == [2, 1, 1] and len(c.free) == 6
    assert sorted(c.free + taken(c)) == list(range(10))
    c.release(0)
    assert c.rows == [0, 1, 4] and c.kv_len.tolist() == [0, 1, 4] and len(c.free) == 8


def test_refusals_change_nothing():
    c = make()
    c.extend([20, 4, 0])
    before = (list(c.rows), [list(p) for p in c.pages], list(c.free), c.new)
    for n in ([1, 0, 0], [0, 20, 0], [0, 4, 20], [0, -1, 0], [1, 1]):  # max_rows, max_rows, pages, negative, too few
        with pytest.raises(u.UnigistError):
            c.extend(n)
    with pytest.raises(u.UnigistError):
        c.evict([1])
    with pytest.raises(u.UnigistError):
        c.evict([-1, 0, 0])
    with pytest.raises(u.UnigistError):
        c.evict([19, 3, 0])  # five and one pages, while four are free
    assert before == (c.rows, c.pages, c.free, c.new)
    with pytest.raises(u.UnigistError):
        make(weights=False).evict([0, 0, 0])
    with pytest.raises(u.UnigistError):
        make(dtype=torch.uint8)  # no scales


@pytest.mark.parametrize("keep", [[1, 1, 1, 1], [1, 1], [5, 2, 1]], ids=["too many", "too few", "refused by the call"])
def test_an_eviction_that_is_refused_changes_nothing(keep):
    c = make()  # on the CPU: the call itself refuses
    c.extend([9, 4, 1])
    before = (list(c.rows), [list(p) for p in c.pages], list(c.free), c.kv_len.tolist())
    with pytest.raises(u.UnigistError):
        c.evict(keep)
    assert before == (c.rows, c.pages, c.free, c.kv_len.tolist())
