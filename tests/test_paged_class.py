"""PagedKVCache on the CPU, over stand-ins for the calls that it makes: what it hands to them and what it refuses."""
import numpy as np
import pytest
import torch

import oracle
import paper_2509_15763_amd as u


def evict(k, v, table, kv_len, weight, keep, k_out, v_out, table_out, max_kv, max_keep, sinks=0, recent=0, weight_out=None):
    """paged_evict by the oracle's selection; on one pool, no page is both read and written."""
    B, Hkv, page = table.shape[0], k.shape[1], k.shape[2]
    if k_out is k:
        assert not set(table[table >= 0].tolist()) & set(table_out[table_out >= 0].tolist())
    rows = torch.zeros(B, dtype=torch.int32)
    kept = torch.full((B, Hkv, max_keep), -1, dtype=torch.int32)
    for b in range(B):
        L, n = int(kv_len[b]), min(int(keep[b]), int(kv_len[b]))
        assert 0 <= L <= max_kv and int(keep[b]) <= max_keep
        at = lambda t, j: (int(t[b, j // page]), j % page)
        for h in range(Hkv):
            w = np.array([float(weight[at(table, j)[0], h, at(table, j)[1]]) for j in range(L)])
            for i, j in enumerate(oracle.paged_select(w, n, sinks, recent)):
                kept[b, h, i] = int(j)
                (p, s), (po, so) = at(table, j), at(table_out, i)
                assert p >= 0 and po >= 0
                for x, y in ((k, k_out), (v, v_out), (weight, weight_out)):
                    y[po, h, so] = x[p, h, s]
        rows[b] = n
    return rows, kept


def attn(q, k, v, table, kv_len, r, W, cu=None, **kw):
    return q, (r, W, kw["sinks"])


@pytest.fixture
def calls(monkeypatch):
    monkeypatch.setattr(u.binding, "paged_evict", evict)
    monkeypatch.setattr(u.binding, "paged_attn", attn)
    monkeypatch.setattr(u.binding, "paged_append", lambda *a, **kw: None)


def make(**kw):
    a = dict(B=3, Hkv=2, n_pages=10, page=4, max_rows=20, D=8, device="cpu", weights=True)
    a.update(kw)
    return u.PagedKVCache(**a)


def queries(c):
    return torch.zeros(4, sum(c.new), c.D, dtype=torch.bfloat16)


def test_a_mask_that_hides_rows_of_an_evicted_sequence_is_refused(calls):
    # rows 0, 1, .. of an evicted sequence are survivors, others for every head: "every fifth row" or "the last four" means nothing
    c = make()
    c.extend([12, 8, 0])
    c.attend(queries(c), 4, 4)
    c.evict([6, 8, 0])
    c.extend([1, 1, 1])
    for kw in (dict(W=4), dict(W=6), dict(W=1, sinks=6), dict(W=6, window_mode=u.UNIGIST_WINDOW_UNITS)):
        with pytest.raises(u.UnigistError, match="renumbered"):
            c.attend(queries(c), 4, **kw)
    for kw in (dict(W=7), dict(W=1 << 22), dict(W=1, sinks=7)):  # sequence 0 has 7 rows now; the others (9 and 1) keep their mask
        c.attend(queries(c), 4, **kw)
    c.extend([0, 1, 1])  # no new row of sequence 0
    c.attend(queries(c), 4, 4)
    c.extend([1, 0, 0])
    with pytest.raises(u.UnigistError, match="renumbered"):
        c.attend(queries(c), 4, 7)
    c.release(0)
    c.extend([9, 0, 0])  # another sequence in its place
    c.attend(queries(c), 4, 4)
    c.evict([0, 10, 2])  # all of it
    c.extend([5, 1, 0])
    c.attend(queries(c), 4, 4)


def fill(c, rows, seed):
    """Rows of random values and weights for every sequence; -> what each holds."""
    g = torch.Generator().manual_seed(seed)
    c.extend(rows)
    for x in (c.k, c.v, c.weight):
        x.copy_(torch.randn(x.shape, generator=g))
    return contents(c)


def contents(c):
    """Per sequence its rows of k, v and weight, [Hkv, rows, ..]."""
    return [[oracle.paged_rows(x.double().numpy(), c.pages[b], c.rows[b])[0] for x in (c.k, c.v, c.weight[..., None])] for b in range(c.B)]


@pytest.mark.parametrize("n_pages,rows,keep", [(10, [20, 20], [4, 4]),               # a full pool
                                               (10, [20, 20], [17, 19]),             # all pages needed again
                                               (11, [20, 20], [20, 8]),              # two pages needed, one free
                                               (11, [20, 20], [7, 3]),               # the first cut's pages serve the second
                                               (16, [20, 20, 19, 3], [16, 1, 19, 0]),
                                               (30, [20, 20], [4, 4])])              # room for all
def test_a_pool_without_room_for_what_stays_is_cut_all_the_same(calls, n_pages, rows, keep):
    c = make(B=len(rows), n_pages=n_pages)
    before = fill(c, rows, 1)
    got, kept = c.evict(keep, sinks=1, recent=2)
    stay = [min(k, r) for k, r in zip(keep, rows)]
    assert c.rows == stay == got.tolist() and c.kv_len.tolist() == stay and c.new == [0] * len(rows)
    assert kept.shape == (len(rows), c.Hkv, max(stay))
    assert sorted(c.free + [p for ps in c.pages for p in ps]) == list(range(n_pages))
    for b, after in enumerate(contents(c)):
        assert len(c.pages[b]) == -(-stay[b] // c.page) and c.table[b, :len(c.pages[b])].tolist() == c.pages[b]
        for h in range(c.Hkv):
            want = list(range(rows[b])) if stay[b] == rows[b] else oracle.paged_select(before[b][2][h, :, 0], stay[b], 1, 2)
            assert kept[b, h].tolist() == list(want) + [-1] * (max(stay) - stay[b])
            for x, y in zip(before[b], after):
                assert np.array_equal(x[h][want], y[h])


def test_an_eviction_that_fails_halfway_leaves_whole_sequences(calls, monkeypatch):
    c = make(B=2, n_pages=11)
    before = fill(c, [20, 20], 2)
    done = []

    def second_fails(*a, **kw):
        if done:
            raise u.UnigistError("no memory, say")
        done.append(1)
        return evict(*a, **kw)

    monkeypatch.setattr(u.binding, "paged_evict", second_fails)
    with pytest.raises(u.UnigistError):
        c.evict([7, 3])
    assert c.rows == [20, 3] and c.kv_len.tolist() == [20, 3] and sorted(c.free + [p for ps in c.pages for p in ps]) == list(range(11))
    for x, y in zip(before[0], contents(c)[0]):
        assert np.array_equal(x, y)


def test_too_few_rows_are_refused(calls):
    # they would be written as, and attend as, the last rows of the sequences that the tensor still reaches
    c = make()
    c.extend([3, 0, 2])
    for T in (0, 4):
        x = torch.zeros(2, T, 8, dtype=torch.bfloat16)
        with pytest.raises(u.UnigistError, match="row for each"):
            c.append(x, x)
        with pytest.raises(u.UnigistError, match="row for each"):
            c.attend(x, 4, 100)
    for T in (5, 8):  # rows behind the last sequence are left as they are
        x = torch.zeros(2, T, 8, dtype=torch.bfloat16)
        c.append(x, x)
        c.attend(x, 4, 100)
    with pytest.raises(u.UnigistError, match="row for each"):
        c.attend(x[0], 4, 100)
