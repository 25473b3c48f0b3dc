"""GPU: new rows into pages and eviction by weight, bit for bit against the oracle; a run of all of them together."""
import numpy as np
import pytest
import torch

import oracle
import paper_2509_15763_amd as u
from paper_2509_15763_amd import synth
from _paged import Paged
from _parity import TOL_LSE_BF16, max_abs, out_ok, to_np

pytestmark = pytest.mark.gpu
ALL = 1 << 22


def bits(x):
    return (x.view(torch.int16) if x.dtype == torch.bfloat16 else x).cpu().numpy()


def wide(x, scale):
    """bf16 or codes times scale, float64."""
    return oracle.dequantize_e4m3(x.cpu().numpy(), scale.cpu().numpy()) if x.dtype == torch.uint8 else to_np(x)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens,news,page,Hkv,D", [([1], [1], 16, 1, 128), ([300, 5, 77], [1, 1, 1], 16, 8, 128), ([400, 90, 30], [130, 0, 30], 7, 2, 64),
                                                  ([50, 60], [3, 41], 64, 3, 48), ([3, 9], [6, 2], 16, 2, 128), ([40, 0], [40, 0], 1, 2, 16)])
def test_append(lens, news, page, Hkv, D, e4m3):
    case = Paged(lens, news, page, Hkv, Hkv, D, e4m3=e4m3, seed=21, behind=3, missing=[(0, 1)] if lens[0] > page else ())
    g = torch.Generator().manual_seed(22)
    kn, vn = (torch.randn(case.T, Hkv, D, generator=g).mul(2.5).to(torch.bfloat16) for _ in range(2))
    want = [case.k.clone(), case.v.clone(), case.weight.clone()]
    for b, (L, n) in enumerate(zip(lens, news)):
        for i in range(n):
            j, t = L - n + i, int(case.cu[b]) + i
            pg = int(case.table[b, j // page]) if j >= 0 else -1
            if not 0 <= pg < case.k.shape[0]:
                continue
            for x, new, sc in ((want[0], kn, case.ks), (want[1], vn, case.vs)):
                x[pg, :, j % page] = torch.from_numpy(oracle.quantize_e4m3(new[t].float().numpy()[None, :, None], sc.numpy()))[0, :, 0] if e4m3 else new[t]
            want[2][pg, :, j % page] = 0
    for layout in (lambda x: x.transpose(0, 1), lambda x: x.transpose(0, 1).contiguous()):
        c = case.cuda()
        u.paged_append(c.k, c.v, c.table, c.kv_len, layout(kn.cuda()), layout(vn.cuda()), cu=c.cu, weight=c.weight, **c.scales)
        for got, x in zip((c.k, c.v, c.weight), want):
            assert np.array_equal(bits(got), bits(x))
    c = case.cuda()  # unequal layouts, no weights
    u.paged_append(c.k, c.v, c.table, c.kv_len, kn.cuda().transpose(0, 1), vn.cuda().transpose(0, 1).contiguous(), cu=c.cu, **c.scales)
    assert np.array_equal(bits(c.k), bits(want[0])) and np.array_equal(bits(c.v), bits(want[1])) and torch.equal(c.weight, case.weight.cuda())


def test_append_keeps_not_a_number_and_saturates():
    case = Paged([16], [16], 16, 1, 1, 16, e4m3=True, seed=23)
    x = torch.zeros(16, 1, 16)
    x[0], x[1], x[2] = float("nan"), 3e38, -3e38
    c = case.cuda()
    u.paged_append(c.k, c.v, c.table, c.kv_len, x.bfloat16().cuda().transpose(0, 1), x.bfloat16().cuda().transpose(0, 1), cu=c.cu, **c.scales)
    row = c.k[int(case.table[0, 0]), 0].cpu()
    assert ((row[0] & 0x7F) == 0x7F).all() and (row[1] == 0x7E).all() and (row[2] == 0xFE).all() and (row[3:] & 0x7F == 0).all()


def evict(case, weight, keep, sinks, recent, to_page=None, same_pool=False, missing_to=(), max_kv=None, max_keep=None):
    """Runs it and compares everything with the oracle; -> rows."""
    c = case.cuda()
    c.weight = weight.cuda()
    page, B, Hkv = to_page or case.page, len(case.lens), case.Hkv
    stay = [min(k, n) if 0 <= k else 0 for k, n in zip(keep, case.lens)]
    per = [-(-n // page) for n in stay]
    ids = torch.randperm(sum(per) + 1, generator=torch.Generator().manual_seed(5))
    table = torch.full((B, max(max(per), 1)), -1, dtype=torch.int32)
    at = 0
    first = case.k.shape[0] if same_pool else 0
    for b in range(B):
        table[b, :per[b]] = ids[at:at + per[b]].int() + first
        at += per[b]
    for b, pg in missing_to:
        table[b, pg] = -1
    new = sum(per) + 1
    if same_pool:
        grow = lambda x: torch.cat([x, x.new_full((new,) + x.shape[1:], 9)])
        c.k, c.v, c.weight = grow(c.k), grow(c.v), grow(c.weight)
        ko, vo, wo = c.k, c.v, c.weight
    else:
        ko, vo = (torch.full((new, Hkv, page, case.D), 9, dtype=case.k.dtype, device="cuda") for _ in range(2))
        wo = torch.full((new, Hkv, page), 9.0, device="cuda")
    before = [x.clone().cpu() for x in (ko, vo, wo)]
    src = [x.clone().cpu() for x in (c.k, c.v, c.weight)]
    max_kv, max_keep = max_kv or case.max_kv, max_keep or max(max(keep), 1)
    rows, kept = u.paged_evict(c.k, c.v, c.table, c.kv_len, c.weight, torch.tensor(keep, dtype=torch.int32).cuda(), ko, vo, table.cuda(), max_kv, max_keep,
                               sinks=sinks, recent=recent, weight_out=wo)
    rows, kept = rows.cpu().tolist(), kept.cpu().numpy()
    n_src = case.k.shape[0]
    for b in range(B):
        L = case.lens[b]
        ok = 0 <= keep[b] <= max_keep and 0 <= L <= max_kv
        ok = ok and all(0 <= int(p) < n_src for p in case.table[b, :-(-L // case.page)])
        ok = ok and all(int(p) >= 0 for p in table[b, :per[b]])
        if not ok:
            assert rows[b] == -1 and (kept[b] == -1).all()
            continue
        assert rows[b] == stay[b]
        for h in range(Hkv):
            w = np.array([float(src[2][int(case.table[b, j // case.page]), h, j % case.page]) for j in range(L)])
            want = oracle.paged_select(w, stay[b], sinks, recent)
            assert np.array_equal(kept[b, h, :stay[b]], want) and (kept[b, h, stay[b]:] == -1).all(), (b, h)
            for i, j in enumerate(want):
                for x, s in zip(before, src):
                    x[int(table[b, i // page]), h, i % page] = s[int(case.table[b, j // case.page]), h, j % case.page]
    for got, x in zip((ko, vo, wo), before):
        assert np.array_equal(bits(got), bits(x), equal_nan=got.dtype == torch.float32)
    return rows


@pytest.mark.parametrize("e4m3,D", [(False, 128), (True, 128), (False, 72), (True, 48)])
@pytest.mark.parametrize("lens,keep,page,to_page", [([300, 17, 1, 90], [64, 17, 1, 33], 16, None), ([1000, 2500], [900, 16], 64, 7), ([40, 30], [0, 50], 1, 16),
                                                    ([130, 0], [129, 5], 130, 3)])
def test_evict(lens, keep, page, to_page, e4m3, D):
    case = Paged(lens, [0] * len(lens), page, 2, 2, D, e4m3=e4m3, seed=24)
    evict(case, torch.randn(case.weight.shape).exp(), keep, 0, 0, to_page)
    evict(case, torch.randn(case.weight.shape).exp(), keep, 4, 8, to_page)
    evict(case, torch.randn(case.weight.shape), keep, 0, 3, to_page, same_pool=to_page is None)


@pytest.mark.parametrize("values", [[0.0], [0.0, -0.0, 1.0], [float("nan"), 1.0], [float("inf"), -float("inf"), 0.0, float("nan")], [1e-45, -1e-45, 3e38, -3e38],
                                    [1.0, 1.0 + 2 ** -23, 1.0 - 2 ** -24]])
def test_ties_and_odd_weights(values):
    case = Paged([700, 1500], [0, 0], 16, 2, 2, 64, seed=25)
    pick = torch.randint(len(values), case.weight.shape, generator=torch.Generator().manual_seed(6))
    w = torch.tensor(values)[pick]
    for keep, sinks, recent in (([350, 700], 0, 0), ([1, 1499], 2, 3), ([5, 9], 10, 10), ([699, 3], 0, 1 << 30), ([20, 20], 1 << 30, 0)):
        evict(case, w, keep, sinks, recent)


def test_long_sequences():
    # more rows than one pass over a workgroup's threads or memory takes
    case = Paged([40000, 70000], [0, 0], 256, 2, 1, 16, seed=26)
    evict(case, torch.randn(case.weight.shape).mul(2).exp(), [4000, 69000], 4, 64)


def test_refused_sequences_are_left_alone():
    case = Paged([100, 100, 100, 100, 100], [0] * 5, 16, 2, 2, 64, seed=27, missing=[(1, 2)])
    w = torch.rand(case.weight.shape)
    assert evict(case, w, [50, 50, -1, 70, 20], 0, 0, max_keep=60, missing_to=[(4, 1)]) == [50, -1, -1, -1, -1]
    assert evict(case, w, [50, 50, 50, 50, 50], 0, 0, max_kv=99) == [-1] * 5


def test_evict_captured_and_replayed():
    case = Paged([900, 500], [0, 0], 16, 2, 2, 64, seed=28)
    c = case.cuda()
    ko, vo = (torch.zeros(60, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wo = torch.zeros(60, 2, 16, device="cuda")
    to = torch.arange(60, dtype=torch.int32, device="cuda").view(2, 30)
    keep = torch.tensor([300, 400], dtype=torch.int32, device="cuda")

    def step():
        return u.paged_evict(c.k, c.v, c.table, c.kv_len, c.weight, keep, ko, vo, to, 900, 400, sinks=2, recent=5, weight_out=wo)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        rows, kept = step()
    for n in range(3):
        c.weight.copy_(torch.rand(c.weight.shape, generator=torch.Generator().manual_seed(n)))
        keep.copy_(torch.tensor([300 - n, 400 - 50 * n], dtype=torch.int32))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (rows, kept, wo, ko.view(torch.int16))]
        r2, k2 = step()
        torch.cuda.synchronize()
        for a, b in zip(got, (r2, k2, wo, ko.view(torch.int16))):
            assert torch.equal(a, b)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_a_run_of_all_of_them(e4m3):
    """Two prompts in chunks, an eviction, tokens on top: every call against the oracle over the rows that should be there."""
    Hq, Hkv, D, page, cols, n_pages = 8, 2, 128, 16, 40, 120
    g = torch.Generator().manual_seed(30)
    ks, vs = synth.e4m3_scales(Hkv, 3) if e4m3 else (None, None)
    dtype = torch.uint8 if e4m3 else torch.bfloat16
    k, v = (torch.full((n_pages, Hkv, page, D), 0x7F if e4m3 else float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    weight = torch.full((n_pages, Hkv, page), float("nan"), device="cuda")
    scales = dict(k_scale=None if ks is None else ks.cuda(), v_scale=None if vs is None else vs.cuda())
    table = torch.full((2, cols), -1, dtype=torch.int32)
    free = torch.randperm(n_pages, generator=g).tolist()
    rows = [[np.zeros((Hkv, 0, D)), np.zeros((Hkv, 0, D)), np.zeros((Hkv, 0))] for _ in range(2)]  # what the oracle has: k, v, weight

    def step(news, weigh, decay):
        cu = [0, news[0], sum(news)]
        T = cu[-1]
        q, kn, vn = (torch.randn(T, H, D, generator=g).to(torch.bfloat16) for H in (Hq, Hkv, Hkv))
        lens = [rows[b][0].shape[1] + news[b] for b in range(2)]
        for b in range(2):
            for pg in range(-(-lens[b] // page)):
                if table[b, pg] < 0:
                    table[b, pg] = free.pop()
        t, cud, kv = table.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
        u.paged_append(k, v, t, kv, kn.cuda().transpose(0, 1), vn.cuda().transpose(0, 1), cu=cud, weight=weight, **scales)
        out, lse = u.paged_attn(q.cuda().transpose(0, 1), k, v, t, kv, 4, ALL, cu=cud, max_new=max(news), max_kv=max(lens), weight=weight, weigh=weigh,
                                decay=decay, **scales)
        for b in range(2):
            new = slice(cu[b], cu[b + 1])
            for i, (x, sc) in enumerate(((kn, ks), (vn, vs))):
                x = x[new].transpose(0, 1)
                x = oracle.dequantize_e4m3(oracle.quantize_e4m3(x[None].float().numpy(), sc.numpy()), sc.numpy())[0] if e4m3 else x.double().numpy()
                rows[b][i] = np.concatenate([rows[b][i], x], 1)
            rows[b][2] = np.concatenate([rows[b][2], np.zeros((Hkv, news[b]))], 1)
            L = lens[b]
            pool = [x.transpose(1, 0, 2)[:, :, None] for x in rows[b][:2]]  # one row a page
            o, l, added = oracle.paged_attn(q[new].transpose(0, 1).double().numpy(), pool[0], pool[1], [list(range(L))], [L], [0, news[b]], 4, ALL, weigh=weigh)
            assert out_ok(to_np(out[:, new]), o) and max_abs(to_np(lse[:, new]), l) <= TOL_LSE_BF16
            rows[b][2] = decay * rows[b][2] + added[0]
            got = np.stack([weight[int(table[b, j // page]), :, j % page].cpu().double().numpy() for j in range(L)], 1)
            assert (np.abs(got - rows[b][2]) <= 3e-4 * rows[b][2] + 1e-9).all()
            rows[b][2] = got  # the selection below is between the numbers that are there
        return lens

    step([200, 130], 1, 1.0)
    lens = step([150, 3], 8, 0.5)
    keep = [120, 60]
    to = torch.full((2, cols), -1, dtype=torch.int32)
    for b in range(2):
        for pg in range(-(-keep[b] // page)):
            to[b, pg] = free.pop()
    got, kept = u.paged_evict(k, v, table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), weight, torch.tensor(keep, dtype=torch.int32).cuda(), k, v, to.cuda(),
                              max(lens), max(keep), sinks=4, recent=16, weight_out=weight)
    assert got.cpu().tolist() == keep
    for b in range(2):
        free.extend(int(p) for p in table[b] if p >= 0)
        sel = np.stack([oracle.paged_select(rows[b][2][h], keep[b], 4, 16) for h in range(Hkv)])
        assert np.array_equal(kept[b, :, :keep[b]].cpu().numpy(), sel)
        rows[b] = [np.stack([x[h][sel[h]] for h in range(Hkv)]) for x in rows[b]]
    table.copy_(to)
    for news in ([1, 1], [5, 1], [1, 40]):
        step(news, 1, 1.0)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_the_cache_class(e4m3):
    """Prompts in chunks, tokens, an eviction of one of two sequences, more tokens, a sequence that leaves and one that comes."""
    Hq, Hkv, D, page = 8, 2, 64, 16
    ks, vs = synth.e4m3_scales(Hkv, 4, device="cuda") if e4m3 else (None, None)
    cache = u.PagedKVCache(2, Hkv, 64, page, 400, D, dtype=torch.uint8 if e4m3 else torch.bfloat16, k_scale=ks, v_scale=vs, weights=True)
    g = torch.Generator().manual_seed(31)
    values = lambda: tuple(wide(x, s) for x, s in ((cache.k, ks), (cache.v, vs)))

    def step(n, weigh=0, **kw):
        cache.extend(n)
        q, kn, vn = (torch.randn(sum(n), H, D, generator=g).to(torch.bfloat16).cuda().transpose(0, 1) for H in (Hq, Hkv, Hkv))
        cache.append(kn, vn)
        out, lse = cache.attend(q, 4, ALL, weigh=weigh, **kw)
        k, v = values()
        o, l, _ = oracle.paged_attn(to_np(q), k, v, cache.pages, cache.rows, cache.cu.cpu().tolist(), 4, ALL)
        assert out_ok(to_np(out), o) and max_abs(to_np(lse), l) <= TOL_LSE_BF16
        for b, m in enumerate(n):  # the newest row is what was appended
            if m and not e4m3:
                r = cache.rows[b] - 1
                assert torch.equal(cache.k[cache.pages[b][r // page], :, r % page], kn[:, sum(n[:b + 1]) - 1])

    step([130, 60])
    step([50, 1], weigh=16)
    step([1, 1], weigh=1)
    k, v = values()
    before, _ = oracle.paged_rows(k, cache.pages[0], cache.rows[0])
    w = np.stack([[float(cache.weight[cache.pages[0][j // page], h, j % page]) for j in range(cache.rows[0])] for h in range(Hkv)])
    free = len(cache.free)
    rows, kept = cache.evict([70, 1000], sinks=2, recent=8)
    assert rows.cpu().tolist() == [70, 62] and cache.rows == [70, 62] and len(cache.free) == free + 12 - 5
    assert kept[1, :, :62].cpu().tolist() == [list(range(62))] * Hkv
    after, _ = oracle.paged_rows(values()[0], cache.pages[0], 70)
    for h in range(Hkv):
        sel = oracle.paged_select(w[h], 70, 2, 8)
        assert kept[0, h, :70].cpu().tolist() == sel.tolist() and np.array_equal(after[h], before[h][sel])
    step([1, 1], weigh=1)
    step([3, 20], weigh=4, decay=0.5)
    cache.release(0)
    step([40, 1], weigh=1)
    assert sorted(cache.free + [p for ps in cache.pages for p in ps]) == list(range(64))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("n_pages,keep", [(21, [90, 33, 20]), (21, [145, 99, 60]), (22, [60, 100, 16]), (40, [90, 33, 20])],
                         ids=["full", "full, all pages needed again", "a cut's pages serve the next", "room"])
def test_the_cache_class_evicts_from_a_full_pool(n_pages, keep, e4m3):
    Hkv, D, page, rows = 2, 64, 16, [150, 100, 64]
    ks, vs = synth.e4m3_scales(Hkv, 4, device="cuda") if e4m3 else (None, None)
    cache = u.PagedKVCache(3, Hkv, n_pages, page, 200, D, dtype=torch.uint8 if e4m3 else torch.bfloat16, k_scale=ks, v_scale=vs, weights=True)
    g = torch.Generator().manual_seed(33)
    for n in ([150, 80, 64], [0, 20, 0]):
        cache.extend(n)
        kn, vn = (torch.randn(sum(n), Hkv, D, generator=g).to(torch.bfloat16).cuda().transpose(0, 1) for _ in range(2))
        cache.append(kn, vn)
    assert len(cache.free) == n_pages - 21
    cache.weight.copy_(torch.randn(cache.weight.shape, generator=g).exp())
    hold = lambda: [[oracle.paged_rows(x.cpu().numpy(), cache.pages[b], cache.rows[b])[0] for x in (cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.weight)]
                    for b in range(3)]
    before = hold()
    got, kept = cache.evict(keep, sinks=2, recent=9)
    assert got.cpu().tolist() == [min(k, r) for k, r in zip(keep, rows)] == cache.rows
    for b, after in enumerate(hold()):
        for h in range(Hkv):
            sel = oracle.paged_select(before[b][2][h].astype(np.float64), cache.rows[b], 2, 9)
            assert kept[b, h].cpu().tolist() == sel.tolist() + [-1] * (max(cache.rows) - cache.rows[b])
            for x, y in zip(before[b], after):
                assert np.array_equal(x[h][sel], y[h])
    assert sorted(cache.free + [p for ps in cache.pages for p in ps]) == list(range(n_pages))
    cache.extend([1, 1, 1])
    q, kn, vn = (torch.randn(3, H, D, generator=g).to(torch.bfloat16).cuda().transpose(0, 1) for H in (8, Hkv, Hkv))
    cache.append(kn, vn)
    out, lse = cache.attend(q, 4, ALL)
    k, v = (wide(x, s) for x, s in ((cache.k, ks), (cache.v, vs)))
    o, l, _ = oracle.paged_attn(to_np(q), k, v, cache.pages, cache.rows, cache.cu.cpu().tolist(), 4, ALL)
    assert out_ok(to_np(out), o) and max_abs(to_np(lse), l) <= TOL_LSE_BF16


def test_append_of_as_many_rows_as_four_billion_threads():
    # 16 lanes a row: 2^28 rows are 2^32 threads, more than one axis of a launch takes
    T, Hkv, D, page = 1 << 22, 64, 8, 4096
    new = torch.randint(-32768, 32767, (Hkv, T, D), dtype=torch.int16, device="cuda").view(torch.bfloat16)
    k, v = (torch.zeros(T // page, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.arange(T // page, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    length, cu = torch.tensor([T], dtype=torch.int32, device="cuda"), torch.tensor([0, T], dtype=torch.int32, device="cuda")
    u.paged_append(k, v, table, length, new, new, cu=cu)
    for x in (k, v):
        for p in (0, 1, 77, T // page - 2, T // page - 1):
            assert torch.equal(x[int(table[0, p])].view(torch.int16), new[:, p * page:(p + 1) * page].view(torch.int16))
    assert torch.equal(k.view(torch.int16), v.view(torch.int16))
    rows = torch.tensor([0, 1, T // 2, T - 1], device="cuda")
    for h in range(Hkv):
        at = table[0].long()[rows // page]
        assert torch.equal(k[at, h, rows % page].view(torch.int16), new[h, rows].view(torch.int16))


def test_evict_captured_and_replayed_with_other_tables():
    # the pages move between the replays, on both sides
    case = Paged([900, 500], [0, 0], 16, 2, 2, 64, seed=32)
    c = case.cuda()
    pool = c.k.shape[0]
    ko, vo = (torch.zeros(60, 2, 16, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    wo = torch.zeros(60, 2, 16, device="cuda")
    to = torch.arange(60, dtype=torch.int32, device="cuda").view(2, 30)
    keep = torch.tensor([300, 400], dtype=torch.int32, device="cuda")
    first = [x.clone() for x in (c.k, c.v, c.weight, c.table)]

    def step():
        return u.paged_evict(c.k, c.v, c.table, c.kv_len, c.weight, keep, ko, vo, to, 900, 400, sinks=2, recent=5, weight_out=wo)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        rows, kept = step()
    for x in (ko, vo, wo):
        x.zero_()
    r2, k2 = step()
    want = [x.clone() for x in (ko.view(torch.int16), vo.view(torch.int16), wo)]
    for n in range(3):
        gen = torch.Generator().manual_seed(n)
        move, out = torch.randperm(pool, generator=gen).cuda(), torch.randperm(60, generator=gen).cuda()
        for x, y in zip((c.k, c.v, c.weight), first):
            x[move] = y
        c.table.copy_(torch.where(first[3] >= 0, move[first[3].clamp(min=0).long()].int(), first[3]))
        to.copy_(out.int().view(2, 30))
        for x in (ko, vo, wo):
            x.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(rows, r2) and torch.equal(kept, k2)
        for x, y in zip((ko.view(torch.int16), vo.view(torch.int16), wo), want):
            assert torch.equal(x[out], y)
