"""GPU parity of attention over a paged cache, and of the weights it adds up, against the fp64 oracle.

Tolerances: out and lse as everywhere (flat 1e-2 with the stored result's half step on top from |out| = 2; 1e-4).  A weight is a sum
of exp(s - lse) with s and lse in fp32: an error of lse up to the 1e-4 it is held to and one of s of the same origin change
each term by at most 2e-4 of itself, and decay * weight is one rounded product of 2^-24."""
import numpy as np
import pytest
import torch

import oracle
import paper_2509_15763_amd as u
from paper_2509_15763_amd import synth
from _paged import Paged
from _parity import TOL_LSE_BF16, TOL_OUT_BF16, max_abs, out_ok, to_np

pytestmark = pytest.mark.gpu
ALL = 1 << 22  # a window that holds everything


def run(c, r, W, sinks=0, units=False, **kw):
    return u.paged_attn(c.q.transpose(0, 1), c.k, c.v, c.table, c.kv_len, r, W, cu=c.cu, max_new=c.max_new, max_kv=c.max_kv, sinks=sinks,
                        window_mode=int(units), **c.scales, **kw)


def check(case, r, W, weigh=0, decay=1.0, **mask):
    c = case.cuda()
    more = dict(weight=c.weight, weigh=weigh, decay=decay) if weigh else {}
    out, lse = run(c, r, W, **mask, **more)
    torch.cuda.synchronize()
    wo, wl, added = case.want(r, W, weigh=weigh, **mask)
    n = int(case.cu[-1])
    out, lse = to_np(out)[:, :n], to_np(lse)[:, :n]
    wo, wl = wo[:, :n], wl[:, :n]
    assert np.array_equal(np.isinf(lse), np.isinf(wl)) and np.array_equal(np.isnan(out), np.isnan(wo))
    keep = ~np.isnan(wl)
    assert np.array_equal(keep, ~np.isnan(lse))
    out, lse, wo, wl = out[keep], lse[keep], wo[keep], wl[keep]
    none = np.isinf(wl)
    assert (out[none] == 0).all() and (lse[none] < 0).all()
    eo, el = max_abs(out, wo), max_abs(lse[~none], wl[~none])
    print(f"  out {eo:.3e} lse {el:.3e}", flush=True)
    assert out_ok(out, wo) and el <= TOL_LSE_BF16
    if weigh:
        got, want = to_np(c.weight), case.want_weight(added, decay)
        assert (np.abs(got - want) <= 2e-4 * want + 1e-9).all(), float(np.abs(got - want).max())
    return out, lse


# lens, news, page, Hq, Hkv, D
CASES = {
    "one key": ([1], [1], 16, 4, 1, 128),
    "decode": ([300, 1, 77, 1000], [1, 1, 1, 1], 16, 8, 2, 128),
    "decode, page of one row": ([40, 13], [1, 1], 1, 4, 2, 64),
    "decode, odd page": ([200, 333], [1, 1], 7, 4, 4, 64),
    "decode, slab": ([130, 259], [1, 1], 259, 8, 1, 128),
    "decode long": ([5000], [1], 64, 8, 2, 128),
    "decode, group of 32": ([500, 90], [1, 1], 32, 32, 1, 128),
    "decode, group of 7": ([500, 90], [1, 1], 32, 14, 2, 96),
    "decode, group of 48": ([300, 150], [1, 1], 16, 48, 1, 64),
    "decode, D 8": ([100, 40], [1, 1], 16, 4, 2, 8),
    "drafts": ([700, 8, 64, 129], [8, 3, 5, 2], 32, 8, 2, 128),
    "drafts, D 64": ([1500, 900], [4, 7], 16, 4, 1, 64),
    "drafts of 16, groups of 4": ([900, 16, 17], [16, 16, 9], 16, 8, 2, 128),
    "chunk": ([400], [400], 64, 4, 1, 128),
    "chunk at the end": ([900, 500], [130, 257], 32, 4, 2, 128),
    "chunk, no groups": ([333], [200], 16, 2, 2, 64),
    "chunk, group of 3, D 96": ([301, 150], [150, 77], 24, 6, 2, 96),
    "chunk, group of 5": ([301], [130], 16, 5, 1, 80),
    "mixed": ([600, 1, 350, 90], [300, 1, 1, 33], 16, 8, 2, 128),
    "no new rows, no rows": ([100, 50, 0, 30], [3, 0, 0, 30], 16, 4, 2, 128),
    "more new rows than rows": ([2, 5], [6, 1], 16, 4, 2, 64),
}


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("name", CASES)
def test_causal(name, e4m3):
    lens, news, page, Hq, Hkv, D = CASES[name]
    if e4m3 and D % 16:
        D = 16
    check(Paged(lens, news, page, Hq, Hkv, D, e4m3=e4m3, seed=3), 4, ALL)


MASKS = [(4, 16, dict()), (2, 100, dict(sinks=5)), (1, 1, dict()), (3, 4, dict(sinks=7, units=True)), (1 << 30, 33, dict()),
         (8, 1 << 30, dict(units=True)), (5, 2, dict(sinks=1 << 30))]


@pytest.mark.parametrize("r,W,mask", MASKS)
@pytest.mark.parametrize("name", ["decode", "decode, odd page", "drafts", "chunk at the end", "chunk, group of 3, D 96", "mixed",
                                  "more new rows than rows"])
def test_gist_masks(name, r, W, mask):
    check(Paged(*CASES[name], seed=4), r, W, **mask)


@pytest.mark.parametrize("name", ["decode", "drafts", "mixed"])
def test_gist_mask_over_codes(name):
    check(Paged(*CASES[name], e4m3=True, seed=5), 4, 50, sinks=3)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("news", [[1, 1, 1], [5, 3, 2], [200, 70, 1]], ids=["decode", "drafts", "chunk"])
def test_pages_that_are_not_there(news, e4m3):
    # the first, one in the middle, the last (which holds the new rows' own keys), all of a sequence
    missing = [(0, 0), (0, 3), (1, 18), (2, 0), (2, 1), (2, 2), (2, 3), (2, 4)]
    case = Paged([400, 300, 70], news, 16, 8, 2, 128, e4m3=e4m3, seed=6, missing=missing)
    check(case, 4, ALL)
    check(case, 4, 40, sinks=2)


@pytest.mark.parametrize("last", [250, 256])  # 250: the places behind them, which become rows in use, hold NaN
@pytest.mark.parametrize("cols", [None, 50])
def test_a_table_shorter_or_longer_than_the_rows(cols, last):
    case = Paged([100, last], [1, 40], 16, 4, 2, 64, seed=7, cols=cols)
    if cols is None:  # lengths beyond what the table has pages for: those rows are not there
        case.lens = [100, 300]
        case.kv_len = torch.tensor(case.lens, dtype=torch.int32)
    check(case, 4, ALL)


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens,news", [([130], [4]), ([200, 90], [130, 8])], ids=["drafts", "chunk"])
def test_what_later_rows_hold_does_not_reach_earlier_ones(lens, news, e4m3, what):
    # the last new row of each sequence is not finite: every row before it is as if it were not there
    if e4m3 and what == what:
        pytest.skip("E4M3 has no infinities")
    case = Paged(lens, news, 16, 4, 2, 128, e4m3=e4m3, seed=8)
    clean = run(case.cuda(), 4, ALL)
    for b, L in enumerate(lens):
        pg, slot = int(case.table[b, (L - 1) // 16]), (L - 1) % 16
        case.k[pg, :, slot] = 0x7F if e4m3 else what
        case.v[pg, :, slot] = 0xFF if e4m3 else what
    out, lse = run(case.cuda(), 4, ALL)
    last = [int(x) - 1 for x in case.cu[1:]]
    rows = [t for t in range(case.T) if t not in last]
    assert max_abs(to_np(out[:, rows]), to_np(clean[0][:, rows])) <= 2 * TOL_OUT_BF16
    assert max_abs(to_np(lse[:, rows]), to_np(clean[1][:, rows])) <= 2 * TOL_LSE_BF16


def test_what_lies_outside_the_window_does_not_reach_it():
    case = Paged([400, 300], [1, 60], 16, 4, 2, 128, seed=9)
    r, W = 4, 50
    clean = run(case.cuda(), r, W)
    for b, L in enumerate(case.lens):  # a raw row that leaves the window of the later new rows and one far outside it
        first = L - case.news[b]
        for j in (first - W + 1 + 8, 11):
            while (j + 1) % (r + 1) == 0:
                j += 1
            pg = int(case.table[b, j // 16])
            case.v[pg, :, j % 16] = float("nan")
            case.k[pg, :, j % 16] = float("inf")
    out, _ = run(case.cuda(), r, W)
    hit = []
    for b, L in enumerate(case.lens):
        first = L - case.news[b]
        j = first - W + 1 + 8
        while (j + 1) % (r + 1) == 0:
            j += 1
        hit += [int(case.cu[b]) + i for i in range(case.news[b]) if first + i - j < W]
    rows = [t for t in range(case.T) if t not in hit]
    assert rows and max_abs(to_np(out[:, rows]), to_np(clean[0][:, rows])) <= 2 * TOL_OUT_BF16
    assert torch.isnan(out[:, hit].float()).all()


@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_values_that_are_not_finite_far_apart(e4m3, D):
    # one element of V at both ends of the window, of gists left of it and of new rows: it reaches the rows that see it and no other
    # element of them, however many steps of a walk, slices and sequences lie between
    r, W, at, what = 4, 1500, 3, float("nan") if e4m3 else float("inf")
    case = Paged([3000, 2000, 900], [700, 300, 900], 64, 4, 2, D, e4m3=e4m3, seed=21)
    clean, clean_lse = run(case.cuda(), r, W)
    seen = torch.zeros(case.T, dtype=torch.bool)
    for b, (L, n) in enumerate(zip(case.lens, case.news)):
        for j in (L - n - W + 8, L - n - W + 40, 4, L - 43, L - 3):
            if j < 0 or (j == 4 and b != 1):
                continue
            case.v[int(case.table[b, j // 64]), :, j % 64, at] = 0x7F if e4m3 else what
            for i in range(n):
                p = L - n + i
                seen[int(case.cu[b]) + i] |= j <= p and (p - j < W or (j + 1) % (r + 1) == 0)
    assert 0 < int(seen.sum()) < case.T
    out, lse = run(case.cuda(), r, W)
    assert torch.equal(lse, clean_lse) or max_abs(to_np(lse), to_np(clean_lse)) <= 2 * TOL_LSE_BF16
    got = out[..., at].float().cpu()
    assert (torch.isnan(got) if e4m3 else got == what)[:, seen].all()
    out[:, seen.to(out.device), at] = clean[:, seen.to(out.device), at]
    assert max_abs(to_np(out), to_np(clean)) <= 2 * TOL_OUT_BF16


@pytest.mark.parametrize("weigh,decay", [(1, 1.0), (3, 0.0), (100, 0.5), (1 << 30, 1.0)])
@pytest.mark.parametrize("name", ["one key", "decode", "decode, odd page", "decode, group of 32", "decode, group of 48", "drafts", "drafts, D 64",
                                  "chunk", "chunk, group of 3, D 96", "chunk at the end", "mixed", "no new rows, no rows", "more new rows than rows"])
def test_weights(name, weigh, decay):
    case = Paged(*CASES[name], seed=10)
    if decay == 0:
        case.weight.fill_(float("nan"))  # overwritten where there are rows of a sequence with new ones
        c = case.cuda()
        run(c, 4, ALL, weight=c.weight, weigh=weigh, decay=decay)
        want = case.want_weight(case.want(4, ALL, weigh=weigh)[2], decay)
        got = to_np(c.weight)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        assert (np.abs(got[ok] - want[ok]) <= 2e-4 * want[ok] + 1e-9).all()
        return
    check(case, 4, ALL, weigh=weigh, decay=decay)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("name", ["decode", "drafts", "mixed"])
def test_weights_under_a_mask_and_missing_pages(name, e4m3):
    lens, news, page, Hq, Hkv, D = CASES[name]
    check(Paged(lens, news, page, Hq, Hkv, D, e4m3=e4m3, seed=11, missing=[(0, 0), (0, 2)]), 4, 20, weigh=2, decay=0.5, sinks=3)


def test_weights_of_one_row_sum_to_one():
    # softmax weights of a row sum to 1: over the pool, the number of (row, head) pairs counted; fp32 sums of n terms of 2^-24 each
    case = Paged([3000, 700], [70, 5], 64, 8, 2, 128, seed=12)
    c = case.cuda()
    run(c, 4, ALL, weight=c.weight.zero_(), weigh=64, decay=1.0)
    assert abs(float(c.weight.double().sum()) - 8 * (64 + 5)) <= 8 * 69 * 2e-4


def test_rows_behind_the_last_sequence_and_other_layouts():
    case = Paged([300, 90, 40], [130, 1, 3], 16, 8, 2, 128, seed=13, behind=5)
    c = case.cuda()
    n = int(case.cu[-1])
    want, wl = run(c, 4, ALL)[0][:, :n], run(c, 4, ALL)[1][:, :n]
    B, T, Hq, D = 3, case.T, 8, 128
    cache = u.binding._paged_cache(c.k, c.v, c.table, None, None, None)
    import ctypes as C
    mask = (130, 300, 4, ALL, 0, 0)
    need = u.unigist_paged_attn_workspace(C.byref(cache), B, Hq, T, *mask, 0)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    # q, k and v side by side as one projection leaves them; heads in front; a slice of a longer buffer
    fused = torch.randn(T, Hq + 4, D, device="cuda").bfloat16()
    fused[:, :Hq] = c.q
    for q in (fused[:, :Hq].transpose(0, 1), c.q.transpose(0, 1).contiguous()):
        out = torch.full((T, Hq + 4, D) if q.stride(1) != D else (Hq, T, D), 7.0, dtype=torch.bfloat16, device="cuda")
        view = out[:, :Hq].transpose(0, 1) if q.stride(1) != D else out
        assert view.stride() == q.stride()
        lse = torch.full((Hq, T), 7.0, device="cuda")
        st = u.unigist_paged_attn(C.byref(cache), q.data_ptr(), view.data_ptr(), lse.data_ptr(), B, Hq, T, c.cu.data_ptr(), c.kv_len.data_ptr(),
                                  *mask, q.stride(0), q.stride(1), 0, 1.0, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert st == 0
        assert torch.equal(view[:, :n], want) and torch.equal(lse[:, :n], wl)
        assert (view[:, n:] == 7).all() and (lse[:, n:] == 7).all()
        if q.stride(1) != D:
            assert (out[:, Hq:] == 7).all()
    o2, l2 = u.paged_attn(fused[:, :Hq].transpose(0, 1), c.k, c.v, c.table, c.kv_len, 4, ALL, cu=c.cu)  # loosest bounds
    assert max_abs(to_np(o2[:, :n]), to_np(want)) <= TOL_OUT_BF16 and max_abs(to_np(l2[:, :n]), to_np(wl)) <= TOL_LSE_BF16
    odd = torch.empty(T * Hq * D + 1, device="cuda", dtype=torch.bfloat16)[1:].view(T, Hq, D).copy_(c.q)  # not 16-byte aligned: copied
    o3, _ = u.paged_attn(odd.transpose(0, 1), c.k, c.v, c.table, c.kv_len, 4, ALL, cu=c.cu, max_new=130, max_kv=300)
    assert torch.equal(o3[:, :n], want)


def test_broadcast_heads_and_no_rows():
    case = Paged([50, 60], [1, 1], 16, 4, 2, 64, seed=14).cuda()
    one = case.q[:, :1].transpose(0, 1)
    a, _ = u.paged_attn(one.expand(4, 2, 64), case.k, case.v, case.table, case.kv_len, 4, ALL)
    b, _ = u.paged_attn(one.repeat(4, 1, 1), case.k, case.v, case.table, case.kv_len, 4, ALL)
    assert torch.equal(a, b)
    out, lse = u.paged_attn(case.q[:0].transpose(0, 1), case.k, case.v, case.table, case.kv_len, 4, ALL, cu=torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert out.shape == (4, 0, 64) and lse.shape == (4, 0)


def test_agrees_with_the_other_paths_of_the_library():
    # the same rows in one piece: training kernel, decode, chunk-wise prefill
    L, page, Hq, Hkv, D, r, W = 1500, 16, 8, 2, 128, 4, 200
    q, k, v, _ = synth.attn_inputs(1, Hq, Hkv, L, D, seed=15, device="cuda")
    full, flse = u.attn_fwd(q, k, v, r, W)
    n_pages = -(-L // page)
    perm = torch.randperm(n_pages, generator=torch.Generator().manual_seed(1)).cuda()
    pad = n_pages * page - L

    def pages(x):
        x = torch.nn.functional.pad(x[0], (0, 0, 0, pad)).view(Hkv, n_pages, page, D).transpose(0, 1)
        return torch.empty_like(x, memory_format=torch.contiguous_format).index_copy_(0, perm, x.contiguous())

    kp, vp, table = pages(k), pages(v), perm.int()[None].contiguous()
    kv = torch.tensor([L], dtype=torch.int32, device="cuda")
    for n in (1, 4, 300, L):
        cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
        out, lse = u.paged_attn(q[0, :, L - n:], kp, vp, table, kv, r, W, cu=cu, max_new=n, max_kv=L)
        assert max_abs(to_np(out), to_np(full[0, :, L - n:])) <= TOL_OUT_BF16 and max_abs(to_np(lse), to_np(flse[0, :, L - n:])) <= TOL_LSE_BF16
    d, dl = u.decode(q[:, :, -1].contiguous(), k, v)
    out, lse = u.paged_attn(q[0, :, L - 1:], kp, vp, table, kv, r, ALL)
    assert max_abs(to_np(out[:, 0]), to_np(d[0])) <= TOL_OUT_BF16 and max_abs(to_np(lse[:, 0]), to_np(dl[0])) <= TOL_LSE_BF16
    # a slab is a pool of one page a sequence
    out2, lse2 = u.paged_attn(q[0, :, L - 1:], k, v, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), kv, r, ALL)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("news", [[1, 1], [3, 40], [300, 1]], ids=["decode", "drafts", "chunk"])
def test_captured_and_replayed(news):
    case = Paged([900, 500], news, 16, 8, 2, 128, seed=16)
    c = case.cuda()
    need = 64 << 20
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    start = c.weight.clone()

    def step():
        return run(c, 4, ALL, weight=c.weight, weigh=2, decay=0.5, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()  # two graphs share the workspace
    with torch.cuda.graph(g, stream=side):
        out, lse = step()
    with torch.cuda.graph(g2, stream=side):
        out2, _ = step()
    for n in range(3):
        c.q.copy_(torch.randn(c.q.shape, generator=torch.Generator().manual_seed(n)))
        c.kv_len.copy_(torch.tensor([900 - 37 * n, 500 - n], dtype=torch.int32))  # lengths change between replays
        c.weight.copy_(start)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got, gw = (out.clone(), lse.clone()), c.weight.clone()
        c.weight.copy_(start)
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(gw, c.weight), n
        g2.replay()
        torch.cuda.synchronize()
        assert torch.equal(out2, want[0])


def test_pools_beyond_four_gigabytes():
    # the pages in use lie at the end of a pool of 5 GB (each of k and v)
    case = Paged([700, 300], [1, 70], 64, 8, 2, 128, seed=17)
    c = case.cuda()
    want, wl = run(c, 4, ALL, weight=c.weight, weigh=3, decay=0.0)
    big = 5 * (1 << 30) // (2 * 64 * 128 * 2)
    n = case.k.shape[0]
    d = case.cuda()
    d.k, d.v = (torch.empty(big, 2, 64, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    d.k[big - n:], d.v[big - n:] = case.k.cuda(), case.v.cuda()
    d.weight = torch.zeros(big, 2, 64, device="cuda")
    d.table = torch.where(d.table >= 0, d.table + (big - n), d.table)
    out, lse = run(d, 4, ALL, weight=d.weight, weigh=3, decay=0.0)
    assert torch.equal(out, want) and torch.equal(lse, wl)
    used = ~torch.isnan(c.k[..., 0].float())
    assert torch.equal(d.weight[big - n:][used], c.weight[used])


def test_results_repeat_bit_for_bit_and_on_other_streams():
    case = Paged([2000, 900, 33], [200, 1, 5], 32, 8, 2, 128, seed=18)
    c = case.cuda()
    first = run(c, 4, 300, weight=c.weight, weigh=8, decay=0.0)
    w = c.weight.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(c, 4, 300, weight=c.weight, weigh=8, decay=0.0)
    torch.cuda.synchronize()
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1]) and torch.equal(w, c.weight)


def test_a_query_that_is_no_number_concerns_what_it_sees():
    # new row 1 of 3 (decode) and of 200 (chunk) is NaN: its own outputs, and the weights of the rows up to its position
    for news in ([3], [200]):
        case = Paged([400], news, 16, 4, 2, 128, seed=19)
        clean = case.cuda()
        want, _ = run(clean, 4, ALL, weight=clean.weight, weigh=1 << 20, decay=0.0)
        case.q[1, 0] = float("nan")  # one of the two heads of kv head 0
        c = case.cuda()
        out, lse = run(c, 4, ALL, weight=c.weight, weigh=1 << 20, decay=0.0)
        assert torch.isnan(out[0, 1].float()).all() and torch.isnan(lse[0, 1])
        out[0, 1], want[0, 1] = 0, 0
        assert torch.equal(out, want)
        p = 400 - news[0] + 1
        for j in range(400):
            pg, slot = int(case.table[0, j // 16]), j % 16
            assert bool(torch.isnan(c.weight[pg, 0, slot])) == (j <= p)
            assert abs(float(c.weight[pg, 1, slot]) - float(clean.weight[pg, 1, slot])) <= 1e-6


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_many_tiles_agree_with_the_training_kernel(e4m3):
    # more tiles than CUs: every row of a sequence against the forward kernel, and the weights against those of a slice of its rows
    L, page, Hq, Hkv, D, r, W = 9000, 64, 8, 2, 128, 4, 700
    q, k, v, _ = synth.attn_inputs(1, Hq, Hkv, L, D, seed=20, device="cuda")
    scales = {}
    if e4m3:
        ks, vs = synth.e4m3_scales(Hkv, 2, device="cuda")
        k8, v8 = u.quantize_e4m3(k, ks), u.quantize_e4m3(v, vs)
        wide = lambda c, s: (c.view(torch.float8_e4m3fn).float() * s[:, None, None]).to(torch.bfloat16)
        k, v, scales = wide(k8, ks), wide(v8, vs), dict(k_scale=ks, v_scale=vs)  # rounds where code * scale is no bf16 value
    n_pages = -(-L // page)

    def pages(x):
        return torch.nn.functional.pad(x[0], (0, 0, 0, n_pages * page - L)).view(Hkv, n_pages, page, D).transpose(0, 1).contiguous()

    kp, vp = (pages(k8), pages(v8)) if e4m3 else (pages(k), pages(v))
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda")[None]
    kv, cu = torch.tensor([L], dtype=torch.int32, device="cuda"), torch.tensor([0, L], dtype=torch.int32, device="cuda")
    for mask in (dict(), dict(sinks=5), dict(sinks=3, window_mode=1)):
        WW = 40 if mask.get("window_mode") else W
        full, flse = u.attn_fwd(q, k, v, r, WW, **mask)
        weight = torch.zeros(n_pages, Hkv, page, device="cuda")
        out, lse = u.paged_attn(q[0], kp, vp, table, kv, r, WW, cu=cu, max_new=L, max_kv=L, weight=weight, weigh=300, **mask, **scales)
        # codes: the forward reads k and v rounded to bf16, 2^-9 of each product's size on either side
        assert max_abs(to_np(out), to_np(full[0])) <= (3 if e4m3 else 1) * TOL_OUT_BF16
        assert max_abs(to_np(lse), to_np(flse[0])) <= (1e-2 if e4m3 else TOL_LSE_BF16)
        assert abs(float(weight.double().sum()) - 300 * Hq) <= 300 * Hq * 2e-4
        w2 = torch.zeros_like(weight)
        c2 = torch.tensor([0, 300], dtype=torch.int32, device="cuda")
        u.paged_attn(q[0, :, L - 300:], kp, vp, table, kv, r, WW, cu=c2, max_new=300, max_kv=L, weight=w2, weigh=300, **mask, **scales)
        assert float((weight - w2).abs().max()) <= 2e-4 * float(weight.max())


def test_hundreds_of_sequences():
    # more sequences than a wave has lanes: tokens, drafts and chunks side by side
    lens, news = [], []
    for b in range(150):
        news.append((1, 1, 3, 40, 0, 9)[b % 6])
        lens.append(news[-1] + (b * 37) % 200)
    check(Paged(lens, news, 16, 4, 2, 64, seed=21), 4, ALL, weigh=2, decay=1.0)


@pytest.mark.parametrize("lens,news", [([300, 77], [1, 1]), ([3000, 500], [1, 3]), ([5000, 900], [70, 1]), ([900, 400], [600, 300])],
                         ids=["one slice", "slices", "sliced chunk", "chunks"])
def test_results_in_place_of_the_queries(lens, news):
    import ctypes as C
    case = Paged(lens, news, 16, 8, 2, 128, seed=22)
    c = case.cuda()
    want, wl = run(c, 4, ALL)
    cache = u.binding._paged_cache(c.k, c.v, c.table, None, None, None)
    mask = (c.max_new, c.max_kv, 4, ALL, 0, 0)
    need = u.unigist_paged_attn_workspace(C.byref(cache), 2, 8, c.T, *mask, 0)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    lse = torch.empty(8, c.T, device="cuda")
    st = u.unigist_paged_attn(C.byref(cache), c.q.data_ptr(), c.q.data_ptr(), lse.data_ptr(), 2, 8, c.T, c.cu.data_ptr(), c.kv_len.data_ptr(), *mask, 128, 8 * 128,
                              0, 1.0, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert st == 0 and torch.equal(c.q.transpose(0, 1), want) and torch.equal(lse, wl)


def test_a_workspace_that_is_not_one_piece_of_memory_is_refused():
    c = Paged([900, 500], [1, 1], 16, 8, 2, 128, seed=23).cuda()
    for ws in (torch.empty(1, dtype=torch.uint8, device="cuda").expand(64 << 20), torch.empty(128 << 20, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(u.UnigistError):
            run(c, 4, ALL, workspace=ws)
    run(c, 4, ALL, workspace=torch.empty(16 << 20, dtype=torch.float32, device="cuda"))


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
def test_more_tiles_than_the_partial_results_have_room_for(e4m3):
    # 40 drafts that the chunk kernel takes (20 columns) beside a chunk: 42 tiles of each of 8 kv heads where there is room for 126 slices,
    # less than the five of every tile that one chunk would be cut in
    news = [5] * 20 + [33] + [5] * 20 + [1] * 3
    lens = [400 + 17 * b for b in range(20)] + [2500] + [1800 - 31 * b for b in range(20)] + [2000, 1, 300]
    check(Paged(lens, news, 64, 32, 8, 128, e4m3=e4m3, seed=24), 4, ALL)


@pytest.mark.parametrize("B", [300, 5000])
def test_tiles_of_thousands_of_sequences(B):
    # several sequences a lane, more than 64 of them; most without tiles, some at the ends of a lane's range
    lens, news = [], []
    for b in range(B):
        news.append({0: 1, 1: 0, 2: 1, 3: 0, 4: 5, 78: 40, 79: 33, 80: 70}.get(b % 97, 0) if b else 40)
        lens.append(news[-1] + (b * 37) % (200 if B < 1000 else 20))
    news[-1], lens[-1] = 35, 60
    check(Paged(lens, news, 16, 4, 1, 64, seed=25), 4, ALL)


def test_one_row_a_sequence_with_a_group_of_many_heads():
    # more columns than the decode kernel takes, without boundaries
    case = Paged([300, 90, 700], [1, 1, 1], 16, 80, 2, 64, seed=26)
    c = case.cuda()
    want, wl = run(c, 4, ALL)
    out, lse = u.paged_attn(c.q.transpose(0, 1), c.k, c.v, c.table, c.kv_len, 4, ALL)
    wo, ll, _ = case.want(4, ALL)
    for x, y in ((out, lse), (want, wl)):
        assert out_ok(to_np(x), wo) and max_abs(to_np(y), ll) <= TOL_LSE_BF16


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("L", [6000, 20000])
def test_a_chunk_in_dozens_of_slices(L, e4m3):
    # four tiles over one kv head, cut into slices of 256 rows and more: 23 of them, or as many as there are at most (32)
    case = Paged([L], [64], 64, 8, 1, 128, e4m3=e4m3, seed=27)
    g = torch.Generator().manual_seed(28)
    for h, j in enumerate((3, 700, L // 2, L - 2000, L - 900, L - 300, L - 70)):  # head h: a key that outweighs all others together in one slice
        x = case.q[:, h].float().mean(0) + 0.3 * torch.randn(128, generator=g)
        x = (x * 40 / x.norm()).to(torch.bfloat16)  # |x| = 40, |q| about 11
        case.q[:, h] = (0.3 * case.q[:, h].float() + x.float() / 4).to(torch.bfloat16)  # scores of about 10 * 40 / 11 = 35
        if e4m3:
            x = torch.from_numpy(oracle.quantize_e4m3(x.float().numpy()[None, None, None], case.ks.numpy()))[0, 0, 0]
        case.k[int(case.table[0, j // 64]), 0, j % 64] = x
    check(case, 4, ALL)
    check(case, 4, ALL, weigh=40, decay=0.5)


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens,news", [([300, 1, 77, 1000], [1, 1, 1, 1]), ([700, 8, 64, 129], [8, 3, 5, 2]), ([700, 1, 64, 129], [33, 1, 5, 1])],
                         ids=["tokens", "drafts", "with a chunk"])
def test_weights_of_few_columns_without_kept_scores(lens, news, e4m3):
    # a bound of 2^23 rows: the scores would take more than the workspace may, and are made a second time
    import ctypes as C
    case = Paged(lens, news, 16, 16, 2, 64, e4m3=e4m3, seed=29, missing=[(0, 2)])
    c = case.cuda()
    cache = u.binding._paged_cache(c.k, c.v, c.table, case.ks, case.vs, c.weight, values=False)
    if e4m3:
        cache.k_scale, cache.v_scale = c.ks.data_ptr(), c.vs.data_ptr()
    size = lambda weigh: u.unigist_paged_attn_workspace(C.byref(cache), 4, 16, c.T, c.max_new, 1 << 23, 4, ALL * 2, 0, 0, weigh)
    assert size(100) == size(0) > 0
    wo, wl, added = case.want(4, 1 << 23, weigh=100)
    out, lse = u.paged_attn(c.q.transpose(0, 1), c.k, c.v, c.table, c.kv_len, 4, 1 << 23, cu=c.cu, max_new=c.max_new, max_kv=1 << 23, weight=c.weight, weigh=100,
                            decay=0.5, **c.scales)
    want = case.want_weight(added, 0.5)
    assert out_ok(to_np(out), wo) and max_abs(to_np(lse), wl) <= TOL_LSE_BF16
    assert (np.abs(to_np(c.weight) - want) <= 2e-4 * want + 1e-9).all()


@pytest.mark.parametrize("e4m3", [False, True], ids=["bf16", "e4m3"])
@pytest.mark.parametrize("lens,news", [([300, 150], [1, 1]), ([300, 150, 40], [1, 9, 20])], ids=["tokens", "two rows a tile"])
def test_a_group_of_64_heads(lens, news, e4m3):
    check(Paged(lens, news, 16, 64, 1, 128, e4m3=e4m3, seed=30), 4, ALL)
    check(Paged(lens, news, 16, 64, 1, 128, e4m3=e4m3, seed=30), 4, 30, weigh=3, sinks=2)


@pytest.mark.parametrize("news", [[1, 1], [3, 40], [300, 1]], ids=["decode", "drafts", "chunk"])
def test_captured_and_replayed_with_other_tables(news):
    # the pages move between the replays, and with them the weights
    case = Paged([900, 500], news, 16, 8, 2, 128, seed=31)
    c = case.cuda()
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
    first = [x.clone() for x in (c.k, c.v, c.weight, c.table)]

    def step():
        return run(c, 4, ALL, weight=c.weight, weigh=2, decay=0.5, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out, lse = step()
    c.weight.copy_(first[2])
    want = [x.clone() for x in step()]
    weight = c.weight.clone()
    for n in range(3):
        to = torch.randperm(c.k.shape[0], generator=torch.Generator().manual_seed(n)).cuda()  # page p becomes page to[p]
        for x, y in zip((c.k, c.v, c.weight), first):
            x[to] = y
        c.table.copy_(torch.where(first[3] >= 0, to[first[3].clamp(min=0).long()].int(), first[3]))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(c.weight[to], weight), n
