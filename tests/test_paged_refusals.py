"""What the paged entry points refuse, before anything is launched (no GPU needed: no pointer is followed)."""
import ctypes as C

import pytest
import torch

import paper_2509_15763_amd as u

FAKE = 0x1000
OK, EINVAL, EUNSUPPORTED = 0, 1, 2


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=None, v_scale=None, weight=FAKE, table=FAKE, n_pages=10, page=16, table_cols=4, Hkv=2, D=64, dt=0)
    a.update(kw)
    return u.binding._PagedCache(*a.values())


def attn(c=None, **kw):
    a = dict(q=FAKE, out=FAKE, lse=FAKE, B=2, Hq=4, T=3, cu=FAKE, kv_len=FAKE, max_new=2, max_kv=64, r=4, W=8, sinks=0, mode=0, hs=64, rs=256, weigh=1,
             decay=1.0, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    return u.unigist_paged_attn(C.byref(c or cache()), *a.values())


def size(c=None, **kw):
    a = dict(B=2, Hq=4, T=3, max_new=2, max_kv=64, r=4, W=8, sinks=0, mode=0, weigh=1)
    a.update(kw)
    return u.unigist_paged_attn_workspace(C.byref(c or cache()), *a.values())


def append(c=None, **kw):
    a = dict(k=FAKE, v=FAKE, hs=64, rs=128, B=2, T=3, cu=FAKE, kv_len=FAKE)
    a.update(kw)
    return u.unigist_paged_append(C.byref(c or cache()), *a.values())


def evict(src=None, dst=None, **kw):
    a = dict(B=2, kv_len=FAKE, keep=FAKE, max_kv=64, max_keep=32, sinks=0, recent=0, kept=FAKE, rows=FAKE)
    a.update(kw)
    return u.unigist_paged_evict(C.byref(src or cache()), C.byref(dst or cache()), *a.values())


BAD_CACHES = [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(table=None), EINVAL), (dict(k=FAKE + 8), EINVAL), (dict(v=FAKE + 2), EINVAL), (dict(n_pages=0), EINVAL),
              (dict(page=0), EINVAL), (dict(table_cols=0), EINVAL), (dict(Hkv=0), EINVAL), (dict(D=0), EINVAL), (dict(D=4), EUNSUPPORTED), (dict(D=100), EUNSUPPORTED),
              (dict(D=136), EUNSUPPORTED), (dict(dt=1), EUNSUPPORTED), (dict(dt=7), EUNSUPPORTED), (dict(dt=2, D=72), EUNSUPPORTED),
              (dict(n_pages=1 << 20, page=1 << 10), EUNSUPPORTED), (dict(n_pages=1 << 19, page=513), EUNSUPPORTED), (dict(n_pages=0x7FFFFFFF, page=0x7FFFFFFF, Hkv=0x7FFFFFFF), EUNSUPPORTED)]


@pytest.mark.parametrize("kw,want", BAD_CACHES)
def test_descriptors(kw, want):
    c = cache(**kw)
    assert attn(c) == want and size(c) == 0 and append(c) == want and evict(c) == want and evict(None, c) == want


def test_codes_need_scales():
    for kw in (dict(), dict(k_scale=FAKE), dict(v_scale=FAKE)):
        c = cache(dt=2, **kw)
        assert attn(c) == EINVAL and size(c) == 0 and append(c) == EINVAL


@pytest.mark.parametrize("kw,want", [(dict(B=0), EINVAL), (dict(T=-1), EINVAL), (dict(Hq=3), EINVAL), (dict(Hq=0), EINVAL), (dict(max_new=0), EINVAL),
                                     (dict(max_kv=0), EINVAL), (dict(r=0), EINVAL), (dict(W=0), EINVAL), (dict(sinks=-1), EINVAL), (dict(mode=2), EINVAL),
                                     (dict(weigh=-1), EINVAL), (dict(B=1 << 20), EUNSUPPORTED), (dict(max_kv=(1 << 23) + 1), EUNSUPPORTED),
                                     (dict(T=(1 << 23) + 1), EUNSUPPORTED)])
def test_attn_sizes(kw, want):
    assert attn(**kw) == want and size(**kw) == 0


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(lse=None), dict(cu=None), dict(kv_len=None), dict(q=FAKE + 2), dict(out=FAKE + 8), dict(hs=65), dict(rs=63),
                                dict(rs=56), dict(hs=-64), dict(decay=-1.0), dict(decay=float("nan")), dict(decay=float("inf")), dict(ws=None), dict(ws=FAKE + 16),
                                dict(ws_bytes=0)])
def test_attn_arguments(kw):
    assert attn(**kw) == EINVAL


def test_results_on_the_queries_that_the_weights_read_again():
    assert attn(q=FAKE, out=FAKE, weigh=1) == EINVAL


@pytest.mark.parametrize("kw", [dict(q=None), dict(lse=None), dict(cu=None), dict(kv_len=None), dict(q=FAKE + 2), dict(hs=65), dict(rs=63), dict(rs=56), dict(hs=-64),
                                dict(decay=-1.0), dict(decay=float("nan")), dict(decay=float("inf")), dict(ws=None), dict(ws=FAKE + 16), dict(ws_bytes=0)])
def test_attn_arguments_with_results_apart_from_the_queries(kw):
    assert attn(out=FAKE + 4096, **kw) == EINVAL


def test_weights_asked_for_and_not_there():
    assert attn(cache(weight=None)) == EINVAL and size(cache(weight=None)) == 0
    assert size(cache(weight=None), weigh=0) > 0


def test_nothing_to_do():
    # no new rows at all: fine, and nothing is launched
    assert attn(T=0, q=None, out=None) == OK and append(T=0, k=None, v=None) == OK


@pytest.mark.parametrize("kw,want", [(dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(kv_len=None), EINVAL), (dict(cu=None), EINVAL), (dict(k=FAKE + 2), EINVAL),
                                     (dict(hs=4), EINVAL), (dict(rs=60), EINVAL), (dict(rs=1 << 31), EUNSUPPORTED), (dict(B=0), EINVAL), (dict(T=-1), EINVAL)])
def test_append_arguments(kw, want):
    assert append(**kw) == want


@pytest.mark.parametrize("kw,want", [(dict(B=0), EINVAL), (dict(kv_len=None), EINVAL), (dict(keep=None), EINVAL), (dict(kept=None), EINVAL), (dict(rows=None), EINVAL),
                                     (dict(max_kv=0), EINVAL), (dict(max_keep=0), EINVAL), (dict(sinks=-1), EINVAL), (dict(recent=-1), EINVAL),
                                     (dict(max_kv=(1 << 23) + 1), EUNSUPPORTED), (dict(max_keep=(1 << 23) + 1), EUNSUPPORTED), (dict(B=1 << 17), EUNSUPPORTED)])
def test_evict_arguments(kw, want):
    assert evict(**kw) == want


def test_evict_between_unlike_pools():
    assert evict(cache(weight=None)) == EINVAL
    for kw in (dict(Hkv=1), dict(D=128), dict(dt=2)):
        assert evict(None, cache(**kw)) == EINVAL


def test_the_workspace_does_not_depend_on_what_lies_in_device_memory():
    assert size() == size(cache(k=FAKE + 4096, table=FAKE + 4))


def test_bindings_refuse_tensors_that_are_not_on_the_gpu():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    t, n = torch.zeros(1, 2, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    q = torch.zeros(4, 1, 64, dtype=torch.bfloat16)
    for call in (lambda: u.paged_attn(q, k, k, t, n, 4, 8), lambda: u.paged_append(k, k, t, n, q[:2], q[:2]),
                 lambda: u.paged_evict(k, k, t, n, torch.zeros(4, 2, 16), n, k, k, t, 10, 5)):
        with pytest.raises(u.UnigistError):
            call()
    with pytest.raises(u.UnigistError):
        u.paged_attn(q, k.float(), k.float(), t, n, 4, 8)
    with pytest.raises(u.UnigistError):
        u.paged_attn(q, k.byte(), k.byte(), t, n, 4, 8)  # codes without scales


@pytest.mark.parametrize("B,T,max_new,max_kv", [(64, 95, 32, 32000), (256, 767, 512, 32768), (1024, 1087, 64, 16384), (1024, 1032, 9, 131072), (64, 64, 64, 12000),
                                                (65535, 65635, 100, 1 << 23)])
def test_the_workspace_goes_by_the_new_rows_and_not_by_the_sequences(B, T, max_new, max_kv):
    # one chunk among tokens: partial results of the tokens' slices (1 GiB at most) and of what one chunk takes alone, not of a tile a sequence
    c = cache(n_pages=1 << 15, page=64, Hkv=8, D=128)
    kw = dict(Hq=32, max_new=max_new, max_kv=max_kv, W=1 << 23, weigh=0)
    alone = size(c, B=1, T=max_new, **kw)
    tokens = size(c, B=B, T=B, **dict(kw, max_new=1))
    # 16 columns for the tokens where there is a chunk, 4 else; twice the chunk's tiles, and 64 MiB
    assert size(c, B=B, T=T, **kw) <= min(4 * tokens, 1 << 30) + 3 * alone + (80 << 20)


def test_more_workgroups_than_a_launch_takes():
    # 2^24 workgroups of 256 threads of the chunk kernel
    c = cache(n_pages=1 << 15, page=16, Hkv=51, D=8)
    assert size(c, B=65535, Hq=255, T=1 << 23, max_new=1 << 23, max_kv=1 << 23, weigh=0) == 0
    assert attn(c, B=65535, Hq=255, T=1 << 23, max_new=1 << 23, max_kv=1 << 23, weigh=0, hs=8, rs=8 * 255, out=FAKE + 4096) == EUNSUPPORTED


@pytest.mark.parametrize("G", [1, 4, 8])
def test_scores_are_kept_for_the_rows_that_count(G):
    # one token of each counts: its G columns, where a chunk beside them makes room for 16
    c = cache(n_pages=1 << 15, page=64, Hkv=8, D=128)
    kw = dict(B=48, Hq=8 * G, T=48 + 63, max_new=64, max_kv=16384, W=1 << 23)
    more = size(c, weigh=1, **kw) - size(c, weigh=0, **kw)
    assert more == 48 * 8 * G * 16384 * 4


def test_heads_of_the_results_on_each_other():
    for hs in (0, 56):
        assert attn(hs=hs, out=FAKE + 4096) == EINVAL
