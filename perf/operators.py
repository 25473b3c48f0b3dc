"""Operators over a paged cache, as a serving loop calls them, for timing.

A case is a dict of plain values; its "kind" says which operator it goes through:

  append    the new rows of a batch are written into their pages (bf16, or quantised to E4M3 codes)
  attn      attention of the new rows of a batch, one to thousands a sequence, over their pages
  weigh     the same, and the attention weight that every cached row received is added up
  evict     the cache of every sequence is cut to its rows of most weight

The pool is k, v [pages, kv heads, page, D] and row j of sequence b lies in page table[b, j // page], slot j % page.  kv_len[b]
rows are in use, the last n_b of them new; the new rows of the batch follow each other in q, k_new and v_new
([T, H, D] as projection layers leave them, passed as [H, T, D] views), those of sequence b from cu[b] on.  Pages of a
sequence lie anywhere in the pool.
"""
import math

import torch

own = False  # True: the framework's calls, False: the same in elementary torch operations

DEV = "cuda"
CAUSAL = 1 << 22  # a window that holds every row: plain causal attention


def listed():
    return [
        # interactive decoding of one sequence with a short history: latency
        dict(name="step_1_2k", kind="attn", B=1, Hq=32, Hkv=8, D=128, page=16, kv=2001, new="one", n=1, ragged=False, e4m3=False,
             r=4, W=CAUSAL, sinks=0),
        # serving: a token for each of 64 sequences of different lengths
        dict(name="step_64_ragged", kind="attn", B=64, Hq=32, Hkv=8, D=128, page=64, kv=12000, new="one", n=1, ragged=True,
             e4m3=False, r=4, W=CAUSAL, sinks=0),
        # a token for each of 48 sequences with 32K positions in 8-bit pages, gist-masked: gists and the window are read
        dict(name="step_48_gist_e4m3", kind="attn", B=48, Hq=32, Hkv=8, D=128, page=128, kv=32000, new="one", n=1, ragged=False,
             e4m3=True, r=4, W=1024, sinks=4),
        # three to eight drafted tokens of 16 sequences are scored at once, head dimension 64
        dict(name="draft_16", kind="attn", B=16, Hq=16, Hkv=4, D=64, page=32, kv=5001, new="spread", n=8, ragged=True, e4m3=False,
             r=8, W=CAUSAL, sinks=0),
        # continuous batching of a gist model: a chunk of a prompt beside 15 sequences that decode
        dict(name="mixed_16", kind="attn", B=16, Hq=32, Hkv=8, D=128, page=64, kv=8192, new="mixed", n=1000, ragged=True,
             e4m3=False, r=4, W=512, sinks=0),
        # the last chunk of a 32K prompt, plain causal
        dict(name="chunk_4k_at_28k", kind="attn", B=1, Hq=32, Hkv=8, D=128, page=64, kv=32768, new="all", n=4096, ragged=False,
             e4m3=False, r=4, W=CAUSAL, sinks=0),
        # the end of a prompt looks back: what the last 64 queries attend to decides what is kept
        dict(name="weigh_64_of_32k", kind="weigh", B=1, Hq=32, Hkv=8, D=128, page=64, kv=32000, new="all", n=64, ragged=False,
             e4m3=False, r=4, W=CAUSAL, sinks=0, weigh=64, decay=0.0),
        # every decoding step of 32 sequences adds to the weights
        dict(name="weigh_step_32", kind="weigh", B=32, Hq=32, Hkv=8, D=128, page=32, kv=4100, new="one", n=1, ragged=True,
             e4m3=False, r=4, W=CAUSAL, sinks=0, weigh=1, decay=1.0),
        # the rows of one decoding step
        dict(name="append_64", kind="append", B=64, Hkv=8, D=128, page=64, kv=1500, new="one", n=1, ragged=True, e4m3=False),
        # the rows of three prompt chunks, quantised
        dict(name="append_chunks_e4m3", kind="append", B=3, Hkv=8, D=128, page=16, kv=6000, new="spread", n=4001, ragged=True,
             e4m3=True),
        # a 32K prompt is cut to an eighth
        dict(name="evict_32k_to_4k", kind="evict", B=1, Hkv=8, D=128, page=64, kv=32768, ragged=False, e4m3=False, keep=4096,
             sinks=4, recent=64),
        # 64 decoding sequences have outgrown their budget by 256 rows
        dict(name="evict_64_to_2k", kind="evict", B=64, Hkv=8, D=128, page=64, kv=2304, ragged=False, e4m3=False, keep=2048,
             sinks=4, recent=512),
    ]


# ---------------------------------------------------------------- drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = ((32, 8), (32, 8), (16, 4), (16, 16), (8, 1), (28, 4))


def draw(rng):
    """One more case of the ranges above; the sizes are redrawn until the pass costs no more than the largest listed one."""
    while True:
        c = _draw(rng)
        w = work(c)
        n, kv = _news(c), _lens(c)
        padded = 4.0 * c["B"] * c.get("Hq", 0) * max(n) * max(kv)  # scores of the plain form
        if w["flops"] <= 2.1e12 and w["bytes"] <= 2.2e9 and padded <= 18e9 and _pool_bytes(c) <= 4e9:
            return c


def _draw(rng):
    kind = rng.choice(("attn", "attn", "attn", "weigh", "weigh", "append", "evict"))
    Hq, Hkv = rng.choice(_HEADS)
    c = dict(kind=kind, B=_log(rng, 1, 64), Hkv=Hkv, D=rng.choice((128, 128, 128, 64, 64, 96)),
             page=rng.choice((16, 16, 32, 64, 64, 128, 256)), ragged=rng.random() < 0.6, e4m3=rng.random() < 0.35)
    if kind == "evict":
        kv = _log(rng, 200, 40000)
        keep = max(1, int(kv * rng.uniform(0.05, 0.95)))
        return dict(c, kv=kv, keep=keep, sinks=rng.choice((0, 4, 4)), recent=min(keep // 2, _log(rng, 1, 512)))
    new = rng.choice(("one", "one", "spread", "spread", "mixed", "all"))
    n = {"one": 1, "spread": _log(rng, 2, 16), "mixed": _log(rng, 32, 2048), "all": _log(rng, 2, 4096)}[new]
    if kind == "append" and new == "spread":
        n = _log(rng, 2, 4096)
    kv = n + _log(rng, 1, 32000)
    c.update(new=new, n=n, kv=kv)
    if kind == "append":
        return c
    gist = rng.random() < 0.4
    c.update(Hq=Hq, r=rng.choice((2, 4, 8, 16)), W=_log(rng, 64, 2048) if gist else CAUSAL, sinks=rng.choice((0, 4, 128)) if gist else 0)
    if kind == "weigh":
        c.update(weigh=rng.choice((1, 32, 64)), decay=rng.choice((0.0, 0.95, 1.0)))
    return c


# ---------------------------------------------------------------- sizes
def _news(case):
    """New rows per sequence."""
    B, n, new = case["B"], case.get("n", 0), case.get("new", "all")
    if new == "mixed":
        return [n] + [1] * (B - 1)
    if new == "spread":  # from a third up
        return [max(1, round(n * (1 / 3 + 2 / 3 * ((b * 0.618 + 1) % 1 if b else 1)))) for b in range(B)]
    return [n] * B


def _lens(case):
    """Rows in use per sequence, the new ones among them: the same for all, or spread from a sixteenth upwards."""
    B, kv, news = case["B"], case["kv"], _news(case)
    if not case["ragged"]:
        return [kv] * B
    return [max(n, round(kv * (1 / 16 + 15 / 16 * ((b * 0.618) % 1 if b else 1)))) for b, n in enumerate(news)]


def _pages(case):
    return [-(-x // case["page"]) for x in _lens(case)]


def _pool_bytes(case):
    return 2.0 * (sum(_pages(case)) + 3) * case["Hkv"] * case["page"] * case["D"] * (1 if case["e4m3"] else 2)


def _visible(case, L, n):
    """(pairs a head has to compute, rows that some query sees) of a sequence of L rows, the last n of them new."""
    r, W, S = case["r"], case["W"], case["sinks"]
    p = torch.arange(L - n, L, dtype=torch.int64)
    lo = (p - W + 1).clamp(min=0)
    always = lambda x: torch.where(x <= S, x, S + torch.div((x - S).clamp(min=0), r + 1, rounding_mode="floor"))  # of them below x
    pairs = int((p + 1 - lo + always(lo)).sum())
    first = int(lo[0])
    return pairs, L - first + int(always(torch.tensor(first)))


def work(case):
    B, Hkv, D, eb = case["B"], case["Hkv"], case["D"], 1 if case["e4m3"] else 2
    kind, lens, news = case["kind"], _lens(case), _news(case)
    row = 2 * Hkv * D * eb  # bytes of one row of both caches
    if kind == "append":
        return {"bytes": float(sum(news) * (2 * Hkv * D * 2 + row)), "flops": 0.0}
    if kind == "evict":
        kept = sum(min(case["keep"], x) for x in lens)
        return {"bytes": float(sum(lens) * Hkv * 4 + kept * (2 * row + 4 * Hkv * 2)), "flops": 0.0}
    pairs, rows = (sum(x) for x in zip(*(_visible(case, L, n) for L, n in zip(lens, news))))
    Hq, T = case["Hq"], sum(news)
    b = T * Hq * (4 * D + 4) + rows * row
    if kind == "weigh":
        b += sum(lens) * Hkv * (4 if case["decay"] == 0 else 8)
    return {"bytes": float(b), "flops": 4.0 * D * Hq * pairs}


# ---------------------------------------------------------------- inputs
def _scales(H, gen):
    """One scale per kv head, about the largest magnitude of unit-variance data / 448."""
    return [(lo + 0.004 * torch.rand(H, generator=gen, device=DEV)).float() for lo in (0.0093, 0.0107)]


def _table(pages, cols, first, gen):
    """Every sequence's pages, dealt from a shuffled pool; places that a sequence does not use hold -1."""
    ids = (torch.randperm(sum(pages), generator=gen, device=DEV) + first).to(torch.int32)
    have = torch.arange(cols, device=DEV)[None, :] < torch.tensor(pages, device=DEV)[:, None]
    t = torch.full((len(pages), cols), -1, dtype=torch.int32, device=DEV)
    t[have] = ids
    return t


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    B, Hkv, D, page, kind = case["B"], case["Hkv"], case["D"], case["page"], case["kind"]
    lens, news, pages = _lens(case), _news(case), _pages(case)
    n_pages = sum(pages) + 3
    s = dict(case)
    s["table"] = _table(pages, max(pages), 2, gen)
    s["kv_len"] = _ints(lens)
    s["ks"], s["vs"] = _scales(Hkv, gen) if case["e4m3"] else (None, None)

    def randn(*shape):
        return torch.randn(*shape, generator=gen, device=DEV).to(torch.bfloat16)

    def pool(scale):
        x = randn(n_pages, Hkv, page, D)
        return x if scale is None else (x.float() / scale[:, None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)

    s["k"], s["v"] = pool(s["ks"]), pool(s["vs"])
    if kind != "evict":
        T = sum(news)
        cu = [0]
        for n in news:
            cu.append(cu[-1] + n)
        s["cu"], s["T"], s["max_new"], s["max_kv"] = _ints(cu), T, max(news), max(lens)
    if kind in ("attn", "weigh"):
        s["q"] = randn(T, case["Hq"], D).transpose(0, 1)
    if kind == "append":
        s["k_new"], s["v_new"] = randn(T, Hkv, D).transpose(0, 1), randn(T, Hkv, D).transpose(0, 1)
    if kind == "weigh":  # about what one more query leaves
        s["weight"] = torch.rand(n_pages, Hkv, page, generator=gen, device=DEV).mul_(case["Hq"] / Hkv / s["max_kv"])
    if kind == "evict":  # what a row received so far spans several orders of magnitude; some received nothing
        w = torch.randn(n_pages, Hkv, page, generator=gen, device=DEV).mul_(2).exp_()
        s["weight"] = w.mul_(torch.rand(w.shape, generator=gen, device=DEV) > 0.05)
    if kind == "evict":
        keep = [min(case["keep"], x) for x in lens]
        to = [-(-x // page) for x in keep]
        s["keep"], s["max_kv"], s["max_keep"] = _ints(keep), max(lens), max(keep)
        s["table_out"] = _table(to, max(to), 1, gen)
        shape = (sum(to) + 2, Hkv, page, D)
        s["k_out"], s["v_out"] = (torch.zeros(shape, dtype=s["k"].dtype, device=DEV) for _ in range(2))
        s["weight_out"] = torch.zeros(shape[:3], device=DEV)
    return s


# ---------------------------------------------------------------- one pass
def run(state):
    return (_run_own if own else _run_plain)(state)


def _codes(s, x):
    """8-bit codes as the numbers they stand for (times the head's scale)."""
    return x.view(torch.float8_e4m3fn) if s["e4m3"] else x


def _run_own(s):
    import paper_2509_15763_amd as u
    kind = s["kind"]
    if kind == "append":
        u.paged_append(s["k"], s["v"], s["table"], s["kv_len"], s["k_new"], s["v_new"], cu=s["cu"], k_scale=s["ks"], v_scale=s["vs"])
        return _codes(s, s["k"]), _codes(s, s["v"])
    if kind == "evict":
        rows, kept = u.paged_evict(s["k"], s["v"], s["table"], s["kv_len"], s["weight"], s["keep"], s["k_out"], s["v_out"],
                                   s["table_out"], s["max_kv"], s["max_keep"], sinks=s["sinks"], recent=s["recent"],
                                   weight_out=s["weight_out"])
        return rows, kept, _codes(s, s["k_out"]), _codes(s, s["v_out"]), s["weight_out"]
    more = dict(weight=s["weight"], weigh=s["weigh"], decay=s["decay"]) if kind == "weigh" else {}
    out, lse = u.paged_attn(s["q"], s["k"], s["v"], s["table"], s["kv_len"], s["r"], s["W"], cu=s["cu"], max_new=s["max_new"],
                            max_kv=s["max_kv"], sinks=s["sinks"], k_scale=s["ks"], v_scale=s["vs"], **more)
    return (out, lse, s["weight"]) if kind == "weigh" else (out, lse)


def _slots(s, table, rows):
    """(page, slot) of the row numbers `rows` [B, n]."""
    page = torch.gather(table.long(), 1, torch.div(rows, s["page"], rounding_mode="floor"))
    return page, rows % s["page"]


def _seq_of(s):
    """For each new row of the batch: its sequence, its number among that sequence's new rows."""
    t = torch.arange(s["T"], device=DEV)
    b = torch.searchsorted(s["cu"][1:].long().contiguous(), t, right=True)
    return b, t - s["cu"].long()[b]


def _run_plain(s):
    return {"append": _plain_append, "evict": _plain_evict}.get(s["kind"], _plain_attn)(s)


def _plain_append(s):
    b, i = _seq_of(s)
    row = (s["kv_len"].long() - (s["cu"][1:] - s["cu"][:-1]).long())[b] + i
    page = s["table"].long()[b, torch.div(row, s["page"], rounding_mode="floor")]

    def put(pool, new, scale):
        x = new.transpose(0, 1)  # [T, Hkv, D]
        if s["e4m3"]:
            x = (x.float() / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        pool[page, :, row % s["page"]] = x

    put(s["k"], s["k_new"], s["ks"])
    put(s["v"], s["v_new"], s["vs"])
    return _codes(s, s["k"]), _codes(s, s["v"])


def _dense(s, pool, scale):
    """The pages of every sequence one after the other, in 32 bits: [B, Hkv, rows, D]."""
    x = pool[s["table"].long().clamp(min=0)]
    x = x.view(torch.float8_e4m3fn).float() * scale[:, None, None] if s["e4m3"] else x.float()
    return x.transpose(1, 2).flatten(2, 3)


def _plain_attn(s):
    B, Hq, Hkv, D, n = s["B"], s["Hq"], s["Hkv"], s["D"], s["max_new"]
    G, cu, kv = Hq // Hkv, s["cu"].long(), s["kv_len"].long()
    have = (cu[1:] - cu[:-1])[:, None]                                      # new rows
    i = torch.arange(n, device=DEV)[None, :]
    q = s["q"].transpose(0, 1)[(cu[:-1, None] + i).clamp(max=s["T"] - 1)].float()  # [B, n, Hq, D], rows past `have` unused
    q = q.reshape(B, n, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * n, D)
    k, v = _dense(s, s["k"], s["ks"]), _dense(s, s["v"], s["vs"])
    L = k.shape[2]
    p = (kv[:, None] - have + i)[:, :, None]                                # position of a query
    j = torch.arange(L, device=DEV)[None, None, :]
    always = (j < s["sinks"]) | ((j - s["sinks"] + 1) % (s["r"] + 1) == 0)
    sees = (j <= p) & (j < kv[:, None, None]) & (always | (j > p - s["W"])) & (i < have)[:, :, None]
    x = torch.matmul(q, k.transpose(2, 3)).mul_(D ** -0.5).view(B, Hkv, G, n, L)
    x.masked_fill_(~sees[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp(min=-3e38)                           # a row that sees nothing: all of exp(-inf)
    e = x.sub_(m).exp_()
    l = e.sum(-1, keepdim=True)
    out = torch.matmul(e.view(B, Hkv, G * n, L), v).view(B, Hkv, G, n, D) / torch.where(l > 0, l, 1)
    b, at = _seq_of(s)
    lse = torch.where(l > 0, m + torch.log(l), -math.inf)[..., 0]
    out = out.reshape(B, Hq, n, D).permute(1, 0, 2, 3)[:, b, at].to(torch.bfloat16)
    lse = lse.reshape(B, Hq, n).permute(1, 0, 2)[:, b, at]
    if s["kind"] != "weigh":
        return out, lse
    late = (i >= have - s["weigh"])[:, None, None, :, None]                 # the last queries of each sequence
    add = torch.where(late & (l > 0), e / torch.where(l > 0, l, 1), 0).sum((2, 3))  # [B, Hkv, L]
    rows = torch.arange(L, device=DEV)[None, :].expand(B, L)
    rows = torch.where(rows < kv[:, None], rows, 0)                         # rows past the end repeat row 0
    page, slot = _slots(s, s["table"], rows)
    add = torch.gather(add, 2, rows[:, None].expand(B, Hkv, L)).transpose(1, 2)
    s["weight"][page, :, slot] = add + (s["decay"] * s["weight"][page, :, slot] if s["decay"] else 0)
    return out, lse, s["weight"]


def _plain_evict(s):
    B, Hkv, kv, keep = s["B"], s["Hkv"], s["kv_len"].long()[:, None], s["keep"].long()[:, None]
    rows = torch.arange(s["max_kv"], device=DEV)[None, :].expand(B, -1)
    page, slot = _slots(s, s["table"], torch.minimum(rows, kv - 1))
    w = s["weight"][page, :, slot].transpose(1, 2)                          # [B, Hkv, rows]
    first = (rows < s["sinks"]) | (rows >= kv - s["recent"])
    w = torch.where(first[:, None], math.inf, w).masked_fill((rows >= kv)[:, None], -math.inf)
    order = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :s["max_keep"]]
    at = torch.arange(s["max_keep"], device=DEV)[None, :].expand(B, -1)
    order = torch.sort(order.masked_fill((at >= keep)[:, None], s["max_kv"]), dim=-1).values
    kept = order.masked_fill((at >= keep)[:, None], -1).to(torch.int32)
    at = torch.where(at < keep, at, 0)                                      # places past the end repeat place 0
    order = torch.gather(order, 2, at[:, None].expand_as(order))            # [B, Hkv, kept rows]
    page, slot = _slots(s, s["table_out"], at)
    h = torch.arange(Hkv, device=DEV)[None, :, None]
    src = torch.gather(s["table"].long()[:, None].expand(B, Hkv, -1), 2, torch.div(order, s["page"], rounding_mode="floor"))
    s["k_out"][page[:, None], h, slot[:, None]] = s["k"][src, h, order % s["page"]]
    s["v_out"][page[:, None], h, slot[:, None]] = s["v"][src, h, order % s["page"]]
    s["weight_out"][page[:, None], h, slot[:, None]] = s["weight"][src, h, order % s["page"]]
    return s["keep"].clone(), kept, _codes(s, s["k_out"]), _codes(s, s["v_out"]), s["weight_out"]


# ---------------------------------------------------------------- from the definition, in 64 bits
def exact(case, seed):
    """Sequence by sequence, head by head of the definition; evict moves values and has no others than these."""
    if case["kind"] == "evict":
        return None
    s = prepare(case, seed)
    lens, news, D, P, Hkv = _lens(case), _news(case), case["D"], case["page"], case["Hkv"]
    if case["kind"] == "append":  # codes: the quotient before its rounding
        got = []
        for pool, new, scale in ((s["k"], s["k_new"], s["ks"]), (s["v"], s["v_new"], s["vs"])):
            x, t0 = _codes(s, pool).double(), 0
            for b, (L, n) in enumerate(zip(lens, news)):
                j = torch.arange(L - n, L, device=DEV)
                rows = new[:, t0:t0 + n].double()
                if case["e4m3"]:
                    rows = (rows / scale.double()[:, None, None]).clamp(-448, 448)
                x[s["table"][b, j // P].long(), :, j % P] = rows.transpose(0, 1)
                t0 += n
            got.append(x)
        return tuple(got)
    Hq = case["Hq"]
    G, T = Hq // Hkv, s["T"]
    out = torch.zeros(Hq, T, D, dtype=torch.float64, device=DEV)
    lse = torch.full((Hq, T), -math.inf, dtype=torch.float64, device=DEV)
    weight = s["weight"].double() if case["kind"] == "weigh" else None
    t0 = 0
    for b, (L, n) in enumerate(zip(lens, news)):
        j = torch.arange(L, device=DEV)
        page, slot = s["table"][b, j // P].long(), j % P
        pos = torch.arange(L - n, L, device=DEV)
        gist = (j >= case["sinks"]) & ((j - case["sinks"] + 1) % (case["r"] + 1) == 0)
        keep = (j < case["sinks"]) | gist
        for h in range(Hkv):
            def rows(pool, scale):
                x = pool[page, h, slot]
                return x.view(torch.float8_e4m3fn).double() * scale[h].double() if case["e4m3"] else x.double()

            k, v = rows(s["k"], s["ks"]), rows(s["v"], s["vs"])
            got = torch.zeros(L, dtype=torch.float64, device=DEV)
            for g in range(G):
                hq = h * G + g
                for a in range(0, n, 1024):
                    p = pos[a:a + 1024, None]
                    vis = (p >= j) & (keep | (p - j < case["W"]))
                    sc = (s["q"][hq, t0 + a:t0 + min(n, a + 1024)].double() @ k.T) / math.sqrt(D)
                    ls = torch.logsumexp(torch.where(vis, sc, -math.inf), -1)
                    pr = torch.where(vis, torch.exp(sc - ls[:, None]), 0.0)
                    rr = slice(t0 + a, t0 + min(n, a + 1024))
                    out[hq, rr], lse[hq, rr] = pr @ v, ls
                    if weight is not None:
                        got += pr[p[:, 0] >= L - case["weigh"]].sum(0)
            if weight is not None:
                weight[page, h, slot] = got + (case["decay"] * weight[page, h, slot] if case["decay"] else 0)
        t0 += n
    return (out, lse, weight) if weight is not None else (out, lse)
