"""What is measured of the paged 8-bit cache where requests share pages, and of differential attention over it.

A cache page holds `page` tokens of every kv head as e4m3 codes, [n_pages, H, page, 128], with one float32 scale for each page and
head: value = code * scale. A request's pages stand in its row of the block table; requests that began as one name the same pages.

* fork:        new requests begin as copies of others: their whole pages are shared, the open last page is copied to a fresh one.
* release:     finished requests give back the pages that no running request names, each page once.
* compact:     the pages that requests name move to the front of the pool, the tables and the free stack follow.
* attn_shared: one new token of every request, where groups of requests share their first tokens: shared pages are read once.
* attn_diff:   differential attention. A row of q and of K is two halves of 64; out = softmax(q1 K1) V - lam * softmax(q2 K2) V, then
               a root-mean-square norm over the 128 channels where a gain is given.
"""
import math

import numpy as np
import torch

own = False

D = 128
E4M3_MAX = 448.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # parallel sampling: eight answers to one prompt; the smallest fork, pure latency
        {"name": "fork_1_to_8", "op": "fork", "H": 8, "page": 64, "lens": "5000", "each": 7, "cut": False},
        # a beam search step: 16 prompts, 16 beams each, some taken up at an earlier token
        {"name": "fork_16_to_256", "op": "fork", "H": 8, "page": 64,
         "lens": "16384,1000,777,12001,4096,65,64,63,9999,8191,15000,3,2048,6001,11111,500", "each": 15, "cut": True},
        # seven of eight answers have finished: only what was theirs alone goes back
        {"name": "release_7_of_8", "op": "release", "page": 64, "prompts": 1, "each": 8, "longest": 5000, "gone": 7},
        # a scheduler step of 512 requests, eight to a prompt
        {"name": "release_512", "op": "release", "page": 16, "prompts": 64, "each": 8, "longest": 4096, "gone": 101},
        # a small pool with a few holes
        {"name": "compact_small", "op": "compact", "H": 4, "page": 16, "n_pages": 300, "B": 5, "live": 0.8},
        # half a large pool has become free: two thousand pages move before its memory is handed on
        {"name": "compact_half", "op": "compact", "H": 8, "page": 64, "n_pages": 8192, "B": 64, "live": 0.5},
        # eight answers to one short prompt
        {"name": "shared_8x2048", "op": "attn_shared", "dtype": "bf16", "H": 8, "G": 4, "page": 64, "shared": "2048", "rows": "8", "tail": 100},
        # 64 requests behind one long common text
        {"name": "shared_64x32768", "op": "attn_shared", "dtype": "bf16", "H": 8, "G": 4, "page": 64, "shared": "32768", "rows": "64", "tail": 512},
        # float32, seven query heads per kv head, groups of several sizes, requests without a group among them
        {"name": "shared_groups_f32", "op": "attn_shared", "dtype": "f32", "H": 4, "G": 7, "page": 32, "shared": "4000,0,992,32,2016",
         "rows": "5,1,3,2,4", "tail": 333},
        # a decode step of 16 requests at 16384 tokens, two differential heads per kv head
        {"name": "diff_decode_16x16384", "op": "attn_diff", "dtype": "bf16", "H": 8, "G": 2, "page": 64, "lens": "16384" + ",16384" * 15,
         "new": "", "gain": True},
        # float32, three differential heads per kv head, ragged lengths, no norm
        {"name": "diff_decode_ragged_f32", "op": "attn_diff", "dtype": "f32", "H": 5, "G": 3, "page": 32, "lens": "4096,1,2111,333,4000,129",
         "new": "", "gain": False},
        # a chunk of a long prompt beside a decoding request and a fresh short prompt
        {"name": "diff_chunk_1024", "op": "attn_diff", "dtype": "bf16", "H": 8, "G": 2, "page": 64, "lens": "9216,4001,333", "new": "1024,1,333",
         "gain": True},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["fork", "release", "compact", "attn_shared", "attn_shared", "attn_diff", "attn_diff"])
    page = rng.choice([16, 32, 64, 128])
    H = rng.choice([1, 2, 4, 5, 8])
    if op == "fork":
        each, n = _log(rng, 1, 31), _log(rng, 1, 16)
        return {"op": op, "H": H, "page": page, "lens": _text(_log(rng, 1, 16384) for _ in range(n)), "each": each, "cut": rng.random() < 0.5}
    if op == "release":
        prompts, each = _log(rng, 1, 64), _log(rng, 1, 8)
        return {"op": op, "page": page, "prompts": prompts, "each": each, "longest": _log(rng, 16, 8192), "gone": rng.randint(1, prompts * each)}
    if op == "compact":
        return {"op": op, "H": H, "page": page, "n_pages": _log(rng, 100, 8192 * 64 // page // 2), "B": _log(rng, 1, 64),
                "live": rng.choice([0.1, 0.5, 0.9, rng.random()])}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "attn_shared":
        groups = _log(rng, 1, 8)
        rows = [_log(rng, 1, 64 // groups) for _ in range(groups)]
        longest = _log(rng, page, (32768 if dtype == "bf16" else 8192) // groups + page)
        return {"op": op, "dtype": dtype, "H": H, "G": rng.randint(1, 8), "page": page, "rows": _text(rows), "tail": _log(rng, 1, 600),
                "shared": _text(rng.choice([0, rng.randint(0, longest), longest]) // page * page for _ in rows)}
    B = _log(rng, 1, 16)
    longest = _log(rng, 1, 131072 // B)
    lens = [rng.randint(max(1, longest // 3), longest) for _ in range(B)]
    case = {"op": op, "dtype": dtype, "H": H, "G": rng.randint(1, 4), "page": page, "lens": _text(lens), "new": "", "gain": rng.random() < 0.5}
    if rng.random() < 0.5:
        # fewer pairs of a token and a query than in the listed chunk
        most = max(1, (1024 if dtype == "bf16" else 256) * 9216 // (longest * B))
        case["new"] = _text(min(n, _log(rng, 1, min(most, 1024))) for n in lens)
    return case


# ---------------------------------------------------------------------------------------------------- inputs

def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _text(ints):
    return ",".join(str(x) for x in ints)


def _pages(n, page):
    return (n + page - 1) // page


def _device(*arrays):
    return [torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32)).cuda() for a in arrays]


def _handle(case, st):
    """What a program that serves keeps: the handle of its cache."""
    from paper_2507_20030_b200 import binding
    H = case.get("H", 1)
    return binding.Pages(n_kv_heads=H, n_q_heads=H * case.get("G", 1), page_size=case["page"], n_pages=st["n_pages"],
                         max_pages=st["table"].shape[1], max_batch=st["table"].shape[0],
                         kv_dtype=binding.F32 if case.get("dtype") == "f32" else binding.BF16)


def _codes(g, n_pages, H, page, loud):
    """Pages filled earlier from N(0, 1), keys with a few loud channels, as rotary models have them."""
    codes = torch.empty((n_pages, H, page, D), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((n_pages, H), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 26) // (H * page * D))
    for p in range(0, n_pages, step):
        x = torch.randn((min(step, n_pages - p), H, page, D), generator=g, device="cuda")
        if loud is not None:
            x[..., loud] *= 10.0
        s = torch.exp2(torch.ceil(torch.log2(x.abs().amax(dim=(2, 3)) / E4M3_MAX)))
        codes[p:p + step] = (x / s[:, :, None, None]).to(torch.float8_e4m3fn)
        scales[p:p + step] = s
    return codes, scales


def _with_cache(st, case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    loud = torch.randperm(D, generator=g, device="cuda")[:4]
    st["k_pages"], st["k_scale"] = _codes(g, st["n_pages"], case["H"], case["page"], loud)
    st["v_pages"], st["v_scale"] = _codes(g, st["n_pages"], case["H"], case["page"], None)
    return g


def _grouped(r, shared, tails, page, spare, n_pages=None, W=None):
    """Rows of groups that name the same first pages: table, lengths, pages of the pool, those that are free. tails[i]: tokens behind the
    shared ones of each row of group i."""
    rows = sum(len(t) for t in tails)
    n_pages = n_pages or sum(s // page + sum(_pages(t, page) for t in ts) for s, ts in zip(shared, tails)) + spare
    perm = r.permutation(n_pages)
    W = W or max(s // page + _pages(max(ts), page) for s, ts in zip(shared, tails)) + 1
    table, lens, at, b = np.full((rows, W), -1, dtype=np.int64), [], 0, 0
    for s, ts in zip(shared, tails):
        first = s // page
        head = perm[at:at + first]
        at += first
        for t in ts:
            k = _pages(t, page)
            table[b, :first] = head
            table[b, first:first + k] = perm[at:at + k]
            at += k
            lens.append(s + t)
            b += 1
    return table, lens, n_pages, perm[at:]


def prepare(case, seed):
    r = np.random.default_rng(seed)
    st = globals()["_prepare_" + case["op"]](case, seed, r)
    st["op"], st["page"] = case["op"], case["page"]
    if own:
        st["pg"] = _handle(case, st)
    return st


def _prepare_fork(case, seed, r):
    lens, page, each = _ints(case["lens"]), case["page"], case["each"]
    n, forks = len(lens), len(lens) * each
    table, lens, n_pages, spare = _grouped(r, [0] * n, [[t] for t in lens], page, forks + 5)
    batch = n + forks
    order = r.permutation(batch)                          # where the sources lie among the rows, and the rows that the forks get
    rows = np.full((batch, table.shape[1]), -1, dtype=np.int64)
    rows[order[:n]] = table
    kv = np.zeros(batch, dtype=np.int64)
    kv[order[:n]] = lens
    src = np.repeat(order[:n], each)
    length = np.array([r.integers(max(1, t // 2), t + 1) if case["cut"] and r.random() < 0.5 else t for t in kv[src]])
    free = np.full(n_pages, -1, dtype=np.int64)
    free[:len(spare)] = spare
    st = {"n_pages": n_pages}
    st["table"], st["kv_len"], st["src"], st["dst"], st["length"], st["free_pages"], st["n_free"], st["n_free_out"] = _device(
        rows, kv, src, order[n:], length, free, [len(spare)], [0])
    _with_cache(st, case, seed)
    return st


def _prepare_release(case, seed, r):
    page, longest, prompts, each = case["page"], case["longest"], case["prompts"], case["each"]
    tail = max(1, longest // 4)
    tails = [r.integers(1, 1 + tail, each).tolist() for _ in range(prompts)]
    shared = (r.integers(longest // 2, longest + 1, prompts) * 3 // 4 // page * page).tolist()
    common = longest * 3 // 4 // page
    table, lens, n_pages, spare = _grouped(r, shared, tails, page, 0, prompts * (common + each * _pages(tail, page)) + 9,
                                           common + _pages(tail, page) + 1)
    batch = len(lens)
    order = r.permutation(batch)
    n_new = np.ones(batch, dtype=np.int64)
    n_new[r.permutation(batch)[:case["gone"]]] = -1
    free = np.full(n_pages, -1, dtype=np.int64)
    free[:len(spare)] = spare
    st = {"n_pages": n_pages}
    st["table"], st["t_len"], st["n_new"], st["free_pages"], st["n_free"], st["n_free_out"], st["kv_len"] = _device(
        table[order], np.asarray(lens)[order], n_new, free, [len(spare)], [0], np.zeros(batch))
    return st


def _prepare_compact(case, seed, r):
    page, n_pages, B = case["page"], case["n_pages"], case["B"]
    live = max(B, min(n_pages, int(case["live"] * n_pages)))
    held = np.full(B, live // B)
    held[0] += live % B
    more = r.integers(0, live // B, B // 2)               # of two requests one is as much longer as the other is shorter
    held[:B // 2 * 2:2] += more
    held[1:B // 2 * 2:2] -= more
    perm = r.permutation(n_pages)
    table = np.full((B, 2 * (live // B) + B), -1, dtype=np.int64)
    at, kv = 0, []
    for b, k in enumerate(held):
        table[b, :k] = perm[at:at + k]
        if b and r.random() < 0.5:                        # a request that began as a copy of the one before
            k0 = min(int(k), int(held[b - 1]))
            table[b, :k0 // 2] = table[b - 1, :k0 // 2]
        at += k
        kv.append(int(k) * page - int(r.integers(0, page)))
    st = {"n_pages": n_pages}
    st["table"], st["kv_len"], st["table_out"], st["free_pages"], st["n_free"], st["new_id"] = _device(
        table, kv, np.full_like(table, -1), np.full(n_pages, -1), [0], np.zeros(n_pages))
    _with_cache(st, case, seed)
    return st


def _prepare_attn_shared(case, seed, r):
    page, shared, rows = case["page"], _ints(case["shared"]), _ints(case["rows"])
    tails = [r.integers(1, case["tail"] + 1, n).tolist() for n in rows]
    table, lens, n_pages, _ = _grouped(r, shared, tails, page, 3)
    st = {"n_pages": n_pages}
    st["table"], st["kv_len"], st["group_start"], st["shared_len"] = _device(table, lens, np.concatenate([[0], np.cumsum(rows)]), shared)
    g = _with_cache(st, case, seed)
    st["q"] = torch.randn((len(lens), case["H"] * case["G"], D), generator=g, device="cuda").to(DTYPES[case["dtype"]])
    st["out"] = torch.zeros_like(st["q"])
    return st


def _prepare_attn_diff(case, seed, r):
    lens = _ints(case["lens"])
    table, lens, n_pages, _ = _grouped(r, [0] * len(lens), [[n] for n in lens], case["page"], 3)
    new = _ints(case["new"]) or [1] * len(lens)
    st = {"n_pages": n_pages, "most": max(new), "longest": max(lens)}
    st["table"], st["kv_len"], st["starts"] = _device(table, lens, np.concatenate([[0], np.cumsum(new)]))
    st["q_start"] = st["starts"] if case["new"] else None
    g = _with_cache(st, case, seed)
    HQ = case["H"] * case["G"]
    st["q"] = torch.randn((sum(new), HQ, D), generator=g, device="cuda").to(DTYPES[case["dtype"]])
    st["out"] = torch.zeros_like(st["q"])
    # the learned weight of the second map, between 0.2 and 0.8 over a model's layers, and the gain of its norm, times what the model
    # scales the heads with
    st["lam"] = 0.2 + 0.6 * torch.rand(HQ, generator=g, device="cuda")
    st["gain"] = 0.5 * (1.0 + 0.1 * torch.randn(D, generator=g, device="cuda")) if case["gain"] else None
    return st


# ---------------------------------------------------------------------------------------------------- the operators

EPS = 1e-5


def run(st):
    return globals()["_run_" + st["op"]](st)


def _run_fork(st):
    cache = [st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"]]
    out = [st["table"], st["kv_len"], st["n_free_out"]]
    if own:
        st["pg"].fork(st["src"], st["dst"], st["kv_len"], st["table"], st["free_pages"], st["n_free"], st["n_free_out"], *cache,
                      length=st["length"])
        return out + cache
    page, table, src, dst = st["page"], st["table"], st["src"].long(), st["dst"].long()
    W = table.shape[1]
    n = torch.minimum(st["length"], st["kv_len"][src]).long()
    whole, rest = n // page, n % page
    upto = torch.cumsum((rest > 0).long(), 0)
    ok = (rest == 0) | (upto <= st["n_free"].long())
    fresh = st["free_pages"][(st["n_free"].long() - upto).clamp(min=0)].long()
    col = torch.arange(W, device="cuda")
    rows = torch.where(ok[:, None] & (col < whole[:, None]), table[src], table[dst])
    copied = ok & (rest > 0)
    rows = torch.where(copied[:, None] & (col == whole[:, None]), fresh[:, None].int(), rows)
    opened = table[src, whole.clamp(max=W - 1)].long().clamp(min=0)
    table[dst] = rows
    st["kv_len"][dst] = torch.where(ok, n, torch.zeros_like(n)).int()
    st["n_free_out"].copy_(st["n_free"] - copied.sum())
    # what is not copied is written onto itself
    into = torch.where(copied, fresh, opened)
    seen = (torch.arange(page, device="cuda") < rest[:, None])[:, None, :, None]
    for codes, scale in ((st["k_pages"], st["k_scale"]), (st["v_pages"], st["v_scale"])):
        raw = codes.view(torch.uint8)
        raw[into] = torch.where(seen, raw[opened], raw[into])
        scale[into] = scale[opened]
    return out + cache


def _named(table, t, page):
    """Which entries of the block table name a page."""
    return torch.arange(table.shape[1], device="cuda") < ((t.long() + page - 1) // page)[:, None]


def _run_release(st):
    out = [st["free_pages"], st["n_free_out"], st["kv_len"]]
    if own:
        st["pg"].release(st["t_len"], st["n_new"], st["table"], st["free_pages"], st["n_free"], st["kv_len"], st["n_free_out"])
        return out
    table, n_pages = st["table"], st["n_pages"]
    gone = (st["n_new"] < 0)[:, None]
    named = _named(table, st["t_len"], st["page"])
    place = torch.arange(table.numel(), device="cuda").view_as(table)
    ids = torch.where(named, table.long(), torch.full_like(place, n_pages))
    # the first place that names each page; -1 where a running request does
    first = torch.full((n_pages + 1,), table.numel(), device="cuda").scatter_reduce(
        0, ids.flatten(), torch.where(gone, place, torch.full_like(place, -1)).flatten(), "amin")
    back = (named & gone & (first[ids] == place)).flatten()
    height = st["n_free"].long() + torch.cumsum(back.long(), 0)
    stack = torch.cat([st["free_pages"], st["free_pages"].new_zeros(1)])
    stack[torch.where(back, height - 1, torch.full_like(height, n_pages))] = table.flatten()
    st["free_pages"].copy_(stack[:n_pages])
    st["n_free_out"].copy_(height[-1:])
    st["kv_len"].copy_(torch.where(gone[:, 0], torch.zeros_like(st["t_len"]), st["t_len"]))
    return out


def _run_compact(st):
    cache = [st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"]]
    out = [st["table_out"], st["free_pages"], st["n_free"], st["new_id"]]
    if own:
        st["pg"].compact(st["kv_len"], st["table"], st["table_out"], st["free_pages"], st["n_free"], st["new_id"], *cache)
        return out + cache
    table, n_pages = st["table"], st["n_pages"]
    named = _named(table, st["kv_len"], st["page"])
    ids = torch.where(named, table.long(), n_pages)
    live = torch.zeros(n_pages + 1, dtype=torch.bool, device="cuda")
    live[ids.flatten()] = True
    live = live[:n_pages]
    n_live = live.sum()
    at = torch.arange(n_pages, device="cuda")
    hole, moves = ~live & (at < n_live), live & (at >= n_live)
    holes = torch.zeros(n_pages + 1, dtype=torch.long, device="cuda")
    holes[torch.where(hole, torch.cumsum(hole.long(), 0) - 1, n_pages)] = at
    new = torch.where(moves, holes[(torch.cumsum(moves.long(), 0) - 1).clamp(min=0)], torch.where(live, at, -1))
    st["new_id"].copy_(new)
    st["table_out"].copy_(torch.where(named, new[ids.clamp(max=n_pages - 1)], table.long()))
    st["n_free"].copy_((n_pages - n_live).reshape(1))
    st["free_pages"].copy_(torch.where(at < n_pages - n_live, n_pages - 1 - at, st["free_pages"].long()))
    source = torch.nonzero(moves)[:, 0]
    for x in cache:
        x = x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
        x[new[source]] = x[source]
    return out + cache


def _padded(st, which, longest):
    """The cached tokens of every request in 32 bits, [B, H, longest rounded up to pages, 128]; page 0 stands behind a request's end."""
    n = _pages(longest, st["page"])
    ids = torch.where(_named(st["table"], st["kv_len"], st["page"]), st["table"], 0)[:, :n].long()
    x = st[which + "_pages"][ids].float() * st[which + "_scale"][ids][..., None, None]
    return x.transpose(1, 2).reshape(x.shape[0], x.shape[2], -1, D)


def _softmax(s):
    s = torch.exp(s - s.amax(dim=-1, keepdim=True))
    return s / s.sum(dim=-1, keepdim=True)


def _run_attn_shared(st):
    if own:
        st["pg"].attn_shared(st["q"], st["kv_len"], st["table"], st["group_start"], st["shared_len"], st["k_pages"], st["v_pages"],
                             st["k_scale"], st["v_scale"], st["out"])
        return st["out"]
    longest = st["table"].shape[1] * st["page"]
    K, V = _padded(st, "k", longest), _padded(st, "v", longest)
    B, H = K.shape[:2]
    s = st["q"].float().view(B, H, -1, D) @ K.transpose(2, 3) * (1.0 / math.sqrt(D))
    s = s.masked_fill(torch.arange(K.shape[2], device="cuda") >= st["kv_len"][:, None, None, None], -math.inf)
    st["out"].copy_((_softmax(s) @ V).view(B, -1, D))
    return st["out"]


def _run_attn_diff(st):
    if own:
        st["pg"].attn_diff(st["q"], st["kv_len"], st["table"], st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], st["lam"],
                           st["out"], q_start=st["q_start"], gain=st["gain"], eps=EPS)
        return st["out"]
    K, V = _padded(st, "k", st["longest"]), _padded(st, "v", st["longest"])
    B, H, N, _ = K.shape
    q, most = st["q"], st["most"]
    HQ = q.shape[1]
    start = st["starts"].long()
    new = start[1:] - start[:-1]
    i = torch.arange(most, device="cuda")
    there = i < new[:, None]                                                          # [B, most]
    rows = torch.where(there, start[:-1, None] + i, 0)
    x = q[rows].float().view(B, most, H, HQ // H, 2, D // 2).permute(0, 4, 2, 1, 3, 5).reshape(B, 2, H, -1, D // 2)
    k = K.view(B, H, N, 2, D // 2).permute(0, 3, 1, 4, 2)                             # [B, 2, H, 64, N]
    s = x @ k * (1.0 / math.sqrt(D // 2))
    seen = torch.where(there, st["kv_len"][:, None] - new[:, None] + i + 1, 1)         # [B, most]
    hidden = torch.arange(N, device="cuda") >= seen[:, :, None]
    s.view(B, 2, H, most, HQ // H, N).masked_fill_(hidden[:, None, None, :, None, :], -math.inf)
    o = (_softmax(s) @ V[:, None]).view(B, 2, H, most, HQ // H, D)
    o = (o[:, 0] - st["lam"].view(H, 1, HQ // H, 1) * o[:, 1]).transpose(1, 2).reshape(B, most, HQ, D)
    if st["gain"] is not None:
        o = o * torch.rsqrt(o.square().mean(dim=-1, keepdim=True) + EPS) * st["gain"]
    st["out"].copy_(o[there])                                                         # in the order of the rows
    return st["out"]


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    page, op = case["page"], case["op"]
    if op == "fork":
        # rows of the tables; K and V rows of an open page, read once a source, written once a fork
        lens, each, H = _ints(case["lens"]), case["each"], case["H"]
        entries = sum(_pages(t, page) for t in lens)
        rest = sum(t % page for t in lens)
        copies = sum(t % page > 0 for t in lens)
        return {"bytes": 4 * entries * (1 + each) + (1 + each) * (2 * rest * H * D + 8 * copies * H) + 20 * len(lens) * each, "flops": 0}
    if op == "release":
        rows, longest = case["prompts"] * case["each"], case["longest"]
        named = rows * _pages(longest * 11 // 16, page)
        own_pages = case["gone"] * _pages(longest // 8, page)
        return {"bytes": 4 * (named + own_pages + 3 * rows), "flops": 0}
    if op == "compact":
        n, live = case["n_pages"], int(case["live"] * case["n_pages"])
        moved = live * (n - live) // n
        return {"bytes": 2 * moved * case["H"] * (2 * page * D + 8) + 4 * (2 * live + 2 * n - live), "flops": 0}
    H, HQ, size = case["H"], case["H"] * case["G"], 2 if case["dtype"] == "bf16" else 4
    if op == "attn_shared":
        shared, rows = _ints(case["shared"]), _ints(case["rows"])
        tail = (case["tail"] + 1) // 2
        cached = sum(s + n * tail for s, n in zip(shared, rows))
        pairs = sum(n * (s + tail) for s, n in zip(shared, rows))
        return {"bytes": 2 * cached * H * D + 8 * _pages(cached, page) * H + 2 * sum(rows) * HQ * D * size, "flops": 4 * pairs * HQ * D}
    lens = _ints(case["lens"])
    new = _ints(case["new"]) or [1] * len(lens)
    pairs = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))
    return {"bytes": 2 * sum(lens) * H * D + 8 * sum(_pages(n, page) for n in lens) * H + 2 * sum(new) * HQ * D * size,
            "flops": pairs * HQ * (2 * D + 4 * D)}


# ---------------------------------------------------------------------------------------------------- from the definitions, in 64 bits

def exact(case, seed):
    return globals()["_exact_" + case["op"]](case, prepare(case, seed))


def _lists(*tensors):
    return [x.tolist() for x in tensors]


def _back(*lists):
    return [torch.as_tensor(np.asarray(x, dtype=np.int32)) for x in lists]


def _exact_fork(case, st):
    page = case["page"]
    table, kv, src, dst, length, free, (height,) = _lists(*(st[k] for k in ("table", "kv_len", "src", "dst", "length", "free_pages", "n_free")))
    cache = [st[k].view(torch.uint8) if "pages" in k else st[k] for k in ("k_pages", "v_pages", "k_scale", "v_scale")]
    before = list(kv)
    for s, d, n in zip(src, dst, length):
        n = min(n, before[s])
        whole, rest = divmod(n, page)
        if rest and height == 0:
            kv[d] = 0
            continue
        kv[d] = n
        table[d][:whole] = table[s][:whole]
        if rest:
            height -= 1
            table[d][whole] = free[height]
            for x in cache[:2]:
                x[free[height], :, :rest] = x[table[s][whole], :, :rest]
            for x in cache[2:]:
                x[free[height]] = x[table[s][whole]]
    return _back(table, kv, [height]) + [st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"]]


def _exact_release(case, st):
    page = case["page"]
    table, t, n, free, (height,) = _lists(*(st[k] for k in ("table", "t_len", "n_new", "free_pages", "n_free")))
    held = {p for b in range(len(t)) if n[b] >= 0 for p in table[b][:_pages(t[b], page)]}
    for b in range(len(t)):
        if n[b] < 0:
            for p in table[b][:_pages(t[b], page)]:
                if p not in held:
                    held.add(p)
                    free[height] = p
                    height += 1
            t[b] = 0
    return _back(free, [height], t)


def _exact_compact(case, st):
    page, n_pages = case["page"], case["n_pages"]
    table, kv, free = _lists(st["table"], st["kv_len"], st["free_pages"])
    live = {p for row, t in zip(table, kv) for p in row[:_pages(t, page)]}
    n = len(live)
    new = [p if p in live and p < n else -1 for p in range(n_pages)]
    pairs = list(zip(sorted(p for p in live if p >= n), (p for p in range(n) if p not in live)))
    for a, b in pairs:
        new[a] = b
    table = [[new[p] if j < _pages(t, page) else p for j, p in enumerate(row)] for row, t in zip(table, kv)]
    free[:n_pages - n] = range(n_pages - 1, n - 1, -1)
    a, b = torch.tensor(pairs, dtype=torch.long, device="cuda").reshape(-1, 2).T
    for k in ("k_pages", "v_pages", "k_scale", "v_scale"):
        x = st[k].view(torch.uint8) if "pages" in k else st[k]
        x[b] = x[a].clone()
    return _back(table, free, [n_pages - n], new) + [st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"]]


def _bits(x):
    """The value of each e4m3 code, from its bits: sign, 4 exponent bits (bias 7), 3 bits behind the point; no infinities."""
    c = np.arange(256)
    s, e, m = c >> 7, (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0)) * np.where(s == 1, -1.0, 1.0)
    v[[127, 255]] = np.nan
    return torch.as_tensor(v, device=x.device, dtype=torch.float64)[x.view(torch.uint8).long()]


def _values(st, which, b, n):
    ids = st["table"][b, :_pages(n, st["page"])].long()
    x = _bits(st[which + "_pages"][ids]) * st[which + "_scale"].double()[ids][:, :, None, None]
    return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :n]


def _exact_attn_shared(case, st):
    out = st["out"].double()
    for b, n in enumerate(st["kv_len"].tolist()):
        K, V = _values(st, "k", b, n), _values(st, "v", b, n)
        w = torch.softmax(torch.einsum("hgd,hnd->hgn", st["q"][b].double().view(K.shape[0], -1, D), K) / math.sqrt(D), dim=-1)
        out[b] = torch.einsum("hgn,hnd->hgd", w, V).flatten(0, 1)
    return out


def _exact_attn_diff(case, st):
    H, G = case["H"], case["G"]
    out, at = st["out"].double(), 0
    lam = st["lam"].double().view(H, G, 1)
    starts = st["starts"].tolist()
    for b, n in enumerate(st["kv_len"].tolist()):
        m = starts[b + 1] - starts[b]
        K, V = _values(st, "k", b, n), _values(st, "v", b, n)
        for i in range(0, m, 256):                                   # 256 queries at a time
            k = min(256, m - i)
            seen = n - m + i + torch.arange(1, k + 1, device="cuda")
            x = st["q"][at + i:at + i + k].double().view(k, H, G, D)
            maps = []
            for part in (slice(0, 64), slice(64, 128)):
                s = torch.einsum("mhgd,hnd->mhgn", x[..., part], K[..., part]) / 8.0
                s = torch.where(torch.arange(n, device="cuda") < seen[:, None, None, None], s, -math.inf)
                maps.append(torch.einsum("mhgn,hnd->mhgd", torch.softmax(s, dim=-1), V))
            o = maps[0] - lam * maps[1]
            if st["gain"] is not None:
                o = o / torch.sqrt((o * o).mean(dim=-1, keepdim=True) + EPS) * st["gain"].double()
            out[at + i:at + i + k] = o.reshape(k, H * G, D)
        at += m
    return out
