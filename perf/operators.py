"""What is measured of the paged 8-bit cache: its tables, its writes, attention over it, and rows read back out of it.

A cache page holds `page` tokens of every kv head as e4m3 codes, [n_pages, H, page, 128], with one float32 scale (a power of two)
for each page and head: value = code * scale. A request's pages stand in its row of the block table. Four operators:

* tables: pages for the tokens that arrive, out of a stack of free pages, and the slot (page * page_size + row) of each token.
* store:  new tokens into their slots; the page's scale grows when they need it, and its older rows are then rounded again.
* attn:   softmax attention of the newest tokens of every request over its cached tokens, causal among the newest.
* load:   the cached tokens as rows [B, H, L, 128], zero behind the end.
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
        # one decode step's bookkeeping of 16 running requests: the smallest launch, pure latency
        {"name": "tables_decode_16", "op": "tables", "B": 16, "page": 64, "longest": 16384, "tokens": 16, "finished": 0, "free": 16},
        # a scheduler step of 512 requests: most decode, some bring a prompt chunk, some have finished
        {"name": "tables_mixed_512", "op": "tables", "B": 512, "page": 16, "longest": 4096, "tokens": 32768, "finished": 37, "free": 2600},
        # one decode step's K and V of 16 requests
        {"name": "store_decode_16", "op": "store", "dtype": "bf16", "H": 8, "page": 64, "lens": "1024" + ",1024" * 15, "new": "1" + ",1" * 15},
        # a whole prompt of 32768 tokens
        {"name": "store_prefill_32768", "op": "store", "dtype": "bf16", "H": 8, "page": 64, "lens": "32768", "new": "32768"},
        # float32 tokens, ragged chunks that start and end inside pages, an odd number of heads
        {"name": "store_ragged_f32", "op": "store", "dtype": "f32", "H": 5, "page": 32,
         "lens": "1,777,1300,64,65,2049,31,500,33", "new": "1,777,1000,1,33,900,31,2,33"},
        # the first decode steps of one short request: latency
        {"name": "attn_decode_short", "op": "attn", "dtype": "bf16", "H": 8, "G": 4, "page": 16, "lens": "60", "new": ""},
        # a decode step of 16 requests at 16384 tokens
        {"name": "attn_decode_16x16384", "op": "attn", "dtype": "bf16", "H": 8, "G": 4, "page": 64, "lens": "16384" + ",16384" * 15, "new": ""},
        # a decode step of one request at 131072 tokens: the long axis has to be split
        {"name": "attn_decode_131072", "op": "attn", "dtype": "bf16", "H": 8, "G": 4, "page": 64, "lens": "131072", "new": ""},
        # float32 queries, seven query heads per kv head, ragged lengths
        {"name": "attn_decode_ragged_f32", "op": "attn", "dtype": "f32", "H": 4, "G": 7, "page": 32,
         "lens": "4096,1,2111,333,4000,129", "new": ""},
        # a chunk of a long prompt beside a decoding request and a fresh short prompt, two rows of padding behind them
        {"name": "attn_chunk_2048", "op": "attn", "dtype": "bf16", "H": 8, "G": 4, "page": 64, "lens": "18432,9001,333",
         "new": "2048,1,333", "pad": 2},
        # four requests handed over as rows to the prefill transform
        {"name": "load_4x16384", "op": "load", "dtype": "bf16", "H": 8, "page": 64, "lens": "16384,16384,16000,9999", "L": 16384},
        # short float32 rows, one request empty
        {"name": "load_short_f32", "op": "load", "dtype": "f32", "H": 4, "page": 16, "lens": "1000,0,17", "L": 1000},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["tables", "store", "attn", "attn", "load"])
    page = rng.choice([16, 32, 64, 128])
    if op == "tables":
        B = _log(rng, 1, 512)
        tokens = max(B, _log(rng, 1, 32768))
        # now and then pages run out, and the last requests have to wait
        return {"op": op, "B": B, "page": page, "longest": _log(rng, 64, 16384), "tokens": tokens, "finished": rng.randint(0, B // 4),
                "free": B + int(tokens / page * rng.choice([0.5, 1.2, 1.2]))}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    H = rng.choice([1, 2, 4, 5, 8])
    B = _log(rng, 1, 16)
    if op == "store":
        most = _log(rng, 1, 32768 // B)
        new = [rng.randint(1, most) for _ in range(B)]
        return {"op": op, "dtype": dtype, "H": H, "page": page,
                "lens": _text(n + rng.choice([0, rng.randint(0, 300)]) for n in new), "new": _text(new)}
    longest = _log(rng, 1, 131072 // B if op == "attn" else 40000 // B)
    lens = [rng.randint(max(1, longest // 3), longest) for _ in range(B)]
    if op == "load":
        return {"op": op, "dtype": dtype, "H": H, "page": page, "lens": _text(lens), "L": max(lens) + rng.choice([0, rng.randint(0, 70)])}
    case = {"op": op, "dtype": dtype, "H": H, "G": rng.randint(1, 8), "page": page, "lens": _text(lens), "new": ""}
    if rng.random() < 0.5:
        most = _log(rng, 1, max(1, 8192 // B if dtype == "bf16" else 1024 // B))
        # fewer pairs of a token and a query than in the listed chunk
        case["new"] = _text(min(n, rng.randint(1, most), max(1, 2048 * 16384 * 4 // (n * case["G"] * 2 * B))) for n in lens)
        case["pad"] = rng.choice([0, 0, 3])
    return case


# ---------------------------------------------------------------------------------------------------- inputs

def _ints(text):
    return [int(x) for x in text.split(",")] if text else []


def _text(ints):
    return ",".join(str(x) for x in ints)


def _pages(n, page):
    return (n + page - 1) // page


def _requests(case, seed):
    """Lengths before the step and tokens that arrive, as a scheduler holds them: a few prompt chunks, decoding requests, finished ones."""
    r = np.random.default_rng(seed)
    B, longest = case["B"], case["longest"]
    t = r.integers(max(1, longest // 2), longest + 1, B)
    n = np.ones(B, dtype=np.int64)
    order = r.permutation(B)
    chunks = _chunks(case)
    for j in range(chunks):                          # prompt chunks of up to 2048 tokens
        n[order[j % B]] += min(2048, case["tokens"] - B - 2048 * j)
    if case["finished"]:
        n[order[-case["finished"]:]] = -1
    return t, n


def _chunks(case):
    return (case["tokens"] - case["B"] + 2047) // 2048


def _device(*arrays):
    return [torch.as_tensor(np.ascontiguousarray(a, dtype=np.int32)).cuda() for a in arrays]


def _prepare_tables(case, seed):
    B, page = case["B"], case["page"]
    t, n = _requests(case, seed)
    tokens = case["tokens"]
    W = _pages(case["longest"] + 1 + 2048 * -(-_chunks(case) // B), page)
    n_pages = B * _pages(case["longest"], page) + case["free"]
    perm = np.random.default_rng(seed + 1).permutation(n_pages)
    table = np.full((B, W), -1, dtype=np.int64)
    at = 0
    for b in range(B):
        k = int(_pages(t[b], page))
        table[b, :k] = perm[at:at + k]
        at += k
    free = np.full(n_pages, -1, dtype=np.int64)
    free[:case["free"]] = perm[at:at + case["free"]]
    t_len, n_new, table, free_pages, n_free = _device(t, n, table, free, [case["free"]])
    st = {"page": page, "t_len": t_len, "n_new": n_new, "table": table, "free_pages": free_pages, "n_free": n_free,
          "q_start": torch.zeros(B + 1, dtype=torch.int32, device="cuda"), "kv_len": torch.zeros(B, dtype=torch.int32, device="cuda"),
          "slots": torch.zeros(tokens, dtype=torch.int32, device="cuda"), "n_free_out": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if own:
        st["pg"] = _handle(dict(case, H=1, G=1, dtype="bf16"), n_pages, W, B)
    return st


def _handle(case, n_pages, max_pages, batch):
    from paper_2507_20030_b200 import binding
    return binding.Pages(n_kv_heads=case["H"], n_q_heads=case["H"] * case.get("G", 1), page_size=case["page"], n_pages=n_pages,
                         max_pages=max_pages, max_batch=batch, kv_dtype=binding.BF16 if case["dtype"] == "bf16" else binding.F32)


def _rows(g, shape, loud):
    """Keys with a few loud channels, as rotary models have them, or values: N(0, 1)."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if loud is not None:
        x[..., loud] *= 10.0
    return x


def _cache(g, n_pages, H, page, loud):
    """Pages filled earlier: codes [n_pages, H, page, 128] and scales [n_pages, H]."""
    codes = torch.empty((n_pages, H, page, D), dtype=torch.float8_e4m3fn, device="cuda")
    scales = torch.empty((n_pages, H), dtype=torch.float32, device="cuda")
    step = max(1, (1 << 26) // (H * page * D))
    for p in range(0, n_pages, step):
        x = _rows(g, (min(step, n_pages - p), H, page, D), loud)
        s = torch.exp2(torch.ceil(torch.log2(x.abs().amax(dim=(2, 3)) / E4M3_MAX)))
        codes[p:p + step] = (x / s[:, :, None, None]).to(torch.float8_e4m3fn)
        scales[p:p + step] = s
    return codes, scales


def _spread(lens, page, n_pages, seed):
    """A block table whose rows hold scattered pages; -1 behind a request's last page."""
    W = max(1, max(_pages(n, page) for n in lens))
    perm = np.random.default_rng(seed).permutation(n_pages)
    table = np.full((len(lens), W), -1, dtype=np.int64)
    at = 0
    for b, n in enumerate(lens):
        k = _pages(n, page)
        table[b, :k] = perm[at:at + k]
        at += k
    return table


def prepare(case, seed):
    if case["op"] == "tables":
        return _prepare_tables(case, seed)
    H, page, lens, dtype = case["H"], case["page"], _ints(case["lens"]), DTYPES[case["dtype"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    loud = torch.randperm(D, generator=g, device="cuda")[:4]
    n_pages = sum(_pages(n, page) for n in lens) + 3
    table = _spread(lens, page, n_pages, seed)
    k_pages, k_scale = _cache(g, n_pages, H, page, loud)
    v_pages, v_scale = _cache(g, n_pages, H, page, None)
    kv_len, table_d = _device(lens, table)
    st = {"op": case["op"], "page": page, "lens": lens, "k_pages": k_pages, "k_scale": k_scale, "v_pages": v_pages, "v_scale": v_scale,
          "kv_len": kv_len, "table": table_d}
    if case["op"] == "store":
        slots = []
        for b, (n, new) in enumerate(zip(lens, _ints(case["new"]))):
            pos = np.arange(n - new, n)
            slots.append(table[b, pos // page] * page + pos % page)
        slots = np.concatenate(slots)
        st["slots"], = _device(slots)
        k = _rows(g, (len(slots), H, D), loud)
        if max(_ints(case["new"])) == 1:                    # decode: now and then a token is louder than its page so far
            k *= torch.exp(torch.randn((len(slots), 1, 1), generator=g, device="cuda"))
        st["k_new"], st["v_new"] = k.to(dtype), _rows(g, (len(slots), H, D), None).to(dtype)
    elif case["op"] == "load":
        st["L"] = case["L"]
        st["K_out"] = torch.zeros((len(lens), H, case["L"], D), dtype=dtype, device="cuda")
        st["V_out"] = torch.zeros_like(st["K_out"])
    else:
        new = _ints(case["new"]) or [1] * len(lens)
        n_tokens = sum(new) + case.get("pad", 0)
        st["new"] = new
        st["q"] = torch.randn((n_tokens, H * case["G"], D), generator=g, device="cuda").to(dtype)
        st["out"] = torch.zeros_like(st["q"])
        st["q_start"] = None
        if case["new"]:
            st["q_start"], = _device(np.concatenate([[0], np.cumsum(new)]))
    if own:
        st["pg"] = _handle(case, n_pages, table.shape[1], len(lens))
    return st


# ---------------------------------------------------------------------------------------------------- the operators

def run(st):
    if "t_len" in st:
        return _run_tables(st)
    return {"store": _run_store, "attn": _run_attn, "load": _run_load}[st["op"]](st)


def _run_tables(st):
    if own:
        st["pg"].tables(st["t_len"], st["n_new"], st["table"], st["free_pages"], st["n_free"], st["q_start"], st["kv_len"], st["slots"],
                        st["n_free_out"])
        return [st["table"], st["free_pages"], st["n_free_out"], st["q_start"], st["kv_len"], st["slots"]]
    t, n, table, free = st["t_len"].long(), st["n_new"].long(), st["table"], st["free_pages"]
    B, W = table.shape
    tokens = st["slots"].numel()
    n_pages = free.numel()
    page = st["page"]
    col = torch.arange(W, device="cuda")
    # finished requests: their pages go onto the stack, in request order
    old = (t + page - 1) // page
    done = n < 0
    gone = done[:, None] & (col[None, :] < old[:, None])
    place = st["n_free"].long() + torch.cumsum(gone.flatten().long(), 0) - 1
    stack = torch.cat([free, free.new_zeros(1)])
    stack[torch.where(gone.flatten(), place, torch.full_like(place, n_pages))] = table.flatten()
    free.copy_(stack[:n_pages])
    n_avail = st["n_free"].long() + gone.sum()
    # arriving tokens, in request order, as long as pages last
    arrive = n.clamp(min=0)
    start = torch.cat([arrive.new_zeros(1), torch.cumsum(arrive, 0)])
    valid = ~done & (t + arrive <= W * page) & (start[1:] <= tokens)
    need = torch.where(valid, (t + arrive + page - 1) // page - old, torch.zeros_like(old))
    last = torch.cumsum(need, 0)
    ok = valid & ((need == 0) | (last <= n_avail))
    took = torch.where(ok, need, torch.zeros_like(need)).sum()
    kv = torch.where(done, torch.zeros_like(t), torch.where(ok, t + arrive, t))
    j = col[None, :] - old[:, None]
    fresh = ok[:, None] & (j >= 0) & (j < need[:, None])
    source = (n_avail - 1 - ((last - need)[:, None] + j)).clamp(0, n_pages - 1)
    table.copy_(torch.where(fresh, free[source], table))
    i = torch.arange(tokens, device="cuda")
    b = torch.searchsorted(start[1:].contiguous(), i, right=True)
    inside = b < B
    b = b.clamp(max=B - 1)
    pos = t[b] + i - start[b]
    slot = table[b, (pos // page).clamp(max=W - 1)].long() * page + pos % page
    st["slots"].copy_(torch.where(inside & ok[b], slot, torch.full_like(slot, -1)))
    st["q_start"].copy_(start)
    st["kv_len"].copy_(kv)
    st["n_free_out"].copy_(n_avail - took)
    return [table, free, st["n_free_out"], st["q_start"], st["kv_len"], st["slots"]]


def _two_to(x):
    """The smallest power of two s with x / s <= 448, at least 2^-126."""
    m, e = torch.frexp(x)                            # x = m * 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.ldexp(torch.ones_like(x), torch.where(x > 0, e, torch.full_like(e, -126)).clamp(min=-126))


def _round8(x):
    return x.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _run_store(st):
    if own:
        st["pg"].store(st["k_new"], st["v_new"], st["slots"], st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"])
        return [st["k_pages"], st["k_scale"], st["v_pages"], st["v_scale"]]
    page, slots = st["page"], st["slots"].long()
    n_pages, H = st["k_scale"].shape
    at, row = slots // page, slots % page
    first = torch.full((n_pages,), page, dtype=torch.long, device="cuda").scatter_reduce(0, at, row, "amin")
    touched, inverse = torch.unique(at, return_inverse=True)
    first = first[touched]
    for x, codes, scales in ((st["k_new"], st["k_pages"], st["k_scale"]), (st["v_new"], st["v_pages"], st["v_scale"])):
        x = x.float()
        a = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(dim=2)
        top = torch.zeros((touched.numel(), H), device="cuda").scatter_reduce(0, inverse[:, None].expand(-1, H), a, "amax")
        old = scales[touched]
        new = torch.where(first[:, None] == 0, _two_to(top), torch.maximum(old, _two_to(top)))
        older = (torch.arange(page, device="cuda")[None, :] < first[:, None])[:, None, :, None] & (new > old)[:, :, None, None]
        raw = codes.view(torch.uint8)
        again = _round8(codes[touched].float() * old[:, :, None, None] / new[:, :, None, None]).view(torch.uint8)
        raw[touched] = torch.where(older, again, raw[touched])
        scales[touched] = new
        raw[at, :, row] = _round8(x / scales[at][:, :, None]).view(torch.uint8)
    return [st["k_pages"], st["k_scale"], st["v_pages"], st["v_scale"]]


def _gather(st, which, b):
    """The cached tokens of request b in 32 bits, [H, len, 128]."""
    n, page = st["lens"][b], st["page"]
    ids = st["table"][b, :_pages(n, page)].long()
    x = st[which + "_pages"][ids].float() * st[which + "_scale"][ids][:, :, None, None]
    return x.transpose(0, 1).reshape(x.shape[1], -1, D)[:, :n]


def _run_attn(st):
    if own:
        st["pg"].attn(st["q"], st["kv_len"], st["table"], st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], st["out"],
                      q_start=st["q_start"])
        return st["out"]
    q, out = st["q"], st["out"]
    HQ = q.shape[1]
    H = st["k_scale"].shape[1]
    G = HQ // H
    at = 0
    for b, (n, m) in enumerate(zip(st["lens"], st["new"])):
        K, V = _gather(st, "k", b), _gather(st, "v", b)
        hidden = None
        if m > 1:
            hidden = torch.arange(n, device="cuda")[None, None, :] > torch.arange(n - m, n, device="cuda")[:, None, None]
        for h in range(H):
            x = q[at:at + m, h * G:(h + 1) * G].float().reshape(m * G, D)
            s = (x @ K[h].T) * (1.0 / math.sqrt(D))
            if hidden is not None:
                s.view(m, G, n).masked_fill_(hidden, float("-inf"))
            s = torch.exp(s - s.amax(dim=1, keepdim=True))
            o = (s @ V[h]) / s.sum(dim=1, keepdim=True)
            out[at:at + m, h * G:(h + 1) * G] = o.reshape(m, G, D).to(out.dtype)
        at += m
    return out


def _run_load(st):
    if own:
        st["pg"].load(st["kv_len"], st["table"], st["k_pages"], st["v_pages"], st["k_scale"], st["v_scale"], st["L"], st["K_out"],
                      st["V_out"])
        return [st["K_out"], st["V_out"]]
    for which, out in (("k", st["K_out"]), ("v", st["V_out"])):
        for b, n in enumerate(st["lens"]):
            out[b, :, :n] = _gather(st, which, b)[:, :st["L"]].to(out.dtype)
            out[b, :, n:] = 0
    return [st["K_out"], st["V_out"]]


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    page = case["page"]
    if case["op"] == "tables":
        B, tokens = case["B"], case["tokens"]
        fresh = tokens // page + 1
        gone = case["finished"] * _pages(case["longest"] * 3 // 4, page)
        # lengths and counts in, lengths and starts out; a slot for every token; new entries from the stack, pages back onto it
        return {"bytes": 4 * (2 * B + 2 * B + 1 + tokens + 2 * fresh + 2 * gone), "flops": 0}
    H, lens, size = case["H"], _ints(case["lens"]), 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "store":
        n = sum(_ints(case["new"]))
        blocks = sum(_pages(a, page) - (a - b) // page for a, b in zip(lens, _ints(case["new"])))
        return {"bytes": 2 * (n * H * D * (size + 1) + blocks * H * 4) + 4 * n, "flops": 4 * n * H * D}
    blocks = sum(_pages(n, page) for n in lens)
    cached = 2 * sum(lens) * H * D + 2 * blocks * H * 4 + 4 * blocks + 4 * len(lens)
    if case["op"] == "load":
        return {"bytes": cached + 2 * len(lens) * case["L"] * H * D * size, "flops": 2 * sum(lens) * H * D}
    new = _ints(case["new"]) or [1] * len(lens)
    HQ = H * case["G"]
    pairs = sum(m * (n - m) + m * (m + 1) // 2 for n, m in zip(lens, new))
    return {"bytes": cached + 2 * sum(new) * HQ * D * size, "flops": 4 * pairs * HQ * D}


# ---------------------------------------------------------------------------------------------------- from the definitions, in 64 bits

def _bits(x):
    """The value of each e4m3 code, from its bits: sign, 4 exponent bits (bias 7), 3 bits behind the point; no infinities."""
    c = np.arange(256)
    s, e, m = c >> 7, (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0)) * np.where(s == 1, -1.0, 1.0)
    v[[127, 255]] = np.nan
    return torch.as_tensor(v, device=x.device, dtype=torch.float64)[x.view(torch.uint8).long()]


def exact(case, seed):
    if case["op"] == "tables":
        return _exact_tables(case, seed)
    st = prepare(case, seed)
    return {"store": _exact_store, "attn": _exact_attn, "load": _exact_load}[case["op"]](case, st)


def _exact_tables(case, seed):
    st = _prepare_tables(case, seed)
    page = case["page"]
    t, n = st["t_len"].tolist(), st["n_new"].tolist()
    table, free = st["table"].cpu().numpy().copy(), st["free_pages"].cpu().numpy().copy()
    height, tokens = int(st["n_free"].item()), st["slots"].numel()
    for b in range(len(t)):
        if n[b] < 0:
            for j in range(_pages(t[b], page)):
                free[height] = table[b, j]
                height += 1
    kv, start, slots, stuck = [], [0], [-1] * tokens, False
    for b in range(len(t)):
        m = max(n[b], 0)
        first = start[-1]
        start.append(first + m)
        if n[b] < 0:
            kv.append(0)
            continue
        have, want = _pages(t[b], page), _pages(t[b] + m, page)
        if want > table.shape[1] or first + m > tokens or (want > have and (stuck or want - have > height)):
            stuck = stuck or (want <= table.shape[1] and first + m <= tokens)
            kv.append(t[b])
            continue
        for j in range(have, want):
            height -= 1
            table[b, j] = free[height]
        kv.append(t[b] + m)
        for i in range(m):
            slots[first + i] = int(table[b, (t[b] + i) // page]) * page + (t[b] + i) % page
    return [torch.as_tensor(np.asarray(x, dtype=np.int32)) for x in (table, free, [height], start, kv, slots)]


def _exact_store(case, st):
    page, slots = case["page"], st["slots"].tolist()
    rows = {}
    for i, s in enumerate(slots):
        rows.setdefault(s // page, []).append((s % page, i))
    out = []
    for x, codes, scales in ((st["k_new"], st["k_pages"], st["k_scale"]), (st["v_new"], st["v_pages"], st["v_scale"])):
        x = x.double()
        code = codes.clone()
        scale = scales.double()
        for p, got in rows.items():
            r = torch.tensor([a for a, _ in got], device="cuda")
            i = torch.tensor([c for _, c in got], device="cuda")
            lo = got[0][0]
            amax = x[i].abs().amax(dim=(0, 2))                       # [H]
            s = torch.exp2(torch.ceil(torch.log2(amax / E4M3_MAX)).clamp(min=-126))
            if lo > 0:
                s = torch.maximum(s, scale[p])
                before = _bits(codes[p, :, :lo]) * scale[p][:, None, None] / s[:, None, None]
                code[p, :, :lo] = before.to(torch.float8_e4m3fn)
            scale[p] = s
            code[p, :, r] = (x[i].transpose(0, 1) / s[:, None, None]).to(torch.float8_e4m3fn)
        out += [code, scale]
    return out


def _values(st, which, b):
    n, page = st["lens"][b], st["page"]
    ids = st["table"][b, :_pages(n, page)].long()
    x = _bits(st[which + "_pages"][ids]) * st[which + "_scale"].double()[ids][:, :, None, None]
    return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :n]


def _exact_attn(case, st):
    H, G = case["H"], case["G"]
    out = st["out"].double()
    at = 0
    for b, (n, m) in enumerate(zip(st["lens"], st["new"])):
        K, V = _values(st, "k", b), _values(st, "v", b)
        for i in range(0, m, 256):                                   # 256 queries at a time
            k = min(256, m - i)
            seen = n - m + i + torch.arange(1, k + 1, device="cuda")
            hi = n - m + i + k
            x = st["q"][at + i:at + i + k].double().reshape(k, H, G, D)
            s = torch.einsum("mhgd,hnd->hgmn", x, K[:, :hi]) / math.sqrt(D)
            s = torch.where(torch.arange(hi, device="cuda") < seen[:, None], s, -math.inf)
            out[at + i:at + i + k] = torch.einsum("hgmn,hnd->mhgd", torch.softmax(s, dim=-1), V[:, :hi]).reshape(k, H * G, D)
        at += m
    return out


def _exact_load(case, st):
    res = []
    for which in ("k", "v"):
        y = torch.zeros(st["K_out"].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(st["lens"]):
            y[b, :, :n] = _values(st, which, b)
        res.append(y)
    return res
