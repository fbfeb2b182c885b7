"""Attention over the paged 8-bit cache where its arithmetic could lose something, element by element.

The bound of an element is what the call's stated rounding allows, in the element's own terms: half a step of the output type,
and relative errors of the weights times sum_n w[n] |V[n]|, not a share of the largest value in the cache."""
import math

import numpy as np
import pytest
import torch

import pages_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def fk():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2507_20030_b200 import binding, build
    build.build()
    binding.load()
    return binding


# What the header states: a weight's relative error, its floor (in units of the largest weight), an element of q in units of its
# row's largest.  `wide`: bf16 calls with more than eight query columns a sequence.
WEIGHT = {"wide": 2.0 ** -11, "bf16": 2.0 ** -12, "f32": 2.0 ** -24}
FLOOR = {"wide": 2.0 ** -31, "bf16": 2.0 ** -34, "f32": 2.0 ** -46}
QUERY = {"wide": 2.0 ** -17, "bf16": 2.0 ** -17, "f32": 2.0 ** -30}


def check(kind, got, q, K, V, seen, scale=1.0 / math.sqrt(128), floor_v=None):
    """got, q [m, 128] of one kv head, K, V [n, 128], seen [m]: how many tokens each row sees.  Everything in 64 bits.
    floor_v: the largest |V| among the tokens that count, where that is not the largest of all.

    Scores: the products that are not zero added up in float32 (an addition may cut off a whole step, 2^-23 of the sum of
    magnitudes), q's rounding, and three float32 roundings of exponents of up to twice the largest score in base 2; all of
    it moves the numerator and the denominator.  2^-21: exp2 and the division.  Sums of n terms in steps of 16 at least."""
    n = int(seen.max())
    q, K, V = q.double(), K[:n].double(), V[:n].double()
    s = (q @ K.T) * scale
    hidden = torch.arange(n, device=s.device)[None, :] >= seen[:, None]
    w = torch.softmax(s.masked_fill(hidden, -math.inf), dim=1)
    want, share = w @ V, w @ V.abs()
    size = ((q.abs() @ K.abs().T) * scale * (K != 0).sum(dim=1)).masked_fill(hidden, 0.0).amax(dim=1)
    k_sum = K.abs().sum(dim=1).max() * scale
    top_s = s.abs().masked_fill(hidden, 0.0).amax(dim=1)
    score = 2.0 ** -23 * size + QUERY[kind] * q.abs().amax(dim=1) * k_sum + 3 * 2.0 ** -24 * 2 * top_s
    rel = WEIGHT[kind] + 2 * score + 2.0 ** -21 + (n / 16) * 2.0 ** -23
    half = 2.0 ** -24 if kind == "f32" else 2.0 ** -8
    floor = FLOOR[kind] * n * w.amax(dim=1) * (V.abs().max() if floor_v is None else floor_v)
    tol = half * want.abs() + (1 + half) * (rel[:, None] * share + floor[:, None])
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (float((err / tol).max()), float(err.max()), float(want.abs().mean()))


def sequence(rng, n, H, page, loud, value, spread=1.0, mean=0.5):
    """Pages of one sequence, as a float64 K, V [H, n, 128] on the GPU and the call's tensors.  Channel 0 of the keys is loud
    (16) at the first token and zero elsewhere, so that q[0] sets how loud that token is; its value is near zero or like the others'."""
    n_pages = ref.pages_of(n, page)
    table = rng.permutation(n_pages)
    K = rng.standard_normal((H, n, 128)) * spread
    K[:, :, 0] = 0.0
    K[:, 0] = 0.0
    K[:, 0, 0] = 16.0
    V = rng.standard_normal((H, n, 128)) + mean
    if value == "zero":
        V[:, 0] *= 2.0 ** -6
    codes, dense = [], []
    for x, s in ((K, 2.0 ** -4), (V, 2.0 ** -5)):
        c = np.zeros((n_pages, H, page, 128), dtype=np.uint8)
        pad = np.zeros((H, n_pages * page, 128))
        pad[:, :n] = x / s
        c[table] = ref.encode(pad.reshape(H, n_pages, page, 128).transpose(1, 0, 2, 3))
        codes.append(ref.cuda8(c))
        dense.append(torch.from_numpy(np.ascontiguousarray(ref.VALUES[ref.encode(pad)][:, :n] * s)).cuda())
    scales = [torch.full((n_pages, H), s, dtype=torch.float32, device="cuda") for s in (2.0 ** -4, 2.0 ** -5)]
    return table, codes, scales, dense


def queries(rng, rows, heads, loud, dtype):
    """q whose scores are N(0, 1) against the sequence's tokens and `loud` against the first."""
    q = rng.standard_normal((rows, heads, 128))
    q[:, :, 0] = loud * math.sqrt(128) / 16.0
    return torch.from_numpy(q).to(dtype).cuda()


def run(fk, dtype, q, G, page, table, codes, scales, n, B, new):
    """One call in which B sequences share the same pages; `new` tokens of each (None: a decode step)."""
    H = scales[0].shape[1]
    n_pages = len(table)
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=n_pages, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    out = torch.full_like(q, 7.0)
    start = None if new is None else ref.ints(np.arange(B + 1) * new)
    pg.attn(q, ref.ints([n] * B), ref.ints(np.tile(table, (B, 1))), *codes, *scales, out, q_start=start)
    assert pg.device_status() == 0
    pg.close()
    return out


# ------------------------------------------------------------------------------------------------ a loud token

@pytest.mark.parametrize("value", ["zero", "ordinary"])
@pytest.mark.parametrize("loud", [8.0, 10.0, 12.0])
def test_many_columns_beside_a_loud_token(fk, loud, value):
    """A first token 8 to 12 nats above 18431 others (an attention sink), enough units for most to lie in one CTA."""
    rng = np.random.default_rng(int(loud))
    n, G, B, new = 18432, 8, 60, 32
    table, codes, scales, (K, V) = sequence(rng, n, 1, 64, loud, value)
    q = queries(rng, B * new, G, loud, torch.bfloat16)
    out = run(fk, torch.bfloat16, q, G, 64, table, codes, scales, n, B, new)
    seen = (n - new + 1 + torch.arange(new, device="cuda")).repeat_interleave(G)
    for b in range(0, B, 7):
        rows = slice(b * new, (b + 1) * new)
        check("wide", out[rows].reshape(-1, 128), q[rows].reshape(-1, 128), K[0], V[0], seen)


@pytest.mark.parametrize("value", ["zero", "ordinary"])
def test_many_columns_of_equal_scores_beside_a_loud_token(fk, value):
    """All other scores equal: no error of a weight averages out."""
    rng = np.random.default_rng(3)
    n, G, B, new = 18432, 8, 60, 32
    table, codes, scales, (K, V) = sequence(rng, n, 1, 64, 9.8, value, spread=0.0)
    q = queries(rng, B * new, G, 9.8, torch.bfloat16)
    out = run(fk, torch.bfloat16, q, G, 64, table, codes, scales, n, B, new)
    seen = (n - new + 1 + torch.arange(new, device="cuda")).repeat_interleave(G)
    check("wide", out[:new].reshape(-1, 128), q[:new].reshape(-1, 128), K[0], V[0], seen)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("loud,spread", [(10.0, 1.0), (12.0, 1.0), (12.0, 0.0), (14.0, 0.0)])
def test_decode_beside_a_loud_token(fk, dtype, loud, spread):
    """The same in decode steps: more sequences than CTAs, so that whole sequences lie in one."""
    rng = np.random.default_rng(int(loud) + int(spread))
    n, G, B = 16384 if dtype == torch.bfloat16 else 4096, 4, 600
    table, codes, scales, (K, V) = sequence(rng, n, 1, 64, loud, "zero", spread=spread)
    if dtype == torch.float32:                             # the loud value at zero: what remains is the others'
        V[:, 0] = 0.0
        codes[1][int(table[0]), 0, 0] = 0.0
    q = queries(rng, B, G, loud, dtype)
    out = run(fk, dtype, q, G, 64, table, codes, scales, n, B, None)
    kind = "bf16" if dtype == torch.bfloat16 else "f32"
    rows = slice(0, 160)
    check(kind, out[rows].reshape(-1, 128), q[rows].reshape(-1, 128), K[0], V[0], torch.full((160 * G,), n, device="cuda"))


# ------------------------------------------------------------------------------------------------ loud queries

@pytest.mark.parametrize("louder", [2.0 ** 4, 2.0 ** 8, 2.0 ** 12, 2.0 ** 18])
@pytest.mark.parametrize("where", ["head", "token"])
def test_a_loud_query_among_quiet_ones(fk, louder, where):
    """One head, or one token, has a loud element (on a channel where the keys are zero): the rows beside it keep their bits."""
    rng = np.random.default_rng(int(math.log2(louder)))
    n, G, B, new = 600, 4, 3, 40
    table, codes, scales, (K, V) = sequence(rng, n, 2, 32, 0.0, "ordinary")
    codes[0].view(torch.uint8)[int(table[0]), :, 0] = 0
    K[:, 0] = 0.0
    q = queries(rng, B * new, 2 * G, 0.0, torch.bfloat16)
    if where == "head":
        q[:, 2, 0] = louder
    else:
        q[::7, :, 0] = louder
    out = run(fk, torch.bfloat16, q, G, 32, table, codes, scales, n, B, new)
    seen = (n - new + 1 + torch.arange(new, device="cuda")).repeat_interleave(G)
    for b in range(B):
        for h in range(2):
            at = (slice(b * new, (b + 1) * new), slice(h * G, (h + 1) * G))
            check("wide", out[at].reshape(-1, 128), q[at].reshape(-1, 128), K[h], V[h], seen)


# ------------------------------------------------------------------------------------------------ pages of different scales

@pytest.mark.parametrize("kind", ["wide", "bf16", "f32"])
@pytest.mark.parametrize("at", [1, 40])
def test_a_page_of_loud_values_that_hardly_counts(fk, kind, at):
    """One page's values are 2^19 times the others' and its tokens' scores 42 nats down, so that it adds 2^-40 of the output:
    the other pages, with a loud token of their own and equal scores, keep their weights' bits wherever the loud page stands."""
    rng = np.random.default_rng(at)
    n, page, G, loud = 4096, 64, 8, 9.8
    B, new = (150, 16) if kind == "wide" else (600, None)
    dtype = torch.float32 if kind == "f32" else torch.bfloat16
    table, codes, scales, (K, V) = sequence(rng, n, 1, page, loud, "zero", spread=0.0)
    rows = slice(at * page, (at + 1) * page)
    codes[0][int(table[at]), 0, :, 1] = -448.0
    K[0, rows, 1] = -28.0
    scales[1][int(table[at])] *= 2.0 ** 19
    V[0, rows] *= 2.0 ** 19
    q = queries(rng, B * (new or 1), G, loud, dtype)
    q[:, :, 1] = 17.0                                      # 17 * 28 / sqrt(128) = 42
    out = run(fk, dtype, q, G, page, table, codes, scales, n, B, new)
    m = new or 4
    seen = (n - m + 1 + torch.arange(m, device="cuda")) if new else torch.full((m,), n, device="cuda")
    # what the loud page adds is counted as an error of its own share, not as the scale of the others' floor
    check(kind, out[:m].reshape(-1, 128), q[:m].reshape(-1, 128), K[0], V[0], seen.repeat_interleave(G), floor_v=V[0, :page].abs().max())


# ------------------------------------------------------------------------------------------------ shapes

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pow2", [True, False])
@pytest.mark.parametrize("page,H,G,lens,new", [
    (16, 2, 4, [127, 128, 129, 1], None), (128, 1, 7, [2500, 3], None), (32, 3, 1, [5000], None), (64, 1, 8, [640, 12000], None),
    (16, 1, 3, [700, 129, 64], [43, 1, 64]), (64, 2, 5, [5000], [40]), (128, 1, 8, [900, 260], [100, 250]), (32, 1, 2, [2100, 31], [3, 1]),
])
def test_every_element_within_its_own_rounding(fk, dtype, pow2, page, H, G, lens, new):
    """Random pages of different scales, ragged lengths, both widths: the bound of every element is its own."""
    rng = np.random.default_rng(sum(lens) + page + pow2)
    B, W = len(lens), max(ref.pages_of(n, page) for n in lens)
    n_pages = sum(ref.pages_of(n, page) for n in lens) + 1
    table = ref.spread(lens, page, n_pages, W, rng)
    kc, ks = ref.random_cache(rng, n_pages, H, page, lens, table, pow2)
    vc, vs = ref.random_cache(rng, n_pages, H, page, lens, table, pow2)
    n_new = new or [1] * B
    start = np.concatenate([[0], np.cumsum(n_new)])
    q = torch.from_numpy(rng.standard_normal((int(start[-1]), H * G, 128))).to(dtype).cuda()
    pg = fk.Pages(n_kv_heads=H, n_q_heads=H * G, page_size=page, n_pages=n_pages, max_pages=W, max_batch=B,
                  kv_dtype=fk.BF16 if dtype == torch.bfloat16 else fk.F32)
    out = torch.full_like(q, 7.0)
    pg.attn(q, ref.ints(lens), ref.ints(table), ref.cuda8(kc), ref.cuda8(vc), ref.cuda32(ks), ref.cuda32(vs), out,
            q_start=None if new is None else ref.ints(start))
    assert pg.device_status() == 0
    kind = "f32" if dtype == torch.float32 else "wide" if new and int(start[-1]) * G > 8 * B else "bf16"
    for b, (n, m) in enumerate(zip(lens, n_new)):
        K, V = [torch.from_numpy(ref.rows_of(c, s, table[b], n, page)).cuda() for c, s in ((kc, ks), (vc, vs))]
        seen = (n - m + 1 + torch.arange(m, device="cuda")).repeat_interleave(G)
        for h in range(H):
            at = (slice(int(start[b]), int(start[b + 1])), slice(h * G, (h + 1) * G))
            check(kind, out[at].reshape(-1, 128), q[at].reshape(-1, 128), K[h], V[h], seen)
