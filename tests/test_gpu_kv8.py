"""The 8-bit paged cache and attention over it (jf_op_kv8_*) against plain 64-bit arithmetic.

Tolerances. A held value is the code nearest to x' / 2^e: at most half a code step from x', plus what fp32 leaves of the
rotation (two products and a sum, each rounded once: 3 * 2^-24 of the operands' magnitude). Attention: with A =
sum p |v| and dS the largest error of a score (a sum of hd products in fp32: hd * 2^-24 of sum |q k|, times 2 for the
scaling steps), the output is within (2 dS + P) A + its own rounding of the exact one, P the rounding of a probability:
2^-11 for one fp16 term (bf16 models), 2^-20 for two (fp32; ex2 and the sums included), and 2^-8 |out| for bf16 outputs.
"""
import ctypes as C

import numpy as np
import pytest

from tests.parity import need_gpu

pytestmark = pytest.mark.gpu

PAGE, NAN_CODE = 16, 0x7F


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


def decode(codes):
    """e4m3 values in 64 bits."""
    c = codes.astype(np.int64)
    x, m = (c >> 3) & 15, (c & 7).astype(np.float64)
    mag = np.where(x > 0, (1 + m / 8) * 2.0 ** (x - 7.0), m / 8 * 2.0 ** -6)
    return np.where(c & 128, -mag, mag)


def step_of(y):
    """Distance of neighbouring e4m3 values at magnitude y."""
    y = np.maximum(np.abs(y), 2.0 ** -6)
    return 2.0 ** (np.floor(np.log2(y)) - 3)


def nearest(y):
    s = step_of(y)
    return np.clip(np.round(y / s) * s, -448, 448)


def need_exponent(amax):
    e = np.full(amax.shape, -120.0)
    some = amax > 0
    e[some] = np.ceil(np.log2(amax[some] / 448))
    e[some] += (amax[some] > 448 * 2.0 ** e[some])  # (log2 may round down at a boundary)
    e[some] -= (amax[some] <= 448 * 2.0 ** (e[some] - 1))
    return np.clip(e, -120, 119)


class Pool:
    """A cache in scrambled page order, every byte of it arbitrary until written."""

    def __init__(self, torch, per_seq, Hkv, hd, seed=0, spare=2):
        from paper_2512_14681_gb300.kv8 import Kv8Cache

        n = sum(per_seq) + spare
        order = np.random.default_rng(seed).permutation(n)
        table = np.full((len(per_seq), max(per_seq)), -1, np.int32)
        at = 0
        for b, p in enumerate(per_seq):
            table[b, :p] = order[at:at + p]
            at += p
        self.table, self.torch = table, torch
        self.cache = Kv8Cache(torch.full((n, Hkv, PAGE, hd), NAN_CODE, dtype=torch.uint8, device="cuda"),
                              torch.full((n, Hkv, PAGE, hd), 0xFF, dtype=torch.uint8, device="cuda"),
                              torch.full((n, Hkv), 77, dtype=torch.int8, device="cuda"),
                              torch.full((n, Hkv), -77, dtype=torch.int8, device="cuda"), torch.from_numpy(table).cuda())

    def held(self, b, slots):
        """(k, v) of a sequence's slots [0, slots) in 64 bits, [slots][Hkv][hd], and their exponents [pages][Hkv]."""
        pages = self.table[b, :-(-slots // PAGE)]
        out = []
        for codes, exps in ((self.cache.k, self.cache.k_exp), (self.cache.v, self.cache.v_exp)):
            e = exps.cpu().numpy()[pages].astype(np.float64)
            x = decode(codes.cpu().numpy()[pages]) * 2.0 ** e[:, :, None, None]
            out += [x.transpose(0, 2, 1, 3).reshape(-1, x.shape[1], x.shape[3])[:slots], e]
        return out[0], out[2], out[1], out[3]


def rows_of(new, lens):
    from paper_2512_14681_gb300.kv8 import Rows

    return Rows.of(new, lens)


def rotate(x, cs):
    half = x.shape[-1] // 2
    a, b, c, s = x[..., :half], x[..., half:], cs[:, None, :, 0], cs[:, None, :, 1]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


APPENDS = [  # Hq, Hkv, hd, new, lens, source, out, candidates' positions, how the rows lie
    (28, 4, 128, [1], [1003], "bf16", "bf16", False, "packed"),
    (28, 4, 128, [1, 1, 1], [0, 15, 16], "bf16", "f32", False, "packed"),
    (12, 2, 128, [43, 56, 0, 51], [777, 16, 5, 0], "f32", "bf16", True, "packed"),
    (8, 8, 64, [17, 100], [31, 1], "bf16", "bf16", False, "odd"),
    (4, 2, 64, [19, 3], [777, 14], "f32", "f32", False, "odd"),
    (16, 1, 128, [33], [7], "bf16", "bf16", False, "separate"),
    (6, 2, 64, [16, 16, 16], [0, 16, 8], "f32", "f32", True, "separate"),
]


@pytest.mark.parametrize("Hq,Hkv,hd,new,lens,src,dst,tree,lie", APPENDS)
def test_append_rotates_and_rounds_to_the_nearest_code(torch, Hq, Hkv, hd, new, lens, src, dst, tree, lie):
    from paper_2512_14681_gb300.kv8 import rope_table

    types = {"bf16": torch.bfloat16, "f32": torch.float32}
    R, width = sum(new), (Hq + 2 * Hkv) * hd
    g = torch.Generator(device="cuda").manual_seed(R)
    pool = Pool(torch, [-(-(a + n) // PAGE) or 1 for a, n in zip(lens, new)], Hkv, hd)
    pad = {"packed": 0, "odd": 3, "separate": 0}[lie]
    store = torch.randn(R * (width + pad) + 1, generator=g, device="cuda").to(types[src])
    qkv = store[1 if lie == "odd" else 0:][:R * (width + pad)].view(R, width + pad)[:, :width]
    q, k, v = qkv.split([Hq * hd, Hkv * hd, Hkv * hd], 1)
    if lie == "separate":
        q, k, v = (t.contiguous().view(R, -1, hd) for t in (q, k, v))
    rope = rope_table(1200, hd, 1e4)
    # (positions past a context, in a candidate's order)
    pos = np.concatenate([a + (np.arange(n) % 8 if tree else np.arange(n)) for a, n in zip(lens, new)]).astype(np.int32)
    # what the blocks hold before: the tokens below each length, appended first
    seed_rows = rows_of(lens, [0] * len(lens))
    n0 = sum(lens)
    if n0:
        kk = torch.randn(n0, Hkv, hd, generator=g, device="cuda") * 0.3
        pool.cache.append(seed_rows, kk, kk * 2)
    before = [pool.held(b, a) for b, a in enumerate(lens)]
    got_q = pool.cache.append(rows_of(new, lens), k, v, q=q, rope=rope, positions=torch.from_numpy(pos).cuda() if tree else None,
                              q_dtype=types[dst])
    pool.cache.check()
    f64 = lambda t: t.reshape(R, -1, hd).double().cpu().numpy()
    cs = rope.double().cpu().numpy()[pos]
    xk, xv, xq = rotate(f64(k), cs), f64(v), rotate(f64(q), cs)
    size = lambda x: np.sqrt(x[..., :hd // 2] ** 2 + x[..., hd // 2:] ** 2).repeat(2, -1).reshape(*x.shape[:-1], hd // 2, 2)
    mag = lambda x: np.concatenate([size(x)[..., 0], size(x)[..., 1]], -1)
    tol_q = 3 * 2.0 ** -24 * 1.5 * mag(f64(q)) + (2.0 ** -8 * np.abs(xq) if dst == "bf16" else 2.0 ** -24 * np.abs(xq))
    assert got_q.dtype == types[dst]
    assert (np.abs(got_q.double().cpu().numpy() - xq) <= tol_q + 1e-30).all()
    r = 0
    for b, (a, n) in enumerate(zip(lens, new)):
        hk, hv, ek, ev = pool.held(b, a + n)
        for held, x, e, old, eps in ((hk, xk, ek, before[b][0], 3 * 2.0 ** -24 * 1.5 * mag(f64(k))), (hv, xv, ev, before[b][1], None)):
            new_x = x[r:r + n]
            slot = np.arange(a, a + n)
            unit = 2.0 ** e[slot // PAGE][:, :, None]
            off = np.abs(held[a:] - new_x)
            half = step_of(np.maximum(np.abs(held[a:]), np.abs(new_x)) / unit) * unit / 2
            assert (off <= half + (eps[r:r + n] if eps is not None else 0)).all()
            for p in range(a // PAGE, -(-(a + n) // PAGE) if n else 0):  # the smallest exponent, or the block's own
                rows = new_x[(slot // PAGE) == p]
                amax = np.abs(rows).max((0, 2))
                need = need_exponent(amax)
                close = np.abs(amax / (448 * 2.0 ** np.round(np.log2(amax / 448))) - 1) < 1e-6
                if p * PAGE < a:
                    need = np.maximum(need, before[b][2 if x is xk else 3][p])
                assert ((e[p] == need) | close).all()
            # earlier tokens: untouched where the exponent did not grow, else rounded once more
            keep = np.arange(a)
            u = 2.0 ** e[keep // PAGE][:, :, None]
            assert (held[:a] == nearest(old / u) * u).all()
        r += n
    # the same values through read()
    rd = pool.cache.read(rows_of(new, lens), torch.float32)
    r = 0
    for b, (a, n) in enumerate(zip(lens, new)):
        hk, hv, _, _ = pool.held(b, a + n)
        assert (rd[0][r:r + n].double().cpu().numpy() == hk[a:]).all() and (rd[1][r:r + n].double().cpu().numpy() == hv[a:]).all()
        r += n


def test_a_block_that_grows_rounds_what_it_holds_and_a_rejected_draft_is_replaced(torch):
    pool = Pool(torch, [3], 2, 64)
    g = torch.Generator(device="cuda").manual_seed(5)
    small = torch.randn(20, 2, 64, generator=g, device="cuda") * 0.01
    pool.cache.append(rows_of([20], [0]), small, small)
    k0, _, e0, _ = pool.held(0, 20)
    big = torch.randn(9, 2, 64, generator=g, device="cuda") * 300
    pool.cache.append(rows_of([9], [20]), big, big)  # a draft, rejected
    k1, _, e1, _ = pool.held(0, 29)
    assert (e1[0] == e0[0]).all() and (e1[1] > e0[1] + 8).all()
    u = 2.0 ** e1[1][None, :, None]
    assert (k1[:16] == k0[:16]).all() and (k1[16:20] == nearest(k0[16:20] / u) * u).all()
    pool.cache.append(rows_of([1], [20]), small[:1], small[:1])  # the next one starts at the accepted length
    k2, _, e2, _ = pool.held(0, 21)
    assert (e2[1] == e1[1]).all() and (k2[:20] == k1[:20]).all()
    # a fresh start in the same page forgets the exponent
    pool.cache.append(rows_of([4], [16]), small[:4], small[:4])
    _, _, e3, _ = pool.held(0, 20)
    assert (e3[1] < e1[1]).all()
    pool.cache.check()


def test_append_at_the_ends_of_the_range(torch):
    """Blocks of zeros, of the smallest and of the largest fp32 values; a boundary amax = 448 * 2^e; no rope, no queries."""
    pool = Pool(torch, [5], 1, 64)
    x = torch.zeros(80, 1, 64, device="cuda")
    x[16:32] = 1e-38
    x[32:48] = 2.9e38
    x[33, 0, 3] = 3.4e38      # beyond 448 * 2^119: held as that
    x[48, 0, 0] = 448.0       # e = 0 exactly
    x[64, 0, 0] = float(np.nextafter(np.float32(448.0), np.float32(1e9)))  # one more unit: e = 1
    pool.cache.append(rows_of([80], [0]), x, -x)
    pool.cache.check()
    k, v, ek, ev = pool.held(0, 80)
    assert ek[:, 0].tolist() == ev[:, 0].tolist() == [-120, -120, 119, 0, 1]
    xd = x.double().cpu().numpy()
    u = 2.0 ** ek[np.arange(80) // PAGE][:, :, None]
    assert (k == nearest(xd / u) * u).all() and (v == -k).all()
    assert k[33, 0, 3] == 448 * 2.0 ** 119


@pytest.mark.parametrize("bad", ["nan", "inf", "-inf"])
def test_values_without_a_finite_form_are_reported_and_held_finite(torch, bad):
    from paper_2512_14681_gb300._lib import JfError

    pool = Pool(torch, [2], 2, 128)
    x = torch.ones(20, 2, 128, device="cuda", dtype=torch.bfloat16)
    x[3, 1, 100] = float(bad)
    pool.cache.append(rows_of([20], [0]), x, torch.ones_like(x))
    with pytest.raises(JfError, match="without a finite"):
        pool.cache.check()
    pool.cache.check()  # cleared
    k, v, ek, _ = pool.held(0, 20)
    want = np.ones((20, 2, 128))
    want[3, 1, 100] = {"nan": 0.0, "inf": 448 * 2.0 ** ek[0, 1], "-inf": -448 * 2.0 ** ek[0, 1]}[bad]
    assert (k == want).all() and (v == 1).all() and (ek == -8).all()


def test_indexes_out_of_range_are_reported_and_nothing_else_is_touched(torch):
    from paper_2512_14681_gb300._lib import JfError
    from paper_2512_14681_gb300.kv8 import Rows, rope_table

    x = torch.randn(8, 2, 64, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cases = {
        "a page beyond the pool": (dict(page=10 ** 6), Rows(i32(0, 8), i32(0), 8, 8)),
        "no page": (dict(page=-1), Rows(i32(0, 8), i32(0), 8, 8)),
        "longer than the table": ({}, Rows(i32(0, 8), i32(30), 8, 8)),
        "negative length": ({}, Rows(i32(0, 8), i32(-1), 8, 8)),
        "rows beyond the batch": ({}, Rows(i32(0, 9), i32(0), 8, 8)),
        "rows that fall": ({}, Rows(i32(8, 0), i32(0), 8, 8)),
    }
    for name, (how, rows) in cases.items():
        pool = Pool(torch, [2], 2, 64)
        if "page" in how:
            pool.cache.page_table[0, 0] = how["page"]
        for call in (lambda: pool.cache.append(rows, x, x), lambda: pool.cache.read(rows),
                     lambda: pool.cache.attention(rows, x, 0.1)):
            call()
            with pytest.raises(JfError, match="out of range"):
                pool.cache.check()
        assert (pool.cache.k == NAN_CODE).all() and (pool.cache.v == 0xFF).all(), name
    pool = Pool(torch, [2], 2, 64)
    pool.cache.append(rows_of([8], [0]), x, x, rope=rope_table(7, 64, 1e4))  # the last row's position has no entry
    with pytest.raises(JfError, match="out of range"):
        pool.cache.check()


def test_no_rows(torch):
    pool = Pool(torch, [1, 1], 2, 64)
    rows, x = rows_of([0, 0], [3, 0]), torch.empty(0, 2, 64, device="cuda")
    assert pool.cache.append(rows, x, x, q=x).shape == (0, 2, 64)
    assert pool.cache.read(rows)[0].shape == (0, 2, 64) and pool.cache.attention(rows, x, 1.0).shape == (0, 2, 64)
    pool.cache.check()


# ---------------------------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------------------------
def fill(torch, Hkv, hd, totals, seed, v_spread=0, k_spread=0):
    """A pool whose sequences hold `totals` tokens, codes at random; the values' (keys') exponents differ by up to
    v_spread (k_spread) from page to page."""
    pool = Pool(torch, [max(1, -(-t // PAGE)) for t in totals], Hkv, hd, seed)
    rng = np.random.default_rng(seed)
    c = pool.cache
    for codes, exps, spread, typical in ((c.k, c.k_exp, k_spread, -7), (c.v, c.v_exp, v_spread, -8)):
        x = rng.integers(0, 256, codes.shape).astype(np.uint8)
        x[(x & 127) == 127] = 0
        if codes is c.k:  # (a trained model's scores: mostly small products)
            x = np.where(rng.random(x.shape) < 0.9, x & 0xBF, x)
        e = typical + rng.integers(-spread, spread + 1, exps.shape)
        for b, t in enumerate(totals):
            if t % PAGE:
                x[pool.table[b, t // PAGE], :, t % PAGE:] = NAN_CODE
        used = np.concatenate([pool.table[b, :-(-t // PAGE)] for b, t in enumerate(totals)])
        unused = np.setdiff1d(np.arange(codes.shape[0]), used)
        x[unused] = NAN_CODE
        codes.copy_(torch.from_numpy(x))
        exps.copy_(torch.from_numpy(e.astype(np.int8)))
    return pool


def reference(pool, q, new, lens, scale, see=None):
    """(out, A = sum p |v|, lse, dS) in 64 bits; see(b): [n][len + n] truth values (None: causal)."""
    R, Hq, hd = q.shape
    Hkv = pool.cache.n_kv_heads
    out, A, lse, dS = np.zeros(q.shape), np.zeros(q.shape), np.full((R, Hq), -np.inf), np.zeros((R, Hq))
    r = 0
    for b, (a, n) in enumerate(zip(lens, new)):
        if n == 0:
            continue
        k, v, _, _ = pool.held(b, a + n)
        vis = see(b) if see else np.arange(a + n)[None, :] <= a + np.arange(n)[:, None]
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            qh = q[r:r + n, h]
            s = np.where(vis, qh @ k[:, kv].T * scale, -np.inf)
            m = s.max(1, keepdims=True)
            p = np.exp(s - np.where(m == -np.inf, 0, m))
            t = p.sum(1, keepdims=True)
            with np.errstate(divide="ignore"):
                lse[r:r + n, h] = (m + np.log(t))[:, 0]
            p = p / np.where(t > 0, t, 1)
            out[r:r + n, h], A[r:r + n, h] = p @ v[:, kv], p @ np.abs(v[:, kv])
            dS[r:r + n, h] = np.where(vis, np.abs(qh) @ np.abs(k[:, kv]).T * abs(scale), 0).max(1) * hd * 2.0 ** -23
        r += n
    return out, A, lse, dS


def check_attention(torch, pool, q, new, lens, scale, mask=None, see=None, max_rows=None, want_lse=True):
    rows = rows_of(new, lens)
    if max_rows:
        rows.c.max_rows = max_rows
    out, lse = pool.cache.attention(rows, q, scale, mask=mask, want_lse=want_lse)
    again = pool.cache.attention(rows, q, scale, mask=mask)
    pool.cache.check()
    assert torch.equal(out, again)  # the same bits each time
    ref, A, ref_lse, dS = reference(pool, q.reshape(q.shape[0], -1, pool.cache.head_dim).double().cpu().numpy(), new, lens, scale, see)
    bf16 = q.dtype == torch.bfloat16
    tol = (2 * dS + (2.0 ** -11 if bf16 else 2.0 ** -20))[..., None] * A + (2.0 ** -8 * np.abs(ref) if bf16 else 0) + 1e-37
    off = np.abs(out.double().cpu().numpy() - ref)
    assert (off <= tol).all(), (off / tol).max()
    got = lse.double().cpu().numpy()
    none = ref_lse == -np.inf
    assert (got[none] == -np.inf).all()
    assert (np.abs(got - ref_lse)[~none] <= (2 * dS + 1e-6 * (1 + np.abs(np.where(none, 0, ref_lse))))[~none]).all()
    return out


def queries(torch, R, Hq, hd, dtype, seed, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(R, Hq, hd, generator=g, device="cuda") * size).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


SHAPES = [  # Hq, Hkv, hd
    (28, 4, 128), (12, 2, 128), (8, 8, 64), (16, 1, 128), (4, 2, 64), (3, 3, 128), (40, 1, 64),
]
BATCHES = [  # new, lens
    ([1], [0]), ([1], [1]), ([1], [15]), ([1], [16]), ([1], [1023]), ([1], [5000]),
    ([2, 1, 0, 1], [63, 0, 9, 400]), ([5], [0]), ([17], [0]), ([37], [130]), ([64, 3], [0, 999]), ([130], [257]),
    ([1] * 20, [16 * i + i for i in range(20)]),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,hd", SHAPES)
def test_attention_over_lengths_and_rows(torch, dtype, Hq, Hkv, hd):
    for i, (new, lens) in enumerate(BATCHES):
        pool = fill(torch, Hkv, hd, [a + n for a, n in zip(lens, new)], seed=i)
        check_attention(torch, pool, queries(torch, sum(new), Hq, hd, dtype, i), new, lens, hd ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,lens", [([1], [3000]), ([9], [700]), ([50, 1], [40, 2000])])
def test_exponents_that_differ_from_page_to_page(torch, dtype, new, lens):
    """Values whose blocks differ by up to 2^40 (a page of small values that a row attends to keeps its precision beside
    pages of large ones), keys by up to 2^6."""
    for spread in (3, 10, 20):
        pool = fill(torch, 4, 128, [a + n for a, n in zip(lens, new)], seed=spread, v_spread=spread, k_spread=min(spread, 3))
        check_attention(torch, pool, queries(torch, sum(new), 28, 128, dtype, spread, 0.3), new, lens, 128 ** -0.5)


@pytest.mark.parametrize("dtype,n", [("bf16", 1), ("bf16", 40), ("f32", 3)])
def test_a_row_that_attends_to_small_values_only_keeps_their_precision(torch, dtype, n):
    """Every second page's values are 2^60 times the others', and the keys leave them no weight."""
    total = 600 + n
    pool = fill(torch, 2, 128, [total], seed=1)
    c = pool.cache
    pages = torch.from_numpy(pool.table[0].astype(np.int64)).cuda()
    c.v_exp[pages[0::2]] = 30
    c.v_exp[pages[1::2]] = -30
    c.k.zero_()
    c.k_exp.fill_(0)
    c.k[pages[0::2]] = 0x80 | 0x70  # -128 in every dim
    q = torch.full((n, 4, 128), 1.0, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    out = check_attention(torch, pool, q, [n], [600], 0.1)
    assert float(out.abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("e", [-120, -60, 60, 119])
def test_blocks_at_the_ends_of_the_exponents_range(torch, dtype, e):
    pool = fill(torch, 2, 64, [100], seed=3)
    pool.cache.v_exp.fill_(e)
    q = queries(torch, 7, 4, 64, dtype, 2)
    ref, A, _, dS = reference(pool, q.double().cpu().numpy(), [7], [93], 0.125)
    out = pool.cache.attention(rows_of([7], [93]), q, 0.125).double().cpu().numpy()
    bf16 = dtype == "bf16"
    tol = (2 * dS + (2.0 ** -11 if bf16 else 2.0 ** -20))[..., None] * A + (2.0 ** -8 * np.abs(ref) if bf16 else 0)
    tol += 2.0 ** -126 * (2.0 ** -7 if bf16 else 2.0 ** -22)  # subnormal results
    fits = np.abs(ref) < 3.3e38
    assert (np.abs(out - ref)[fits] <= tol[fits]).all()
    # the same exponents on the keys: with queries of the inverse size, the same scores
    pool = fill(torch, 2, 64, [100], seed=3)
    pool.cache.k_exp.fill_(max(min(e, 100), -100))
    check_attention(torch, pool, (q.double() * 2.0 ** (-7 - max(min(e, 100), -100))).to(q.dtype), [7], [93], 0.125)


def tree_bits(see, words):
    n = see.shape[0]
    bits = np.zeros((n, words * 32), np.uint8)
    bits[:, :see.shape[1]] = see
    return np.packbits(bits.reshape(n, words, 4, 8), axis=-1, bitorder="little").reshape(n, words * 4).view(np.int32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,hd", [(12, 2, 128), (8, 8, 64), (28, 4, 128)])
def test_masked_rows(torch, dtype, Hq, Hkv, hd):
    """Random visibility among the new rows, rows that see none of them, and, without a context, rows that see nothing."""
    new, lens = [45, 70, 1, 20, 1], [33, 0, 200, 1000, 0]
    rng = np.random.default_rng(4)
    sees = []
    for n, p in zip(new, (0.5, 0.3, 1.0, 0.0, 0.0)):
        s = rng.random((n, n)) < p
        s[rng.random(n) < 0.2] = False
        sees.append(s)
    words = 3
    mask = torch.from_numpy(np.concatenate([tree_bits(s, words) for s in sees])).cuda()
    pool = fill(torch, Hkv, hd, [a + n for a, n in zip(lens, new)], seed=9)
    vis = lambda b: np.concatenate([np.ones((new[b], lens[b]), bool), sees[b]], 1)
    out = check_attention(torch, pool, queries(torch, sum(new), Hq, hd, dtype, 8), new, lens, hd ** -0.5, mask, vis)
    assert not out[-1].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_what_a_row_does_not_see_does_not_reach_it(torch, dtype):
    """A NaN or an infinity in one row's query stays in that row; codes behind the last token, and pages of other
    sequences, are NaN codes in every test here."""
    new, lens = [30], [100]
    pool = fill(torch, 4, 128, [130], seed=2)
    q = queries(torch, 30, 28, 128, dtype, 3)
    want = pool.cache.attention(rows_of(new, lens), q, 0.1)
    for bad in (float("nan"), float("inf")):
        p = q.clone()
        p[11, 5, 77] = bad
        got = pool.cache.attention(rows_of(new, lens), p, 0.1)
        other = torch.ones(30, 28, dtype=torch.bool, device="cuda")
        other[11, 5] = False
        assert torch.equal(got[other], want[other])
        assert got[11, 5].isnan().any() or bad == float("inf")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_hint_of_the_row_count_and_any_row_stride(torch, dtype):
    new, lens = [3, 40, 1], [500, 77, 2100]
    pool = fill(torch, 4, 128, [a + n for a, n in zip(lens, new)], seed=6)
    q = queries(torch, 44, 28, 128, dtype, 6)
    wide = torch.full((44, 28 * 128 + 3), float("nan"), device="cuda", dtype=q.dtype)
    wide[:, 2:28 * 128 + 2] = q.view(44, -1)
    for hint in (1, 40, 44):
        a = check_attention(torch, pool, q, new, lens, 0.09, max_rows=hint)
        rows = rows_of(new, lens)
        rows.c.max_rows = hint
        assert torch.equal(pool.cache.attention(rows, wide[:, 2:28 * 128 + 2], 0.09), a)


@pytest.mark.parametrize("scale", [0.0, -0.1, 3.0])
def test_any_softmax_scale(torch, scale):
    pool = fill(torch, 2, 128, [330], seed=7)
    for n in (1, 30):
        check_attention(torch, pool, queries(torch, n, 12, 128, "f32", 7, 0.1), [n], [330 - n], scale)
        check_attention(torch, pool, queries(torch, n, 12, 128, "bf16", 7, 0.1), [n], [330 - n], scale)


def test_sharp_softmax_and_growing_maxima(torch):
    """Scores that climb with the position: the running maximum is raised again and again, by a little and by a lot."""
    for n, slope in ((1, 0.02), (1, 3.0), (33, 0.02), (33, 3.0)):
        total = 1500 + n
        pool = fill(torch, 1, 128, [total], seed=8)
        c = pool.cache
        c.k.zero_()
        order = pool.table[0].astype(np.int64)
        codes = np.zeros((c.k.shape[0], 1, PAGE, 128), np.uint8)
        exps = np.zeros((c.k.shape[0], 1), np.int8)
        for i, p in enumerate(order):
            exps[p] = int(np.ceil(np.log2(max(1, i) * slope / 16)))
            want = (16 * i + np.arange(PAGE)) * slope / 16 / 2.0 ** exps[p]
            value = torch.from_numpy(want.astype(np.float32)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
            codes[p, 0, :, 0] = value
        c.k.copy_(torch.from_numpy(codes))
        c.k_exp.copy_(torch.from_numpy(exps))
        for dtype in ("bf16", "f32"):
            q = torch.zeros(n, 4, 128, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
            q[:, :, 0] = 1.0
            check_attention(torch, pool, q, [n], [total - n], 1.0)


def test_a_long_cache(torch):
    """140,000 tokens; pages whose byte offset passes 2^31 in a pool of 2.3 GB."""
    from paper_2512_14681_gb300.kv8 import Kv8Cache

    total, n = 140001, 2
    per = -(-total // PAGE)
    pages = 290000
    pool = Pool.__new__(Pool)
    order = np.random.default_rng(1).permutation(pages)[:per]
    order[-1] = pages - 1
    pool.table, pool.torch = order[None].astype(np.int32), torch
    g = torch.Generator(device="cuda").manual_seed(1)
    codes = lambda: torch.randint(0, 0x60, (pages, 4, PAGE, 128), generator=g, device="cuda", dtype=torch.uint8)
    exps = torch.full((pages, 4), -8, dtype=torch.int8, device="cuda")
    pool.cache = Kv8Cache(codes(), codes(), exps, exps.clone(), torch.from_numpy(pool.table).cuda())
    for n in (1, 20):
        q = queries(torch, n, 4, 128, "bf16", 1)
        out = pool.cache.attention(rows_of([n], [total - n]), q, 0.1).double()
        pool.cache.check()
        k, v = (( (c.view(torch.float8_e4m3fn)[torch.from_numpy(order).cuda()].double() * 2.0 ** -8).transpose(1, 2).reshape(-1, 4, 128)[:total])
                for c in (pool.cache.k, pool.cache.v))
        s = torch.einsum("rhd,khd->rhk", q.double(), k) * 0.1
        late = torch.arange(total, device="cuda")[None, :] > (total - n + torch.arange(n, device="cuda"))[:, None]
        s = s.masked_fill(late[:, None], -float("inf"))
        p = torch.softmax(s, -1)
        ref, A = torch.einsum("rhk,khd->rhd", p, v), torch.einsum("rhk,khd->rhd", p, v.abs())
        dS = torch.einsum("rhd,khd->rhk", q.double().abs(), k.abs()).max(-1).values * 0.1 * 128 * 2.0 ** -23
        tol = (2 * dS + 2.0 ** -11)[..., None] * A + 2.0 ** -8 * ref.abs()
        assert ((out - ref).abs() <= tol).all()


def test_other_streams_and_a_captured_graph(torch):
    """Calls on a stream of their own, in order with what wrote their inputs there; a captured graph follows lengths and
    page table as they are when it is replayed."""
    pool = fill(torch, 4, 128, [400], seed=11)
    pool.cache.page_table = pool.cache.page_table  # (the tensor that the kernels read)
    q = queries(torch, 1, 28, 128, "bf16", 1)
    x = torch.randn(1, 4, 128, device="cuda").bfloat16()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        late = torch.zeros_like(q)
        torch.cuda._sleep(2_000_000)
        late.copy_(q)
    rows = rows_of([1], [300])
    torch.cuda.current_stream().synchronize()
    got = pool.cache.attention(rows, late, 0.1, stream=st)
    st.synchronize()
    assert torch.equal(got, pool.cache.attention(rows, q, 0.1))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    pool.cache.append(rows, x, x, stream=st)
    pool.cache.attention(rows, q, 0.1, stream=st)
    st.synchronize()
    with torch.cuda.graph(graph, stream=st):
        pool.cache.append(rows, x, x)
        out = pool.cache.attention(rows, q, 0.1)
    for n in (299, 17, 0, 350):
        rows.len.fill_(n)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        pool.cache.check()
        assert torch.equal(out, pool.cache.attention(rows_of([1], [n]), q, 0.1))


def test_refusals(torch):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300.kv8 import Kv8Cache, Rows, rope_table

    pool = Pool(torch, [2], 2, 64)
    c, rows = pool.cache, rows_of([4], [0])
    x, q = torch.zeros(4, 2, 64, device="cuda"), torch.zeros(4, 4, 64, device="cuda")

    def refused(status, f):
        with pytest.raises(J.JfError) as e:
            f()
        assert e.value.status == status, e.value

    inv, uns = J.JF_EINVAL, J.JF_EUNSUPPORTED
    refused(inv, lambda: c.append(rows, x[:3], x))
    refused(inv, lambda: c.append(rows, x, x.bfloat16()))
    refused(inv, lambda: c.append(rows, x, x, q=q[:, :3]))           # 3 heads on 2
    refused(inv, lambda: c.append(rows, x, x, rope=rope_table(9, 128, 1e4)))
    refused(inv, lambda: c.append(rows, x, x, positions=torch.zeros(3, dtype=torch.int32, device="cuda")))
    refused(uns, lambda: c.append(rows, x.half(), x.half()))
    refused(inv, lambda: c.append(rows_of([4, 0], [0, 0]), x, x))
    refused(inv, lambda: c.attention(rows, q[:, :3], 1.0))
    refused(inv, lambda: c.attention(rows, q.transpose(1, 2).contiguous().transpose(1, 2), 1.0))
    refused(inv, lambda: c.attention(rows, q, float("nan")))
    refused(inv, lambda: c.attention(rows_of([64], [0]), torch.zeros(64, 4, 64, device="cuda"), 1.0,
                                     mask=torch.zeros(64, 1, dtype=torch.int32, device="cuda")))  # 32 bits for 64 rows
    refused(uns, lambda: c.attention(rows, q.half(), 1.0))
    refused(uns, lambda: c.read(rows, torch.float16))
    refused(inv, lambda: Kv8Cache(c.k, c.v[:1], c.k_exp, c.v_exp, c.page_table))
    refused(inv, lambda: Kv8Cache(c.k, c.v, c.k_exp.int(), c.v_exp, c.page_table))
    refused(inv, lambda: Rows(torch.zeros(1, dtype=torch.int32, device="cuda"), rows.len, 4, 4))
    odd, few = torch.zeros(2, 2, PAGE, 32, dtype=torch.uint8, device="cuda"), torch.zeros(4, 2, 32, device="cuda")
    refused(uns, lambda: Kv8Cache(odd, odd, c.k_exp[:2], c.v_exp[:2], c.page_table).append(rows, few, few))
    # a workspace that is too small, through the C entry
    need = C.c_size_t()
    assert c.lib.jf_op_kv8_attention_workspace_bytes(C.byref(c.c), C.byref(rows.c), J.JF_F32, 4, C.byref(need)) == J.JF_OK
    ws = torch.empty(need.value, dtype=torch.uint8, device="cuda")
    args = (C.byref(c.c), C.byref(rows.c), J.JF_F32, q.data_ptr(), 256, 4, 1.0, None, 0, q.data_ptr(), None, ws.data_ptr())
    assert c.lib.jf_op_kv8_attention(*args, need.value - 1, c.err.data_ptr(), None) == J.JF_ENOMEM
    assert c.lib.jf_op_kv8_attention(*args, need.value, None, None) == J.JF_EINVAL
    torch.cuda.synchronize()
    c.check()


@pytest.mark.parametrize("spread", [0, 9, 25])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,hd,new,lens,masked", [
    (28, 4, 128, [64], [20000], False),              # two row tiles, several chunks of keys a CTA
    (28, 4, 128, [3, 64, 20], [9000, 20000, 130], False),  # units of one and of two tiles in one CTA's share
    (12, 2, 128, [40, 21], [12001, 25000], True),
    (8, 1, 64, [30, 100], [16383, 9000], False),
    (28, 4, 128, [1, 1, 2], [40000, 17, 21111], False),
])
def test_many_chunks_a_share(torch, Hq, Hkv, hd, new, lens, masked, dtype, spread):
    """Long contexts, so that every CTA walks through several chunks and units; values' exponents alike, or differing so much
    that the pages of a chunk go in several steps. (No launch runs into the limit of a wait, which is 2 s.)"""
    import time

    totals = [a + n for a, n in zip(lens, new)]
    pool = fill(torch, Hkv, hd, totals, seed=12, v_spread=spread)
    q = queries(torch, sum(new), Hq, hd, dtype, 5, 0.5)
    sees, mask = None, None
    if masked:
        rng = np.random.default_rng(6)
        sees = [rng.random((n, n)) < 0.5 for n in new]
        mask = torch.from_numpy(np.concatenate([tree_bits(s, 2) for s in sees])).cuda()
    scale = hd ** -0.5
    out = pool.cache.attention(rows_of(new, lens), q, scale, mask=mask)
    torch.cuda.synchronize()
    began = time.monotonic()
    again = pool.cache.attention(rows_of(new, lens), q, scale, mask=mask)
    pool.cache.check()
    assert time.monotonic() - began < 1.0
    assert torch.equal(out, again)
    r = 0
    for b, (a, n) in enumerate(zip(lens, new)):
        pages = torch.from_numpy(pool.table[b, :-(-(a + n) // PAGE)].astype(np.int64)).cuda()
        k, v = (((c[pages].view(torch.float8_e4m3fn).double() * 2.0 ** e[pages].double()[:, :, None, None]).transpose(1, 2).reshape(-1, Hkv, hd)[:a + n])
                for c, e in ((pool.cache.k, pool.cache.k_exp), (pool.cache.v, pool.cache.v_exp)))
        see = torch.ones(n, a + n, dtype=torch.bool, device="cuda")
        see[:, a:] = torch.from_numpy(sees[b]).cuda() if masked else torch.ones(n, n, device="cuda").tril().bool()
        for h in range(Hq):
            kv, qh = h // (Hq // Hkv), q[r:r + n, h].double()
            p = torch.softmax((qh @ k[:, kv].T * scale).masked_fill(~see, -float("inf")), -1)
            ref, A = p @ v[:, kv], p @ v[:, kv].abs()
            dS = (qh.abs() @ k[:, kv].abs().T).masked_fill(~see, 0).max(1).values * scale * hd * 2.0 ** -23
            tol = (2 * dS + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -20))[:, None] * A + (2.0 ** -8 * ref.abs() if dtype == "bf16" else 0)
            off = (out[r:r + n, h].double() - ref).abs()
            assert (off <= tol).all(), (b, h, float((off / tol).max()))
        r += n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,most", [(32, 3), (33, 2), (33, 14), (100, 3), (100, 40), (1024, 2), (1024, 6)])
def test_many_sequences(torch, dtype, n, most):
    """Batches on both sides of the 32 sequences that a warp plans by itself, up to the largest; some without rows."""
    rng = np.random.default_rng(n + most)
    new = [int(x) for x in rng.integers(0, most + 1, n)]
    new[n // 2] = most
    lens = [int(x) for x in rng.integers(0, 70, n)]
    lens[-1] = 900
    pool = fill(torch, 2, 64, [a + k for a, k in zip(lens, new)], seed=n)
    check_attention(torch, pool, queries(torch, sum(new), 12, 64, dtype, n), new, lens, 0.125)


def test_append_to_many_sequences(torch):
    rng = np.random.default_rng(3)
    for n in (33, 200):
        new = [int(x) for x in rng.integers(0, 20, n)]
        lens = [int(x) for x in rng.integers(0, 60, n)]
        test_append_rotates_and_rounds_to_the_nearest_code(torch, 4, 2, 64, new, lens, "bf16", "f32", False, "packed")
