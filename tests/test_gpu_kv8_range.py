"""Attention over values whose blocks' exponents lie anywhere in the format's range, side by side in one context.

Tolerances are those of the attention's other tests (tests/test_gpu_kv8.py), relative to A = sum p |v| of what the row
itself sees: neither a page that it does not see nor one that it gives no weight may cost it precision.
"""
import numpy as np
import pytest

from tests.parity import need_gpu
from tests.test_gpu_kv8 import PAGE, check_attention, fill, queries, tree_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


def pages_of(torch, pool, first, count=1):
    return torch.from_numpy(pool.table[0, first:first + count].astype(np.int64)).cuda()


FORMS = [("bf16", 1, 28, 4, 128), ("bf16", 40, 28, 4, 128), ("bf16", 3, 4, 2, 64), ("bf16", 100, 4, 2, 64), ("f32", 1, 28, 4, 128),
         ("f32", 9, 4, 2, 64)]


@pytest.mark.parametrize("dtype,n,Hq,Hkv,hd", FORMS)
@pytest.mark.parametrize("where", ["first", "middle", "last", "several", "all"])
def test_blocks_of_zeros_beside_ordinary_ones(torch, dtype, n, Hq, Hkv, hd, where):
    """What append writes for a page of values that are all 0: exponent -120."""
    total = 2048
    pool = fill(torch, Hkv, hd, [total], seed=21, v_spread=2)
    c = pool.cache
    c.v &= 0x7F  # (values of one sign, whose sums grow)
    c.v[c.v == 0x7F] = 0
    for at in {"first": [0], "middle": [60], "last": [total // PAGE - 1], "several": [3, 4, 31, 64, 65, 66, 127],
               "all": range(total // PAGE)}[where]:
        c.v[pages_of(torch, pool, at)] = 0
        c.v_exp[pages_of(torch, pool, at)] = -120
    out = check_attention(torch, pool, queries(torch, n, Hq, hd, dtype, 3, 0.3), [n], [total - n], hd ** -0.5)
    assert out.isfinite().all() and (where == "all") == (not out.any())


@pytest.mark.parametrize("dtype,n,Hq,Hkv,hd", FORMS)
@pytest.mark.parametrize("exps", [(-8, -120), (-8, 119), (-120, 119), (-8, -120, 119), (-60, 50, -110, 0)])
def test_exponents_from_both_ends_of_the_range(torch, dtype, n, Hq, Hkv, hd, exps):
    """Pages take the exponents in turn, first in runs of 1, then of 9 pages."""
    total = 1500
    for run in (1, 9):
        pool = fill(torch, Hkv, hd, [total], seed=22)
        for p in range(-(-total // PAGE)):
            pool.cache.v_exp[pages_of(torch, pool, p)] = exps[p // run % len(exps)]
        pool.cache.v &= 0xBF  # (magnitudes below 2, so that every output is a finite number)
        check_attention(torch, pool, queries(torch, n, Hq, hd, dtype, 4, 0.3), [n], [total - n], hd ** -0.5)


@pytest.mark.parametrize("dtype,n,Hq,Hkv,hd", FORMS)
@pytest.mark.parametrize("weight", [-300, -130, -100, -40])
def test_large_values_of_little_weight(torch, dtype, n, Hq, Hkv, hd, weight):
    """Every tenth page holds values 2^110 times the others' and its keys 2^weight of the others' weight: from nothing to
    all of the output."""
    total = 1200
    pool = fill(torch, Hkv, hd, [total], seed=23)
    c = pool.cache
    c.k.zero_()
    c.k_exp.fill_(0)
    c.v &= 0xBF
    big = torch.cat([pages_of(torch, pool, p) for p in range(2, total // PAGE, 10)])
    c.v_exp[big] = 102
    code = int(torch.tensor([-float(2 ** int(np.log2(-weight)))]).to(torch.float8_e4m3fn).view(torch.uint8))
    size = 2.0 ** int(np.log2(-weight))
    c.k[big, :, :, 0] = code
    q = torch.zeros(n, Hq, hd, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    q[:, :, 0] = 1.0
    check_attention(torch, pool, q, [n], [total - n], -weight / size * float(np.log(2.0)))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("e", [119, 60, -120])
def test_values_that_a_row_does_not_see_cost_it_nothing(torch, dtype, e):
    """New rows of which some lie in pages of far larger (or smaller) values: earlier rows, and rows that a tree's mask
    hides them from, keep the precision of their own."""
    n, ctx = 70, 300
    pool = fill(torch, 2, 128, [ctx + n], seed=24)
    pool.cache.v &= 0xBF
    pool.cache.v_exp[pages_of(torch, pool, 20, 2)] = e  # slots 320 .. 351: new rows 20 .. 51
    q = queries(torch, n, 12, 128, dtype, 5, 0.3)
    check_attention(torch, pool, q, [n], [ctx], 128 ** -0.5)
    see = np.tril(np.ones((n, n), bool))
    see[52:60, 20:52] = False
    see[60:, 20] = False
    mask = torch.from_numpy(tree_bits(see, 3)).cuda()
    vis = lambda b: np.concatenate([np.ones((n, ctx), bool), see], 1)
    check_attention(torch, pool, q, [n], [ctx], 128 ** -0.5, mask, vis)
    # without a context: the page comes first for some rows, and never for others
    pool = fill(torch, 2, 128, [n], seed=25)
    pool.cache.v &= 0xBF
    pool.cache.v_exp[pages_of(torch, pool, 0)] = e
    see = np.tril(np.ones((n, n), bool))
    see[16:40, :16] = False
    mask = torch.from_numpy(tree_bits(see, 3)).cuda()
    check_attention(torch, pool, q, [n], [0], 128 ** -0.5, mask, lambda b: see)


def test_an_appended_page_of_zeros(torch):
    """The same through append: padding whose values are 0 between tokens whose values are not."""
    from paper_2512_14681_gb300.kv8 import Kv8Cache, Rows

    cache = Kv8Cache.empty(1, 4096, 2, 64)
    g = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn(4000, 2, 64, generator=g, device="cuda")
    v = torch.rand(4000, 2, 64, generator=g, device="cuda")
    v[3200:3264] = 0
    cache.append(Rows.of([4000], [0]), k, v)
    for n in (1, 64):
        q = torch.randn(n, 8, 64, generator=g, device="cuda").bfloat16()
        out = cache.attention(Rows.of([n], [4000 - n]), q, 0.125).double()
        cache.check()
        rk, rv = (t.double() for t in cache.read(Rows.of([4000], [0])))
        s = torch.einsum("rhd,khd->rhk", q.double(), rk.repeat_interleave(4, 1)) * 0.125
        s = s.masked_fill((torch.arange(4000, device="cuda")[None, :] > 4000 - n + torch.arange(n, device="cuda")[:, None])[:, None], -float("inf"))
        ref = torch.einsum("rhk,khd->rhd", torch.softmax(s, -1), rv.repeat_interleave(4, 1))
        dS = torch.einsum("rhd,khd->rhk", q.double().abs(), rk.abs().repeat_interleave(4, 1)).max(-1).values * 0.125 * 64 * 2.0 ** -23
        assert ((out - ref).abs() <= (2 * dS + 2.0 ** -11)[..., None] * ref + 2.0 ** -8 * ref).all()


@pytest.mark.parametrize("dtype,n,Hq,Hkv,hd", FORMS)
@pytest.mark.parametrize("gap", [32, 96, 128])
def test_weights_that_fall_while_values_grow(torch, dtype, n, Hq, Hkv, hd, gap):
    """Scores climb by 2^32 every two pages; of each two the first holds values of 2^110 times the second's, and 2^-gap of
    its weight. No value is 0: in a dim in which the row's heavy keys were, what it should hold would be that of keys whose
    weight is below 2^-24 of the row's largest, which one fp16 term does not hold."""
    total = 448
    pool = fill(torch, Hkv, hd, [total], seed=26)
    c = pool.cache
    c.k.zero_()
    c.k_exp.fill_(0)
    c.v &= 0xBF
    c.v |= 0x20
    code = lambda x: int(torch.tensor([float(x)]).to(torch.float8_e4m3fn).view(torch.uint8))
    for p in range(total // PAGE):
        c.k[pages_of(torch, pool, p), :, :, 0] = code(32 * (p // 2) - (0 if p % 2 else gap))
        c.v_exp[pages_of(torch, pool, p)] = -8 if p % 2 else 102
    q = torch.zeros(n, Hq, hd, device="cuda", dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    q[:, :, 0] = 1.0
    check_attention(torch, pool, q, [n], [total - n], float(np.log(2.0)))


@pytest.mark.parametrize("dtype,n,Hq,Hkv,hd", FORMS)
@pytest.mark.parametrize("apart", [20, 30, 40])
@pytest.mark.parametrize("order", [(0, 1), (1, 0)])
def test_small_pages_keep_their_share(torch, dtype, n, Hq, Hkv, hd, apart, order):
    """Equal weights; every second page's exponent is `apart` larger, but its values are the smallest codes in all dims but
    one: there the other pages, all of the largest code, hold up to 2^-2 of the output. (The scores are 0, so that nothing
    but the sums rounds.)"""
    for total in (n + 31, 150 + n, 1024):
        pool = fill(torch, Hkv, hd, [total], seed=total)
        for p in range(-(-total // PAGE)):
            big, at = p % 2 == order[0], pages_of(torch, pool, p)
            pool.cache.v_exp[at] = 0 if big else -apart
            pool.cache.v[at] = 1 if big else 0x7E
            if big:
                pool.cache.v[at, :, :, 5] = 0x7E
        check_attention(torch, pool, queries(torch, n, Hq, hd, dtype, 4, 0.0), [n], [total - n], hd ** -0.5)
