"""Attention of packed texts and its backward pass against plain 64-bit arithmetic (tests/packed_ref.py has the bounds)."""
import math

import pytest

from tests import packed_ref as ref
from tests.parity import need_gpu

pytestmark = pytest.mark.gpu

HEADS = [(28, 4, 128, "bf16"), (12, 2, 128, "bf16"), (8, 8, 64, "bf16"), (16, 1, 128, "bf16"), (10, 2, 64, "bf16"), (5, 1, 128, "bf16"),
         (128, 1, 64, "bf16"), (65, 1, 128, "bf16"), (3, 3, 128, "bf16"), (4, 2, 64, "f32"), (12, 2, 128, "f32"), (3, 3, 64, "f32")]
TEXTS = [[1], [1, 0, 2], [0, 0], [17, 18, 19], [35, 36, 37, 0, 73], [127, 128, 129], [255, 1, 257], [64, 63, 65], [300, 0, 45, 700], [1153], [1] * 40]


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


def make(torch, heads, lens, seed=0, before=0, tail=0):
    """q, k, v and d_out as parts of rows of one buffer, keys with some large channels."""
    Hq, Hkv, hd, src = heads
    dtype = {"bf16": torch.bfloat16, "f32": torch.float32}[src]
    g = torch.Generator(device="cuda").manual_seed(seed)
    R = before + sum(lens) + tail
    x = torch.randn(R, 2 * Hq + 2 * Hkv, hd, generator=g, device="cuda")
    x[:, Hq:Hq + Hkv] *= torch.where(torch.rand(hd, generator=g, device="cuda") < 0.05, 3.0, 1.0)
    x = x.to(dtype)
    return x.split([Hq, Hkv, Hkv, Hq], 1), dtype


def texts_of(torch, lens, before=0, tail=0):
    from paper_2512_14681_gb300 import packed as P

    start = [before]
    for n in lens:
        start.append(start[-1] + n)
    return P.Packed(torch.tensor(start, dtype=torch.int32, device="cuda"), start[-1] + tail, max(lens))


def both(torch, texts, lens, q, k, v, d, scale, before=0):
    from paper_2512_14681_gb300 import packed as P

    out, lse = P.attention(texts, q, k, v, scale, want_lse=True)
    w_out, w_lse, t_out, t_lse = ref.forward(torch, lens, before, q, k, v, scale)
    ref.inside(torch, out, w_out, t_out, "out")
    ref.inside(torch, lse, w_lse, t_lse, "lse")
    got = P.attention_grad(texts, q, k, v, out, lse, d, scale)
    want, bounds = ref.backward(torch, lens, before, q, k, v, d, scale, out, lse)
    for x, w, b, name in zip(got, want, bounds, ("dq", "dk", "dv")):
        ref.inside(torch, x, w, b, name)
    P.check()
    return out, lse, *got


@pytest.mark.parametrize("lens", TEXTS, ids=lambda v: "-".join(map(str, v[:5])))
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "%d-%d-%d-%s" % h)
def test_against_64_bits(torch, heads, lens):
    (q, k, v, d), _ = make(torch, heads, lens)
    both(torch, texts_of(torch, lens), lens, q, k, v, d, heads[2] ** -0.5)


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[2], HEADS[9]], ids=lambda h: "%d-%d-%d-%s" % h)
def test_many_texts(torch, heads):
    """More than 32, up to the most that a call takes; a batch long enough that every CTA walks through several units."""
    for lens in ([(7 * i) % 41 for i in range(300)], [(5 * i) % 3 for i in range(1024)], [900, 5, 1100, 0, 513, 1024, 300, 77, 640]):
        (q, k, v, d), _ = make(torch, heads, lens, seed=3)
        both(torch, texts_of(torch, lens), lens, q, k, v, d, heads[2] ** -0.5)


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[4], HEADS[10]], ids=lambda h: "%d-%d-%d-%s" % h)
@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_scales(torch, heads, scale):
    lens = [40, 150]
    (q, k, v, d), _ = make(torch, heads, lens, seed=4)
    both(torch, texts_of(torch, lens), lens, q, k, v, d, scale)


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[2], HEADS[9]], ids=lambda h: "%d-%d-%d-%s" % h)
def test_rows_of_no_text(torch, heads):
    """Rows before the first text and behind the last: NaN in all of them reaches nothing, and they get 0."""
    lens, before, tail = [50, 0, 131], 9, 37
    (q, k, v, d), dtype = make(torch, heads, lens, seed=5, before=before, tail=tail)
    for x in (q, k, v, d):
        x[:before] = math.nan
        x[-tail:] = math.nan
    results = both_of_real(torch, texts_of(torch, lens, before, tail), lens, q, k, v, d, heads[2] ** -0.5, before, tail)
    for x in results:
        for rows in (x[:before], x[-tail:]):
            assert torch.equal(rows, torch.full_like(rows, -math.inf if x.dim() == 2 else 0.0))


def both_of_real(torch, texts, lens, q, k, v, d, scale, before, tail):
    from paper_2512_14681_gb300 import packed as P

    clean = [torch.zeros_like(x) for x in (q, k, v, d)]
    for c, x in zip(clean, (q, k, v, d)):
        c[before:x.shape[0] - tail] = x[before:x.shape[0] - tail]
    out, lse = P.attention(texts, q, k, v, scale, want_lse=True)
    got = P.attention_grad(texts, q, k, v, out, lse, d, scale)
    w_out, w_lse, t_out, t_lse = ref.forward(torch, lens, before, *clean[:3], scale)
    want, bounds = ref.backward(torch, lens, before, *clean, scale, out, lse)
    ref.inside(torch, out, w_out, t_out, "out")
    for x, w, b, name in zip(got, want, bounds, ("dq", "dk", "dv")):
        ref.inside(torch, x, w, b, name)
    P.check()
    return out, lse, *got


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[2], HEADS[3], HEADS[9]], ids=lambda h: "%d-%d-%d-%s" % h)
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_text_that_is_no_number_keeps_it(torch, heads, bad):
    """A NaN or infinity anywhere in one text leaves its neighbours' results bit for bit as they are."""
    from paper_2512_14681_gb300 import packed as P

    lens = [50, 70, 200, 33]
    (q, k, v, d), _ = make(torch, heads, lens, seed=6)
    texts, scale = texts_of(torch, lens), heads[2] ** -0.5
    run = lambda: (lambda o: [*o, *P.attention_grad(texts, q, k, v, o[0], o[1], d, scale)])(P.attention(texts, q, k, v, scale, want_lse=True))
    want = run()
    for x in (q, k, v, d):
        x[50, 0, 3] = bad
        x[119, -1, 60] = bad
        x[85] = -bad
    for x, w in zip(run(), want):
        assert torch.equal(x[:50], w[:50]) and torch.equal(x[120:], w[120:])
    P.check()


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[4], HEADS[9]], ids=lambda h: "%d-%d-%d-%s" % h)
def test_rows_at_any_distance_and_address(torch, heads):
    """Rows that tensor copies cannot read (odd distances and addresses) give what aligned ones give, up to rounding; rows far
    apart the same bits. Gradients go into parts of one buffer's rows and leave what lies beside them."""
    from paper_2512_14681_gb300 import packed as P

    Hq, Hkv, hd, _ = heads
    lens = [33, 190, 1]
    (q, k, v, d), dtype = make(torch, heads, lens, seed=7)
    texts, scale = texts_of(torch, lens), hd ** -0.5
    want = both(torch, texts, lens, *(x.contiguous() for x in (q, k, v, d)), scale)
    far = [torch.cat([x, torch.full_like(x, math.nan)], 1)[:, :x.shape[1]] for x in (q, k, v, d)]
    for x, w in zip(both(torch, texts, lens, *far, scale), want):
        assert torch.equal(x, w)
    odd = []
    for x in (q, k, v, d):
        flat = torch.full((x.shape[0] * (x.shape[1] * hd + 3) + 8,), math.nan, dtype=dtype, device="cuda")
        y = flat.as_strided(x.shape, (x.shape[1] * hd + 3, hd, 1), 1)
        y.copy_(x)
        odd.append(y)
    both(torch, texts, lens, *odd, scale)
    R = sum(lens)
    fused = torch.full((R, (Hq + 2 * Hkv) * hd + 1), 7.0, dtype=dtype, device="cuda")
    parts = [p.unflatten(1, (-1, hd)) for p in fused[:, :-1].split([Hq * hd, Hkv * hd, Hkv * hd], 1)]
    got = P.attention_grad(texts, q, k, v, want[0], want[1], d, scale, grads=parts)
    for x, w in zip(got, want[2:]):
        assert torch.equal(x, w)
    assert (fused[:, -1] == 7).all()
    P.check()


@pytest.mark.parametrize("heads", [HEADS[9], HEADS[10]], ids=lambda h: "%d-%d-%d-%s" % h)
def test_gradient_against_differences(torch, heads):
    """d/dt of sum(out d_out) along a direction, by differences of two steps: what the smaller one is off by is a third of their
    difference (the fourth order beyond it: as much again), and rounding of out counts over the step."""
    from paper_2512_14681_gb300 import packed as P

    lens = [37, 1, 90]
    (q, k, v, d), _ = make(torch, heads, lens, seed=8)
    texts, scale = texts_of(torch, lens), heads[2] ** -0.5
    out, lse = P.attention(texts, q, k, v, scale, want_lse=True)
    grads = P.attention_grad(texts, q, k, v, out, lse, d, scale)
    _, _, t_out, _ = ref.forward(torch, lens, 0, q, k, v, scale)
    noise = (t_out * d.double().abs()).sum().item()
    x = [q, k, v]
    for i in range(3):
        way = torch.randn_like(x[i])

        def loss(t):
            y = list(x)
            y[i] = x[i] + t * way
            return (P.attention(texts, *y, scale).double() * d.double()).sum().item()

        h = 2.0 ** -6
        near, wide = (loss(h) - loss(-h)) / (2 * h), (loss(2 * h) - loss(-2 * h)) / (4 * h)
        moved = (d.double().abs().sum() * 2 ** -24 * 4).item()  # x + t way is rounded too
        got = (grads[i].double() * way.double()).sum().item()
        assert abs(got - near) <= abs(near - wide) * 2 / 3 + 2 * (noise + moved) / (2 * h), (i, got, near, wide)


def test_offsets_beyond_32_bits(torch):
    heads, lens, before = (28, 4, 128, "bf16"), [70, 130], 480000
    Hq, Hkv, hd, _ = heads
    R = before + sum(lens) + 5
    qkv = torch.empty(R, (Hq + 2 * Hkv), hd, dtype=torch.bfloat16, device="cuda")
    assert before * qkv.stride(0) > 2 ** 31
    (q0, k0, v0, d0), _ = make(torch, heads, lens, seed=9)
    qkv[before:before + 200] = torch.cat([q0, k0, v0], 1)
    q, k, v = qkv.split([Hq, Hkv, Hkv], 1)
    d = torch.empty(R, Hq, hd, dtype=torch.bfloat16, device="cuda")
    d[before:before + 200] = d0
    from paper_2512_14681_gb300 import packed as P

    texts, scale = texts_of(torch, lens, before, 5), hd ** -0.5
    out, lse = P.attention(texts, q, k, v, scale, want_lse=True)
    got = P.attention_grad(texts, q, k, v, out, lse, d, scale)
    P.check()
    rows = slice(before, before + 200)
    near = texts_of(torch, lens)
    o, l = P.attention(near, q0, k0, v0, scale, want_lse=True)
    for x, w in zip((out, lse, *got), (o, l, *P.attention_grad(near, q0, k0, v0, o, l, d0, scale))):
        assert torch.equal(x[rows], w)
        assert not torch.isnan(x).any()


def test_more_heads_times_rows_than_32_bits_of_pieces(torch):
    """Over 2^28 rows times heads; those of no text get 0. (out and d_out of the call are q: two buffers of 69 GB.)"""
    from paper_2512_14681_gb300 import packed as P

    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 160 << 30:
        pytest.skip("takes 145 GB")
    heads, lens, before = (128, 1, 128, "bf16"), [70, 130], (1 << 21) + 64
    (q0, k0, v0, _), _ = make(torch, heads, lens, seed=15)
    rows, R, scale = slice(before, before + 200), before + 200, 128 ** -0.5
    q, dq = (torch.full((R, 128, 128), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = (torch.full((R, 1, 128), math.nan, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q[rows], k[rows], v[rows] = q0, k0, v0
    q0 = q0.contiguous()
    _, lse0 = P.attention(texts_of(torch, lens), q0, k0, v0, scale, want_lse=True)
    want = P.attention_grad(texts_of(torch, lens), q0, k0, v0, q0, lse0, q0, scale)
    lse = torch.full((R, 128), math.nan, device="cuda")
    lse[rows] = lse0
    got = P.attention_grad(texts_of(torch, lens, before), q, k, v, q, lse, q, scale, grads=(dq, torch.full_like(k, math.nan), torch.full_like(v, math.nan)))
    P.check()
    for x, w in zip(got, want):
        assert torch.equal(x[rows], w)
        for part in x[:before].split(1 << 18):
            assert part.amax() == 0 and part.amin() == 0
    del q, dq, k, v, got, x, part, lse
    torch.cuda.empty_cache()


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[2], HEADS[9]], ids=lambda h: "%d-%d-%d-%s" % h)
@pytest.mark.parametrize("lens,longest", [([0], 0), ([0, 0, 0], 0), ([0, 0], 40), ([0] * 1024, 1000)], ids=["one", "none-longer-than-0", "two", "most"])
def test_a_batch_without_a_row(torch, heads, lens, longest):
    """All rows are of no text: 0, -infinity."""
    from paper_2512_14681_gb300 import packed as P

    Hq, Hkv, hd, _ = heads
    _, dtype = make(torch, heads, [1])
    n = max(longest, 37)
    q, k, v, d = (torch.full((n, H, hd), math.nan, dtype=dtype, device="cuda") for H in (Hq, Hkv, Hkv, Hq))
    for at in (0, 5, n):
        texts = P.Packed(torch.full((len(lens) + 1,), at, dtype=torch.int32, device="cuda"), n, longest)
        out, lse = P.attention(texts, q, k, v, 0.1, want_lse=True)
        grads = [torch.full_like(x, math.nan) for x in (q, k, v)]
        P.attention_grad(texts, q, k, v, out, lse, d, 0.1, grads=grads)
        P.check()
        assert (lse == -math.inf).all() and all((x == 0).all() for x in (out, *grads))


@pytest.mark.parametrize("start", [[0, 50, 40, 100], [-1, 20, 60, 100], [0, 20, 60, 101], [0, 80, 90, 100]], ids=["falls", "negative", "behind", "long"])
@pytest.mark.parametrize("heads", [HEADS[0], HEADS[9]], ids=lambda h: "%d-%d-%d-%s" % h)
def test_texts_that_do_not_fit_are_reported(torch, heads, start):
    """... and nothing is computed; the next call is none the worse."""
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import packed as P

    (q, k, v, d), _ = make(torch, heads, [100], seed=10)
    texts = P.Packed(torch.tensor(start, dtype=torch.int32, device="cuda"), 100, 70)
    out, lse = P.attention(texts, q, k, v, 0.1, want_lse=True)
    with pytest.raises(J.JfError, match="texts"):
        P.check()
    out.zero_(), lse.zero_()
    grads = [torch.full_like(x, 3.0).contiguous() for x in (q, k, v)]
    P.attention_grad(texts, q, k, v, out, lse, d, 0.1, grads=grads)
    with pytest.raises(J.JfError, match="texts"):
        P.check()
    assert all((g == 3).all() for g in grads)
    both(torch, texts_of(torch, [60, 40]), [60, 40], q, k, v, d, 0.1)


def test_calls_that_are_refused(torch):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import packed as P

    (q, k, v, d), _ = make(torch, HEADS[0], [20], seed=11)
    texts = texts_of(torch, [20])
    out, lse = P.attention(texts, q, k, v, 0.1, want_lse=True)
    wide = torch.zeros(20, 4, 96, device="cuda", dtype=torch.bfloat16)
    bad = [(J.JF_EINVAL, lambda: P.attention(texts, q[:19], k, v, 0.1)), (J.JF_EINVAL, lambda: P.attention(texts, q.float(), k, v, 0.1)),
           (J.JF_EUNSUPPORTED, lambda: P.attention(texts, q.half(), k.half(), v.half(), 0.1)),
           (J.JF_EINVAL, lambda: P.attention(texts, q[:, :27], k, v, 0.1)), (J.JF_EINVAL, lambda: P.attention(texts, q, k[:, :3], v, 0.1)),
           (J.JF_EUNSUPPORTED, lambda: P.attention(texts, wide, wide, wide, 0.1)), (J.JF_EINVAL, lambda: P.attention(texts, q[:1].expand(20, 28, 128), k, v, 0.1)),
           (J.JF_EINVAL, lambda: P.attention(texts, q.transpose(0, 1).contiguous().transpose(0, 1), k, v, 0.1)),
           (J.JF_EINVAL, lambda: P.attention(texts, q, k, v, math.nan)), (J.JF_EINVAL, lambda: P.attention(texts, q, k, v, math.inf)),
           (J.JF_EINVAL, lambda: P.attention(texts, q.cpu(), k.cpu(), v.cpu(), 0.1)),
           (J.JF_EUNSUPPORTED, lambda: P.attention(texts, q.detach().requires_grad_(), k, v, 0.1)),
           (J.JF_EINVAL, lambda: P.attention_grad(texts, q, k, v, out[:19], lse, d, 0.1)), (J.JF_EINVAL, lambda: P.attention_grad(texts, q, k, v, out, lse.double(), d, 0.1)),
           (J.JF_EINVAL, lambda: P.attention_grad(texts, q, k, v, out, lse, d.float(), 0.1)),
           (J.JF_EINVAL, lambda: P.attention_grad(texts, q, k, v, out, lse, d[:1].expand(20, 28, 128), 0.1)),
           (J.JF_EINVAL, lambda: P.attention_grad(texts, q, k, v, out, lse, d, 0.1, grads=(q, k, v[:, :1]))),
           (J.JF_EINVAL, lambda: setattr(texts, "row_start", texts.row_start.clone()))]
    for i, (status, call) in enumerate(bad):
        with pytest.raises(J.JfError) as e:
            call()
        assert e.value.status == status, i
    empty = texts_of(torch, [0])
    o, l = P.attention(empty, q[:0], k[:0], v[:0], 0.1, want_lse=True)
    assert o.shape == (0, 28, 128) and all(g.shape[0] == 0 for g in P.attention_grad(empty, q[:0], k[:0], v[:0], o, l, d[:0], 0.1))


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[2], HEADS[9]], ids=lambda h: "%d-%d-%d-%s" % h)
def test_the_same_bits_every_time(torch, heads):
    """Also on another stream, beside other calls, and from threads."""
    import threading

    from paper_2512_14681_gb300 import packed as P

    lens = [400, 31, 700, 5]
    (q, k, v, d), _ = make(torch, heads, lens, seed=12)
    texts, scale = texts_of(torch, lens), heads[2] ** -0.5

    def run(stream=None):
        out, lse = P.attention(texts, q, k, v, scale, want_lse=True, stream=stream)
        return out, lse, *P.attention_grad(texts, q, k, v, out, lse, d, scale, stream=stream)

    want = run()
    torch.cuda.synchronize()
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(run(), want))
    wrong = []

    def work(i):
        st = torch.cuda.Stream()
        for _ in range(10):
            got = run(st)
            st.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want)):
                wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    P.check()


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[4], HEADS[9]], ids=lambda h: "%d-%d-%d-%s" % h)
def test_a_captured_call_follows_its_texts(torch, heads):
    """Two graphs of one forward and backward pass each, replayed with other lengths and values; eager calls between them."""
    from paper_2512_14681_gb300 import packed as P

    (q, k, v, d), _ = make(torch, heads, [600], seed=13)
    texts, scale = P.Packed.of([600, 0, 0], max_rows=600), heads[2] ** -0.5

    def run():
        out, lse = P.attention(texts, q, k, v, scale, want_lse=True)
        return out, lse, *P.attention_grad(texts, q, k, v, out, lse, d, scale)

    run()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    got = []
    for g in graphs:
        with torch.cuda.graph(g):
            got.append(run())
    for lens in ([200, 350, 50], [0, 0, 1], [599, 0, 1], [128, 129, 130]):
        start = torch.tensor([0, lens[0], lens[0] + lens[1], sum(lens)], dtype=torch.int32)
        texts.row_start.copy_(start)
        q.mul_(-1.0)
        want = run()
        for g in graphs:
            g.replay()
        more = P.attention(P.Packed.of([300, 300]), q, k, v, scale)
        torch.cuda.synchronize()
        for res in got:
            assert all(torch.equal(a, b) for a, b in zip(res, want)), lens
        assert not torch.isnan(more.float()).any()
    P.check()


def test_a_first_call_that_is_captured(torch, monkeypatch):
    from paper_2512_14681_gb300 import packed as P

    heads, lens = HEADS[0], [30, 9]
    (q, k, v, d), _ = make(torch, heads, lens, seed=16)
    monkeypatch.setattr(P, "_err", {})
    texts = P.Packed.of(lens, max_rows=1000)  # (no text is longer than all rows)
    assert texts.max_rows == 39
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = P.attention(texts, q, k, v, 0.1, want_lse=True)
        grads = P.attention_grad(texts, q, k, v, out, lse, d, 0.1)
    graph.replay()
    P.check()
    o, l = P.attention(texts, q, k, v, 0.1, want_lse=True)
    for x, w in zip((out, lse, *grads), (o, l, *P.attention_grad(texts, q, k, v, o, l, d, 0.1))):
        assert torch.equal(x, w)


def test_tensors_of_another_device_than_the_current_one(torch):
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import packed as P

    if torch.cuda.device_count() < 2:
        (q, k, v, _), _ = make(torch, HEADS[9], [5], seed=14)
        cpu = P.Packed.of([5])
        with pytest.raises(J.JfError):
            P.attention(cpu, q, k.cpu(), v, 0.1)
        return
    with torch.cuda.device(1):
        (q, k, v, _), _ = make(torch, HEADS[9], [5], seed=14)
        texts = P.Packed.of([5])
    with pytest.raises(J.JfError):
        P.attention(texts, q, k, v, 0.1)
