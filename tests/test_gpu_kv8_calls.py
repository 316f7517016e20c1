"""Calls of the 8-bit cache's operators that go wrong easily: pages, rows, tensors, streams and devices that do not fit."""
import numpy as np
import pytest

from tests.parity import need_gpu
from tests.test_gpu_kv8 import PAGE, check_attention, fill, queries, reference, rows_of, tree_bits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def torch():
    return need_gpu()


@pytest.mark.parametrize("dtype,n", [("bf16", 2), ("bf16", 50), ("f32", 5)])
@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_a_page_outside_the_pool_is_reported_and_its_keys_left_out(torch, dtype, n, bad):
    """In the middle of a context, at its end, and a sequence of one page (whose rows then see nothing), beside a sequence
    that is in order."""
    from paper_2512_14681_gb300._lib import JfError

    new, lens = [n, n, n], [1000 - n, 500, 0]
    for lost in ((0, 20), (0, 62), (1, 3), (2, 0)):
        pool = fill(torch, 4, 128, [a + k for a, k in zip(lens, new)], seed=31)
        pool.cache.page_table[lost[0], lost[1]] = bad
        q = queries(torch, sum(new), 28, 128, dtype, 7, 0.3)

        def see(b):
            vis = np.arange(lens[b] + n)[None, :] <= lens[b] + np.arange(n)[:, None]
            if b == lost[0]:
                vis[:, lost[1] * PAGE:(lost[1] + 1) * PAGE] = False
            return vis

        out, lse = pool.cache.attention(rows_of(new, lens), q, 128 ** -0.5, want_lse=True)
        with pytest.raises(JfError, match="out of range"):
            pool.cache.check()
        ref, A, ref_lse, dS = reference(pool, q.double().cpu().numpy(), new, lens, 128 ** -0.5, see)
        bf16 = dtype == "bf16"
        tol = (2 * dS + (2.0 ** -11 if bf16 else 2.0 ** -20))[..., None] * A + (2.0 ** -8 * np.abs(ref) if bf16 else 0) + 1e-37
        assert (np.abs(out.double().cpu().numpy() - ref) <= tol).all()
        got, none = lse.double().cpu().numpy(), ref_lse == -np.inf
        assert (got[none] == -np.inf).all()
        ref_lse = np.where(none, 0, ref_lse)
        assert (np.abs(np.where(none, 0, got) - ref_lse) <= 2 * dS + 1e-6 * (1 + np.abs(ref_lse))).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hint", [1, 8, 33, 70])
def test_a_mask_narrower_than_a_sequences_rows(torch, dtype, hint):
    """row_start may hold more rows a sequence than the host's max_rows says (a captured graph's batch has changed): a row
    sees no new row beyond its mask's words, in either form, and no other row's words count."""
    new, lens, words = [5, 70, 40], [200, 33, 0], 1 + (hint - 1) // 32
    pool = fill(torch, 4, 128, [a + n for a, n in zip(lens, new)], seed=41)
    rng = np.random.default_rng(3)
    bits = [rng.random((n, 32 * words)) < 0.7 for n in new]
    mask = torch.from_numpy(np.concatenate([tree_bits(b, words) for b in bits])).cuda()
    store = torch.full((mask.numel() + 64,), -1, dtype=torch.int32, device="cuda")  # (what follows the mask would show)
    store[:mask.numel()] = mask.flatten()

    def see(b):
        new_rows = np.zeros((new[b], new[b]), bool)
        n = min(new[b], 32 * words)
        new_rows[:, :n] = bits[b][:, :n]
        return np.concatenate([np.ones((new[b], lens[b]), bool), new_rows], 1)

    check_attention(torch, pool, queries(torch, sum(new), 28, 128, dtype, 9, 0.3), new, lens, 128 ** -0.5,
                    store[:mask.numel()].view(-1, words), see, max_rows=hint)


def test_rows_that_share_memory_are_refused(torch):
    """Broadcast and overlapping rows of every input; one row may have any stride."""
    from paper_2512_14681_gb300 import _lib as J

    pool = fill(torch, 2, 64, [40], seed=1)
    c, rows = pool.cache, rows_of([4], [20])
    x, q = torch.ones(4, 2, 64, device="cuda"), torch.ones(4, 4, 64, device="cuda")
    for kind in ("broadcast", "overlapping"):
        def shared(t):
            return t[:1].expand(t.shape) if kind == "broadcast" else \
                torch.ones(4 * t[0].numel(), device="cuda").as_strided(t.shape, (t[0].numel() - 1, *t.stride()[1:]))
        for call in (lambda: c.append(rows, shared(x), x), lambda: c.append(rows, x, shared(x)), lambda: c.append(rows, x, x, q=shared(q)),
                     lambda: c.append(rows, shared(x.view(4, 128)), x), lambda: c.attention(rows, shared(q), 0.1),
                     lambda: c.attention(rows, shared(q.view(4, 256)), 0.1)):
            with pytest.raises(J.JfError, match="apart") as e:
                call()
            assert e.value.status == J.JF_EINVAL
    one = rows_of([1], [20])
    want = c.attention(one, q[:1], 0.1)
    for stride in (0, 7, 10 ** 6):
        assert torch.equal(c.attention(one, q.as_strided((1, 4, 64), (stride, 64, 1)), 0.1), want)
    c.check()


def test_a_captured_call_keeps_its_memory(torch):
    """Warmed up and captured on one stream; a larger eager call there, then fresh tensors: replays leave those alone, and
    their results are right. Two graphs of the same capture stream replayed on two others at the same time."""
    pool = fill(torch, 4, 128, [5000], seed=51)
    c, st = pool.cache, torch.cuda.Stream()
    q1, q2, big = (queries(torch, n, 28, 128, "bf16", s) for n, s in ((1, 1), (1, 2), (300, 3)))
    r1, r2 = rows_of([1], [4000]), rows_of([1], [3000])
    want1, want2 = c.attention(r1, q1, 0.1), c.attention(r2, q2, 0.1)
    rb = rows_of([300], [4000])
    torch.cuda.synchronize()
    c.attention(r1, q1, 0.1, stream=st)
    st.synchronize()
    graphs, outs = [], []
    for r, q in ((r1, q1), (r2, q2)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=st):
            outs.append(c.attention(r, q, 0.1))
    c.attention(rb, big, 0.1, stream=st)
    st.synchronize()
    with torch.cuda.stream(st):
        fresh = [torch.full((1 << 18,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(64)]
        fresh += [torch.full((1 << 22,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(16)]
    torch.cuda.synchronize()
    for _ in range(3):
        graphs[0].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want1) and all((t == 0x5A).all() for t in fresh)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(50):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want1) and torch.equal(outs[1], want2)
    c.check()


def test_threads_on_one_stream(torch):
    """Calls of several threads, whose launches may come in any order."""
    import threading

    pool = fill(torch, 4, 128, [6000, 900], seed=52)
    work = [(rows_of([1, 1], [5000 + i, 100 * i + 7]), queries(torch, 2, 28, 128, "bf16", i)) for i in range(4)] + \
        [(rows_of([20, 9], [5000 + i, 100 * i + 7]), queries(torch, 29, 28, 128, "bf16", i)) for i in range(4)]
    want = [pool.cache.attention(r, q, 0.1) for r, q in work]
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        for _ in range(150):
            if not torch.equal(pool.cache.attention(*work[i], 0.1), want[i]):
                wrong.append(i)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    pool.cache.check()


def test_caches_hold_no_workspaces(torch):
    """What a call needs beside its outputs goes back to the allocator: many caches cost no more than one."""
    from paper_2512_14681_gb300.kv8 import Kv8Cache

    caches = [Kv8Cache.empty(1, 1024, 2, 128) for _ in range(6)]
    x, q = torch.randn(64, 2, 128, device="cuda"), queries(torch, 64, 12, 128, "bf16", 1)
    before = torch.cuda.memory_allocated()
    for c in caches:
        c.append(rows_of([64], [0]), x, x)
        c.attention(rows_of([64], [0]), q, 0.1)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() - before < 1 << 20


def test_check_waits_for_every_stream(torch):
    from paper_2512_14681_gb300._lib import JfError

    pool = fill(torch, 2, 64, [40], seed=1)
    q, st = torch.ones(1, 4, 64, device="cuda"), torch.cuda.Stream()
    beyond = rows_of([1], [10 ** 6])
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(200_000_000)
    pool.cache.attention(beyond, q, 0.1, stream=st)
    with pytest.raises(JfError, match="out of range"):
        pool.cache.check()


def test_tensors_of_another_device_are_refused(torch, monkeypatch):
    """Every call whose tensors are not on the current device (a box of one GPU: the current device's number is replaced)."""
    from paper_2512_14681_gb300 import _lib as J
    from paper_2512_14681_gb300 import kv8, logprobs

    pool = fill(torch, 2, 64, [40], seed=1)
    c, rows = pool.cache, rows_of([4], [20])
    x, q = torch.ones(4, 2, 64, device="cuda"), torch.ones(4, 4, 64, device="cuda")
    z, t = torch.randn(4, 100, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    r = logprobs.token_logprobs(z, t)
    monkeypatch.setattr(kv8, "_current_device", lambda: torch.cuda.current_device() + 1)
    for call in (lambda: c.append(rows, x, x), lambda: c.read(rows), lambda: c.attention(rows, q, 0.1),
                 lambda: logprobs.token_logprobs(z, t), lambda: logprobs.token_logprobs_grad(z, t, r.row_stats, r.entropy, 1.0)):
        with pytest.raises(J.JfError, match="current device") as e:
            call()
        assert e.value.status == J.JF_EINVAL
    monkeypatch.undo()
    for bad in (dict(positions=torch.zeros(4, dtype=torch.int32)), dict(positions=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        with pytest.raises(J.JfError, match="positions"):
            c.append(rows, x, x, **bad)
    with pytest.raises(J.JfError, match="mask"):
        c.attention(rows, q, 0.1, mask=torch.zeros(4, 1, dtype=torch.int32))
    c.check()


def test_tensors_that_calls_point_into_cannot_be_replaced(torch):
    """An assignment would have no effect on calls, and let the tensor that they read be freed."""
    from paper_2512_14681_gb300._lib import JfError

    pool, rows = fill(torch, 2, 64, [40], seed=1), rows_of([4], [20])
    for owner, names in ((pool.cache, ("k", "v", "k_exp", "v_exp", "page_table")), (rows, ("row_start", "len", "n_rows", "max_rows"))):
        for name in names:
            was = getattr(owner, name)
            setattr(owner, name, was)
            with pytest.raises(JfError, match=f"{name} cannot be replaced"):
                setattr(owner, name, was.clone() if torch.is_tensor(was) else was + 1)
            assert getattr(owner, name) is was
    q = queries(torch, 4, 4, 64, "f32", 1)
    before = pool.cache.attention(rows, q, 0.1)
    pool.cache.page_table.copy_(pool.cache.page_table.clone())
    assert torch.equal(pool.cache.attention(rows, q, 0.1), before)
