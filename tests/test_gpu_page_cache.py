"""PagedCache and the page calls as programs make them: other streams, captured steps, requests that end."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_pages import DEV, I32, check, dense, ints  # noqa: E402


def late(shape, value, turns=20):
    """A tensor that the current stream fills after a while, and memory that was NaN before."""
    x = torch.full(shape, float("nan"), device=DEV)
    a = torch.ones(4096, 4096, device=DEV)
    torch.cuda.synchronize()
    for _ in range(turns):
        a = a @ a * 1e-4
    return x.copy_(value)


def test_a_call_on_another_stream_comes_behind_its_arguments():
    """Rows that the current stream is still computing when the call is made on another one."""
    import paper_2605_00789_amd as lk
    s, n = torch.cuda.Stream(), 700
    cache = lk.PagedCache(dtype="f32", batch=1, heads=2, head_dim=32, n_pages=60, max_seq_tokens=800, max_new_tokens=n)
    K, V, Q = (torch.randn(*shape, device=DEV) for shape in ((n, 2, 32), (n, 2, 32), (1, 2, 32)))
    cache.append(ints([0, n]))
    out = torch.zeros(1, 2, 32, device=DEV)
    torch.cuda.synchronize()
    cache.write(0, late(K.shape, K), V + 0.0, stream=s)
    later = [torch.full((n, 2, 32), 9.0, device=DEV) for _ in range(4)]          # memory of the call's temporaries, were it free
    cache.attend(0, late(Q.shape, Q), out, stream=s)
    s.synchronize()
    ref, lens = dense([K], [V], Q, 32 ** -0.5)
    check("f32", out, None, ref, 32, lens)
    assert all((x == 9).all() for x in later)


def test_a_stream_that_is_captured_beside_the_current_one():
    """A fork inside a capture (both streams belong to it), and a call on a stream of its own while another one is captured."""
    import paper_2605_00789_amd as lk
    cache = lk.PagedCache(dtype="f32", batch=2, heads=2, head_dim=32, n_pages=60, max_seq_tokens=300, max_new_tokens=8)
    main, side, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    k, q, out = torch.randn(2, 2, 32, device=DEV), torch.randn(2, 2, 32, device=DEV), torch.zeros(2, 2, 32, device=DEV)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=main):
        cache.append(cache.one_each)
        side.wait_stream(main)
        cache.write(0, k, k, stream=side)
        main.wait_stream(side)
        cache.attend(0, q, out)
    rows = [[], []]
    for _ in range(4):
        k.copy_(torch.randn(2, 2, 32, device=DEV))
        graph.replay()
        for b in range(2):
            rows[b].append(k[b].clone())
        ref, lens = dense([torch.stack(r) for r in rows], [torch.stack(r) for r in rows], q, 32 ** -0.5)
        check("f32", out, None, ref, 32, lens)
        torch.zeros(1000, device=DEV).sum().item()


def test_a_write_takes_the_offsets_of_the_append_that_ran_last():
    """A graph with an append of its own is replayed between a prompt's append and an eager write: the write is of the replayed step."""
    import paper_2605_00789_amd as lk
    batch, P = 3, 8
    cache = lk.PagedCache(dtype="f32", batch=batch, heads=1, head_dim=32, n_pages=30, max_seq_tokens=64, max_new_tokens=40, page_tokens=P, layers=2)
    k = torch.zeros(batch, 1, 32, device=DEV)
    k.copy_(torch.arange(1.0, batch + 1, device=DEV).view(batch, 1, 1).expand_as(k))
    cu = ints([0, 2, 4, 6])
    cache.append(cu)
    for layer in range(2):
        cache.write(layer, torch.ones(6, 1, 32, device=DEV), torch.ones(6, 1, 32, device=DEV))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append()
        cache.write(0, k, k)
    more = ints([5, 5, 5, 5])
    for turn in range(3):
        cache.append(more)                                    # nobody gets anything, and the offsets begin behind all rows of a step
        assert cache.cu_new.tolist() == [5] * 4
        graph.replay()
        cache.write(1, k, 2 * k)
        torch.zeros(1000, device=DEV).sum().item()
        assert cache.cu_new.tolist() == [0, 1, 2, 3]
        for b in range(batch):
            pos = 2 + turn
            page = int(cache.table[b, pos // P])
            for layer, factor in ((0, 1.0), (1, 2.0)):
                K, V = cache.pools[layer]
                assert (K[page, pos % P] == b + 1).all() and (V[page, pos % P] == factor * (b + 1)).all()
    cu.fill_(99)                                              # the caller's array is the caller's again
    cache.append()
    cache.write(0, k, k)
    assert cache.seq_lens.tolist() == [6] * 3


def test_a_row_that_was_released_stays_empty_until_it_is_filled():
    """A captured step, replayed for more than a page's tokens while one row of the batch is released and one was never used: these take
    no page from the others, and row b of what is written stays sequence b's."""
    import paper_2605_00789_amd as lk
    batch, P, H, D = 4, 8, 2, 32
    # pages for three sequences of 21 tokens and not one more
    cache = lk.PagedCache(dtype="f32", batch=batch, heads=H, head_dim=D, n_pages=9, max_seq_tokens=64, max_new_tokens=40, page_tokens=P)
    g = torch.Generator(device=DEV).manual_seed(1)
    k, q, out = (torch.zeros(batch, H, D, device=DEV) for _ in range(3))
    lse = torch.zeros(H, batch, device=DEV)
    rows = [torch.zeros(0, H, D, device=DEV) for _ in range(batch)]

    def fill(b, n):
        x = torch.randn(n, H, D, generator=g, device=DEV)
        status = cache.append(ints([0] * (b + 1) + [n] * (batch - b)))
        cache.write(0, x, 2 * x)
        rows[b] = x
        assert status.tolist() == [0] * batch

    def compare(status):
        ref, lens = dense(rows, [2 * r for r in rows], q, D ** -0.5)
        check("f32", out, lse, ref, D, lens)
        assert cache.seq_lens.tolist() == lens and cache.status.tolist() == status
        assert int(cache.free_count) == 9 - sum(-(-n // P) for n in lens)
        assert (out[[b for b in range(batch) if lens[b] == 0]] == 0).all()

    for b in (0, 1, 3):
        fill(b, 3)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.append()
        cache.write(0, k, 2 * k)
        cache.attend(0, q, out, lse=lse)
    def replay():
        for x in (k, q):
            x.copy_(torch.randn(batch, H, D, generator=g, device=DEV))
        graph.replay()
        for b in range(batch):
            if len(rows[b]):
                rows[b] = torch.cat([rows[b], k[b:b + 1]])
        torch.zeros(1000, device=DEV).sum().item()

    for _ in range(6):
        replay()
        compare([0, 0, 3, 0])
    cache.release(ints([0, 1, 0, 0]))
    rows[1] = rows[1][:0]
    for _ in range(12):
        replay()
        compare([0, 3, 3, 0])
    assert cache.seq_lens.tolist() == [21, 0, 0, 21]
    fill(2, 9)                                                # another request takes the row that was never used
    fill(1, 1)
    for _ in range(3):
        replay()
        compare([0] * batch)


def test_a_first_token_of_nothing():
    """append() gives nothing to empty sequences, append(one_each) does."""
    import paper_2605_00789_amd as lk
    cache = lk.PagedCache(dtype="bf16", batch=2, heads=1, head_dim=32, n_pages=4, max_seq_tokens=16, max_new_tokens=4)
    assert cache.append().tolist() == [3, 3] and cache.seq_lens.tolist() == [0, 0] and cache.slots[:2].tolist() == [-1, -1]
    assert cache.append(cache.one_each).tolist() == [0, 0] and cache.seq_lens.tolist() == [1, 1]
    assert cache.append().tolist() == [0, 0] and cache.seq_lens.tolist() == [2, 2] and int(cache.free_count) == 2


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("rows", [70, 3000])
def test_sequences_without_tokens_are_left_out(rows, in_place):
    """skip_empty among prompts, empty prompts, impossible lengths, offsets that fall and a pool that runs short."""
    from paper_2605_00789_amd import binding as B
    P, lens = 8, [0, 3, 0, -2, 8, 0, 5]
    for cu, status, grown in (([0, 2, 4, 4, 6, 8, 10, 40], [3, 0, 0, 2, 0, 3, 1], [0, 5, 0, -2, 10, 0, 5]),
                              ([0, 4, 6, 6, 5, 7, 9, 12], [3, 0, 0, 2, 2, 3, 0], [0, 5, 0, -2, 8, 0, 8])):
        table = torch.full((7, 6), -5, **I32)
        table[1, 0], table[4, 0], table[6, 0] = 9, 8, 7
        pages = B.Pages(table, n_pages=10, page_tokens=P, skip_empty=True)
        old, count = ints(lens), ints([2])
        new, left = (old, count) if in_place else (torch.full_like(old, 99), torch.full_like(count, 99))
        slots, st = torch.full((rows,), -7, **I32), torch.full_like(old, 99)
        B.lightkv_page_alloc(pages, ints(cu), old, ints([5, 6, 0, 0, 0, 0, 0, 0, 0, 0]), count, new, left, slots, status=st)
        assert st.tolist() == status and new.tolist() == grown and left.tolist() == [1 if status[4] == 0 else 2]
        want = [-7] * rows
        for t in range(cu[-1]):
            want[t] = -1
            for b in range(7):
                if status[b] == 0 and cu[b] <= t < cu[b + 1]:
                    pos = lens[b] + t - cu[b]
                    want[t] = (6 if b == 4 else int(table[b, 0])) * P + pos % P
        assert slots.tolist() == want


@pytest.mark.parametrize("hint", [1, 1 << 20], ids=["whole", "split"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinities_under_the_smallest_weights(dtype, hint):
    """Weights of 2^-1 to 2^-126, numbers that one bf16 value holds, against rows with infinities; and against the largest finite value, where
    a weight may be off by 2^-15 of itself or by 2^-133, as its two bf16 parts allow (fp32: 2^-22, the exponential's)."""
    from paper_2605_00789_amd import binding as B
    n, D, P, dt = 126, 32, 8, {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    K, V = (torch.zeros(n, P, 1, D, dtype=dt, device=DEV) for _ in range(2))
    K[:, 1, 0, 0] = -torch.arange(1.0, n + 1, device=DEV).to(dt)
    V[:, :2, 0, 1] = 3.0
    V[:, 1, 0, 0], V[:, 1, 0, 2] = float("inf"), float("-inf")
    V[:, 0, 0, 3], V[:, 1, 0, 3] = 1.0, 2.0 ** 127
    Q, out = torch.zeros(n, 1, D, dtype=dt, device=DEV), torch.empty(n, 1, D, dtype=dt, device=DEV)
    Q[:, 0, 0] = 1.0
    ws = torch.empty(B.lightkv_page_attention_workspace(B.Pages(torch.zeros(n, 1, **I32), K=K, V=V)), dtype=torch.uint8, device=DEV)
    # 0.6931472 * log2(e) is 1 in fp32: the exponents are whole numbers
    B.lightkv_page_attention(B.Pages(torch.arange(n, **I32).view(n, 1), K=K, V=V), ints([2] * n), Q, out, ws, softmax_scale=0.6931471824645996, max_seq_tokens=hint)
    got = out[:, 0].double().cpu()
    assert (got[:, 0] == float("inf")).all() and (got[:, 2] == -float("inf")).all()
    step = torch.finfo(dt).eps / 2
    w = 2.0 ** -torch.arange(1, n + 1, dtype=torch.float64)
    off = w * 2.0 ** -22 + (torch.maximum(w * 2.0 ** -15, torch.tensor(2.0 ** -133, dtype=torch.float64)) if dtype == "bf16" else 0)
    for e, big in ((1, 3.0), (3, 2.0 ** 127)):
        want = (big * w + (3.0 if e == 1 else 1.0)) / (1 + w)
        # the weights' errors against their values, twice (sum and quotient), four roundings in fp32, one to the result's type
        tol = 2 * off * big + want * 4 * 2.0 ** -24
        assert ((got[:, e] - want).abs() <= tol + step * (want + tol)).all(), e


def test_a_stage_that_does_not_fit_leaves_the_cache_as_it_was():
    """Rows of another type, width or layer: refused before any sequence is given tokens that are never written."""
    import types
    import paper_2605_00789_amd as lk
    cache = lk.PagedCache(dtype="bf16", batch=2, heads=4, head_dim=32, n_pages=9, max_seq_tokens=64, max_new_tokens=40)
    def stage(dtype=torch.bfloat16, width=128):
        return types.SimpleNamespace(K=torch.zeros(10, width, dtype=dtype, device=DEV), V=torch.zeros(10, width, dtype=dtype, device=DEV), cu_vis_out=ints([0, 4, 10]))
    for layer, st, error in ((0, stage(torch.float32), ValueError), (0, stage(width=96), ValueError), (1, stage(), IndexError)):
        with pytest.raises(error):
            cache.store_stage(layer, st)
        assert cache.seq_lens.tolist() == [0, 0] and int(cache.free_count) == 9
    assert cache.store_stage(0, stage()).tolist() == [0, 0] and cache.seq_lens.tolist() == [4, 6]
