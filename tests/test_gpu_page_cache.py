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
        cache.append()
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
