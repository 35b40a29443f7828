"""The calls of the paged cache refuse bad arguments on the host, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = 0, 1, 2, 5, 6


@pytest.fixture(scope="module")
def B():
    from paper_2605_00789_amd import binding
    return binding


def at(k):
    """Made-up device addresses far apart: only host-side validation may look at them."""
    return 0x10000000 * (k + 1)


def _pages(B, **over):
    p = B._CPages()
    p.batch, p.n_pages, p.page_tokens, p.max_pages, p.table_stride, p.table = 3, 10, 16, 4, 4, at(0)
    p.heads, p.kv_heads, p.head_dim, p.dtype, p.K, p.V = 8, 2, 64, 1, at(1), at(2)
    p.k_page_stride, p.k_tok_stride, p.k_head_stride = 16 * 128, 128, 64
    p.v_page_stride, p.v_tok_stride, p.v_head_stride = 16 * 128, 64, 16 * 64
    for k, v in over.items():
        setattr(p, k, v)
    return p


TABLE = [
    (dict(table=None), NULL), (dict(batch=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(page_tokens=0), SHAPE),
    (dict(table_stride=3), SHAPE), (dict(table=at(0) + 2), UNSUPPORTED), (dict(batch=4097), UNSUPPORTED),
    (dict(page_tokens=4), UNSUPPORTED), (dict(page_tokens=24), UNSUPPORTED), (dict(page_tokens=2048), UNSUPPORTED),
    (dict(n_pages=1 << 27, page_tokens=16), UNSUPPORTED), (dict(max_pages=1 << 27, table_stride=1 << 27), UNSUPPORTED),
    (dict(max_pages=(1 << 26) + 1, table_stride=1 << 27), UNSUPPORTED),
]
POOLS = TABLE + [
    (dict(kv_heads=0), SHAPE), (dict(heads=0), SHAPE), (dict(heads=7), SHAPE), (dict(head_dim=48), UNSUPPORTED), (dict(head_dim=256), UNSUPPORTED),
    (dict(dtype=2), UNSUPPORTED), (dict(heads=1 << 17), UNSUPPORTED), (dict(K=at(1) + 8), UNSUPPORTED),
    (dict(k_page_stride=-128), SHAPE), (dict(v_tok_stride=-64), SHAPE), (dict(k_head_stride=-64), SHAPE),
    (dict(k_tok_stride=60), UNSUPPORTED), (dict(v_head_stride=68), UNSUPPORTED), (dict(v_page_stride=1001), UNSUPPORTED),
]


def _alloc(B, p, **o):
    a = dict(cu=at(3), lens=at(4), free=at(5), count=at(6), lens_out=at(7), count_out=at(8), slots=at(9), rows=50, status=at(10))
    a.update(o)
    return B._lib.lightkv_page_alloc(C.byref(p) if p is not None else None, a["cu"], a["lens"], a["free"], a["count"], a["lens_out"],
                                     a["count_out"], a["slots"], a["rows"], a["status"], None)


def _free(B, p, **o):
    a = dict(done=at(3), lens=at(4), free=at(5), count=at(6), lens_out=at(7), count_out=at(8))
    a.update(o)
    return B._lib.lightkv_page_free(C.byref(p) if p is not None else None, a["done"], a["lens"], a["free"], a["count"], a["lens_out"], a["count_out"], None)


def _write(B, p, **o):
    a = dict(cu=at(3), slots=at(4), rows=50, K=at(5), kt=128, kh=64, V=at(6), vt=128, vh=64)
    a.update(o)
    return B._lib.lightkv_page_write(C.byref(p) if p is not None else None, a["cu"], a["slots"], a["rows"], a["K"], a["kt"], a["kh"], a["V"], a["vt"], a["vh"], None)


def _attend(B, p, **o):
    a = dict(lens=at(3), bound=0, Q=at(4), qt=512, qh=64, scale=0.0, out=at(5), ot=512, oh=64, lse=at(6), ws=at(7), bytes=1 << 24)
    a.update(o)
    return B._lib.lightkv_page_attention(C.byref(p) if p is not None else None, a["lens"], a["bound"], a["Q"], a["qt"], a["qh"], a["scale"], a["out"],
                                         a["ot"], a["oh"], a["lse"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("over,want", TABLE)
def test_tables(B, over, want):
    assert _alloc(B, _pages(B, **over)) == want
    assert _free(B, _pages(B, **over)) == want


@pytest.mark.parametrize("over,want", POOLS)
def test_pools(B, over, want):
    assert _write(B, _pages(B, **over)) == want
    assert _attend(B, _pages(B, **over)) == want
    n = C.c_size_t(0)
    assert B._lib.lightkv_page_attention_workspace(C.byref(_pages(B, **over)), C.byref(n)) == want


def test_descriptor_is_required(B):
    assert _alloc(B, None) == NULL and _free(B, None) == NULL and _write(B, None) == NULL and _attend(B, None) == NULL
    assert B._lib.lightkv_page_attention_workspace(None, C.byref(C.c_size_t(0))) == NULL
    assert B._lib.lightkv_page_attention_workspace(C.byref(_pages(B)), None) == NULL


def test_alloc_arguments(B):
    p = _pages(B)
    for name in ("cu", "lens", "free", "count", "lens_out", "count_out", "slots"):
        assert _alloc(B, p, **{name: None}) == NULL, name
        assert _alloc(B, p, **{name: at(20) + 2}) == UNSUPPORTED, name
    assert _alloc(B, p, rows=-1) == SHAPE and _alloc(B, p, rows=1 << 31) == UNSUPPORTED
    # outputs may not lie in inputs or in each other; lengths and count may be updated in place, but not half
    assert _alloc(B, p, slots=at(3)) == SHAPE and _alloc(B, p, slots=at(0) + 8) == SHAPE and _alloc(B, p, status=at(9) + 4) == SHAPE
    assert _alloc(B, p, lens_out=at(4) + 4) == SHAPE and _alloc(B, p, lens_out=at(3)) == SHAPE
    assert _alloc(B, p, count_out=at(5) + 36) == SHAPE and _alloc(B, p, slots=at(5)) == SHAPE
    assert _alloc(B, p, lens_out=at(6)) == SHAPE      # the length array over the count


def test_free_arguments(B):
    p = _pages(B)
    for name in ("done", "lens", "free", "count", "lens_out", "count_out"):
        assert _free(B, p, **{name: None}) == NULL, name
        assert _free(B, p, **{name: at(20) + 1}) == UNSUPPORTED, name
    assert _free(B, p, free=at(0)) == SHAPE and _free(B, p, lens_out=at(3)) == SHAPE and _free(B, p, lens_out=at(4) + 4) == SHAPE
    assert _free(B, p, count_out=at(5)) == SHAPE and _free(B, p, free=at(4)) == SHAPE


def test_write_arguments(B):
    p = _pages(B)
    assert _write(B, p, slots=None) == NULL and _write(B, p, K=None, V=None) == NULL
    assert _write(B, _pages(B, V=None)) == NULL                       # rows for a pool that is not there
    assert _write(B, p, rows=-1) == SHAPE and _write(B, p, rows=1 << 31) == UNSUPPORTED
    assert _write(B, p, rows=0) == OK
    assert _write(B, p, K=at(5) + 4) == UNSUPPORTED and _write(B, p, kt=130) == UNSUPPORTED and _write(B, p, vh=33) == UNSUPPORTED
    assert _write(B, p, kt=-128) == SHAPE
    assert _write(B, p, slots=at(4) + 1) == UNSUPPORTED and _write(B, p, cu=at(3) + 2) == UNSUPPORTED
    assert _write(B, p, K=at(1) + 256) == SHAPE and _write(B, p, V=at(1)) == SHAPE and _write(B, p, K=at(2) + 10 * 16 * 256 - 32) == SHAPE


def test_rows_that_share_elements(B):
    """Where a call writes, rows may be in any order but not in each other."""
    for over in (dict(k_tok_stride=64), dict(k_head_stride=32), dict(v_tok_stride=0), dict(k_page_stride=1024), dict(v_head_stride=64), dict(v_page_stride=0)):
        assert _write(B, _pages(B, **over)) == SHAPE, over
    # heads outermost, tokens outermost, one page, gaps: all fine (no rows: nothing is launched)
    for over in (dict(k_head_stride=10 * 16 * 64, k_page_stride=16 * 64, k_tok_stride=64), dict(k_tok_stride=10 * 128, k_page_stride=128),
                 dict(n_pages=1, k_page_stride=0, v_page_stride=8), dict(k_page_stride=8192, k_tok_stride=256, k_head_stride=72)):
        assert _write(B, _pages(B, **over), rows=0) == OK, over
    p = _pages(B)
    for o in (dict(ot=64, oh=128), dict(ot=512, oh=32), dict(ot=448, oh=64), dict(ot=64, oh=64), dict(ot=0), dict(oh=0)):
        assert _attend(B, p, **o) == SHAPE, o
    assert _attend(B, p, ot=64, oh=3 * 64, ws=None) == WORKSPACE       # heads outermost: past this check
    # where a pool is only read, its rows may be one and the same
    assert _attend(B, _pages(B, k_tok_stride=0, v_page_stride=0), ws=None) == WORKSPACE


def test_attention_arguments(B):
    p = _pages(B)
    for name in ("lens", "Q", "out"):
        assert _attend(B, p, **{name: None}) == NULL, name
    assert _attend(B, _pages(B, V=None)) == NULL
    for bad in (-1.0, float("nan"), float("inf")):
        assert _attend(B, p, scale=bad) == SHAPE
    assert _attend(B, p, bound=-1) == SHAPE
    assert _attend(B, p, Q=at(4) + 8) == UNSUPPORTED and _attend(B, p, qt=509) == UNSUPPORTED and _attend(B, p, oh=68) == UNSUPPORTED
    assert _attend(B, p, lens=at(3) + 2) == UNSUPPORTED and _attend(B, p, lse=at(6) + 2) == UNSUPPORTED
    assert _attend(B, p, out=at(4)) == SHAPE and _attend(B, p, out=at(4) + 512) == SHAPE and _attend(B, p, lse=at(5) + 64) == SHAPE
    assert _attend(B, p, out=at(1)) == SHAPE and _attend(B, p, out=at(2) + 16) == SHAPE and _attend(B, p, ws=at(4)) == SHAPE and _attend(B, p, lse=at(0)) == SHAPE
    assert _attend(B, p, ws=at(0)) == SHAPE and _attend(B, p, lse=at(7) + 512) == SHAPE and _attend(B, p, ws=at(1)) == SHAPE and _attend(B, p, lse=at(2)) == SHAPE
    assert _attend(B, p, oh=32) == SHAPE and _attend(B, p, ot=0) == SHAPE              # rows of the output in each other
    n = C.c_size_t(0)
    assert B._lib.lightkv_page_attention_workspace(C.byref(p), C.byref(n)) == OK and n.value > 0
    assert _attend(B, p, ws=None) == WORKSPACE and _attend(B, p, ws=at(7) + 16) == WORKSPACE and _attend(B, p, bytes=n.value - 1) == WORKSPACE
    # 2^30 tokens in a row are the most; tiles of all rows of the table are counted in 32 bits
    assert _attend(B, _pages(B, max_pages=1 << 26, table_stride=1 << 26), ws=None) == WORKSPACE
    wide = _pages(B, batch=4096, max_pages=1 << 24, table_stride=1 << 24)
    assert _attend(B, wide) == UNSUPPORTED


def test_binding_refuses_host_tensors(B):
    import torch
    with pytest.raises(ValueError):
        B.Pages(torch.zeros(2, 2, dtype=torch.int32), n_pages=4, page_tokens=16)
    with pytest.raises(ValueError):
        B.Pages(torch.zeros(2, 2), n_pages=4, page_tokens=16)


def test_no_page_kernel_keeps_anything_in_scratch_memory(B):
    """Tiles on their way are what these kernels' rate rests on: a load that is parked in scratch memory is waited for first."""
    from test_code_objects import _kernels
    kernels = {k: m for k, m in _kernels(B.lib_path()).items() if "page_" in k}
    for name in ("page_alloc", "page_free", "page_write", "page_attn_whole", "page_attn_split", "page_attn_join"):
        assert any(name in k for k in kernels), name
    scratch = {k: m[".private_segment_fixed_size"] for k, m in kernels.items() if m[".private_segment_fixed_size"]}
    assert not scratch, scratch


def test_calls_refuse_what_is_no_tensor_of_the_cache(B):
    """What the module behind the calls makes of wrong arguments: a ValueError that names the argument, before anything is launched."""
    import torch
    ext, p = B._lk_pages, _pages(B)
    at_p, host, i = C.addressof(p), torch.zeros(3, 8, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.int32)
    for name, call in (("cu_new", lambda: ext.page_alloc(at_p, 0, i, i, i, i, i, i, i, None, 0)), ("done", lambda: ext.page_free(at_p, 0, None, i, i, i, i, i, 0)),
                       ("slots", lambda: ext.page_write(at_p, 0, i, host, host, None, 0)), ("seq_lens", lambda: ext.page_attention(at_p, 0, 3.5, host, host, host, None, 0.0, 0, 0)),
                       ("arguments", lambda: ext.page_attention(at_p, 0)), ("arguments", lambda: ext.page_alloc()), ("cu_new", lambda: ext.page_alloc(at_p, 0, *[None] * 9))):
        with pytest.raises(ValueError, match=name):
            call()
    with pytest.raises((ValueError, TypeError)):
        ext.page_free("x", 0, i, i, i, i, i, i, 0)


def test_the_copy_of_the_offsets(B):
    """It is an output of lightkv_page_alloc: not in what is read, not in the other outputs; cu_new itself has them already."""
    for where, want in ((at(20) + 2, UNSUPPORTED), (at(3) + 4, SHAPE), (at(4), SHAPE), (at(5) + 8, SHAPE), (at(6), SHAPE), (at(0) + 8, SHAPE),
                        (at(9) + 196, SHAPE), (at(7) + 8, SHAPE), (at(8), SHAPE), (at(10), SHAPE), (at(10) - 12, SHAPE)):
        assert _alloc(B, _pages(B, cu_copy=where)) == want, hex(where)
        if where not in (at(7) + 8, at(8)):
            assert _alloc(B, _pages(B, cu_copy=where), lens_out=at(4), count_out=at(6)) == want, hex(where)
    assert _alloc(B, _pages(B, cu_copy=at(3)), lens_out=at(3)) == SHAPE


def test_the_largest_scale(B):
    """Scores are taken times scale * log2(e): a scale that overflows there is refused, the largest one below is not (WORKSPACE: past it)."""
    for scale, want in ((2.4e38, SHAPE), (3.4e38, SHAPE), (2.35e38, WORKSPACE), (1e-45, WORKSPACE), (3.5e38, SHAPE)):
        assert _attend(B, _pages(B), scale=scale, ws=None) == want, scale


def test_a_scale_that_rounds_to_zero(B):
    """Zero selects the default: a scale that only becomes zero in fp32 must not."""
    import torch
    p, host = _pages(B), torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    for scale, what in ((1e-46, "softmax_scale"), (-1e-300, "softmax_scale"), (1e-44, "seq_lens"), (0.0, "seq_lens")):
        with pytest.raises(ValueError, match=what):
            B._lk_pages.page_attention(C.addressof(p), 0, 3.5, host, host, host, None, scale, 0, 0)


def test_a_write_and_what_it_reads(B):
    """Slots and offsets are read while the pools are written."""
    end = at(1) + 10 * 16 * 128 * 2
    for o in (dict(slots=at(1)), dict(slots=at(2) + 4096), dict(slots=end - 4), dict(slots=at(1) - 196), dict(cu=at(2)), dict(cu=end - 4), dict(cu=at(1) - 12)):
        assert _write(B, _pages(B), **o) == SHAPE, o


def test_pools_that_lie_in_each_other(B):
    """Keys and values of one allocation: in turn they are fine, shared elements are not (no rows: nothing is launched)."""
    def both(off, page, tok, head, **over):
        return _pages(B, K=at(1), V=at(1) + 2 * off, k_page_stride=page, v_page_stride=page, k_tok_stride=tok, v_tok_stride=tok,
                      k_head_stride=head, v_head_stride=head, **over)
    for off, page, tok, head in ((2048, 4096, 128, 64), (-2048, 4096, 128, 64), (128, 4096, 256, 64), (64, 4096, 256, 128), (20480, 2048, 128, 64), (-20480, 2048, 128, 64),
                                 (1280, 128, 2560, 64), (64, 4096, 128, 2048), (64, 256, 2560, 128), (2048 + 3 * 4096, 4096, 128, 64)):
        assert _write(B, both(off, page, tok, head), rows=0) == OK, (off, page, tok, head)
    for off, page, tok, head in ((0, 2048, 128, 64), (2048, 2048, 128, 64), (-2048, 2048, 128, 64), (64, 4096, 128, 64), (128, 4096, 128, 64), (2048 - 64, 4096, 128, 64),
                                 (2048 + 64, 4096, 128, 64), (9 * 4096, 4096, 128, 64), (9 * 4096 + 2048 - 32, 4096, 128, 64), (32, 4096, 256, 128), (96, 4096, 256, 128),
                                 (20480 - 64, 2048, 128, 64), (-20480 + 8, 2048, 128, 64), (4096 * 2 + 256 * 3 + 64, 4096, 256, 64)):
        assert _write(B, both(off, page, tok, head), rows=0) == SHAPE, (off, page, tok, head)
        assert _write(B, both(off, page, tok, head), rows=0, V=None) == OK      # one of them alone
    # strides inside a page that differ: pages in turn are told apart, anything closer is refused
    over = dict(K=at(1), k_page_stride=4096, v_page_stride=4096)
    assert _write(B, _pages(B, V=at(1) + 4096, **over), rows=0) == OK and _write(B, _pages(B, V=at(1) + 4096 - 128, **over), rows=0) == SHAPE
    assert _write(B, _pages(B, V=at(1)), rows=0) == SHAPE
    # one page, one head: axes of one entry do not count
    assert _write(B, both(2048, 0, 128, 64, n_pages=1), rows=0) == OK and _write(B, both(64, 0, 128, 7, n_pages=1, kv_heads=1), rows=0) == OK
    assert _write(B, both(32, 0, 128, 64, n_pages=1, kv_heads=1), rows=0) == SHAPE
    # attention only reads them: the same rows may be keys and values
    assert _attend(B, both(0, 2048, 128, 64), ws=None) == WORKSPACE


def test_pools_that_lie_in_each_other_against_every_element(B):
    """The same question answered by listing the elements, for strides and distances drawn at random."""
    import itertools
    import random
    rng = random.Random(5)
    told = {True: 0, False: 0}
    for _ in range(400):
        n, P, H, D = rng.choice([1, 2, 3]), 8, rng.choice([1, 2, 3]), 32
        axes = [("page", n), ("tok", P), ("head", H)]
        rng.shuffle(axes)
        width, stride = D, {}
        for name, k in axes:
            stride[name] = width + rng.choice([0, 0, 32, 64])
            width = stride[name] * (k - 1) + width
            width += -width % 8
        def elements(at0):
            return {at0 + i * stride["page"] + t * stride["tok"] + h * stride["head"] + e for i, t, h in itertools.product(range(n), range(P), range(H)) for e in range(0, D, 8)}
        off = rng.randrange(-width - 64, width + 64) // 8 * 8 if rng.random() < 0.5 else rng.choice([-1, 1]) * (rng.randrange(n + 1) * stride["page"] + rng.randrange(2) * stride["tok"]
                                                                                                          + rng.randrange(2) * stride["head"] + rng.choice([0, 0, 32, 64]))
        shared = bool(elements(0) & elements(off))
        told[shared] += 1
        p = _pages(B, n_pages=n, page_tokens=P, kv_heads=H, heads=H, head_dim=D, K=at(3), V=at(3) + 2 * off,
                   **{"%s_%s_stride" % (kv, name): s for name, s in stride.items() for kv in "kv"})
        assert _write(B, p, rows=0, kh=32, vh=32, kt=32 * H, vt=32 * H, slots=at(30), cu=None, K=at(31), V=at(32)) == (SHAPE if shared else OK), (n, H, stride, off)
    assert min(told.values()) > 80, told
