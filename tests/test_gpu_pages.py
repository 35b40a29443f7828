"""The paged cache on the GPU against plain implementations: a stack of pages on the host for the tables, indexing for the
writes, attention in 64 bits (computed on the host from the rows' values) for lightkv_page_attention."""
import math
import random

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
DEV = "cuda:0"
I32 = dict(dtype=torch.int32, device=DEV)
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def ints(v):
    return torch.tensor(v, **I32)


# ---- tables -----------------------------------------------------------------------------------------------------------
class HostTables:
    """The tables as a program on the host would keep them."""

    def __init__(self, batch, n_pages, P, width, stack):
        self.P, self.width, self.n_pages = P, width, n_pages
        self.table = [[-5] * width for _ in range(batch)]
        self.lens, self.stack, self.count = [0] * batch, list(stack), len(stack)

    def pages(self, n):
        return -(-n // self.P)

    def alloc(self, cu, slots):
        asked, had, status, slots = 0, self.count, [], list(slots)
        rows = len(slots)
        for b in range(len(self.lens)):
            n, L = cu[b + 1] - cu[b], self.lens[b]
            if cu[b] < 0 or n < 0 or cu[b + 1] > rows or L < 0 or L + n > self.width * self.P:
                status.append(2)
            else:
                need = self.pages(L + n) - self.pages(L)
                asked += need
                status.append(1 if need and asked > had else 0)
            if status[-1] == 0:
                for j in range(self.pages(L), self.pages(L + n)):
                    self.count -= 1
                    self.table[b][j] = self.stack[self.count]
                self.lens[b] = L + n
            for t in range(max(cu[b], 0), min(cu[b + 1], rows)):
                pos = L + t - cu[b]
                page = self.table[b][pos // self.P] if status[-1] == 0 else -1
                slots[t] = page * self.P + pos % self.P if 0 <= page < self.n_pages else -1
        return slots, status

    def free(self, done):
        for b, d in enumerate(done):
            if d:
                k = min(self.pages(max(self.lens[b], 0)), self.width)
                for page in self.table[b][:k]:
                    if self.count < self.n_pages:
                        self.stack[self.count:self.count + 1] = [page]
                        self.count += 1
                self.lens[b] = 0


class DeviceTables:
    def __init__(self, batch, n_pages, P, width, stack, in_place, stride=None):
        from paper_2605_00789_amd import binding as B
        self.B, self.in_place = B, in_place
        self.store = torch.full((batch, stride or width), -5, **I32)
        self.table = self.store[:, :width]
        self.pages = B.Pages(self.table, n_pages=n_pages, page_tokens=P)
        self.lens, self.count = torch.zeros(batch, **I32), ints([len(stack)])
        self.stack = torch.full((n_pages,), -3, **I32)
        self.stack[:len(stack)] = ints(stack)

    def _outs(self):
        return (self.lens, self.count) if self.in_place else (torch.full_like(self.lens, -9), torch.full_like(self.count, -9))

    def alloc(self, cu, slots):
        lens, count = self._outs()
        slots, status = ints(slots), torch.full_like(self.lens, -9)
        self.B.lightkv_page_alloc(self.pages, ints(cu), self.lens, self.stack, self.count, lens, count, slots, status=status)
        self.lens, self.count = lens, count
        return slots.tolist(), status.tolist()

    def free(self, done):
        lens, count = self._outs()
        self.B.lightkv_page_free(self.pages, ints(done), self.lens, self.stack, self.count, lens, count)
        self.lens, self.count = lens, count


def same(d, h):
    assert d.lens.tolist() == h.lens
    assert d.count.tolist() == [h.count]
    assert d.stack.tolist()[:h.count] == h.stack[:h.count]
    assert d.table.tolist() == h.table


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("batch,P,width,most,spare", [
    (1, 8, 1, 8, 1), (1, 1024, 3, 2000, 3), (2, 16, 4, 40, 8), (5, 8, 9, 30, 20), (64, 32, 6, 90, 300), (255, 16, 8, 60, 700),
    (256, 16, 8, 60, 900), (257, 8, 12, 50, 1200), (1000, 64, 5, 130, 1500), (4096, 8, 4, 12, 6000)])
def test_tables_over_many_calls(batch, P, width, most, spare, in_place):
    print("[tables]", batch, P, width, most, spare, in_place, flush=True)
    rng = random.Random(batch * 131 + P)
    n_pages = spare + 7
    stack = rng.sample(range(n_pages), spare)
    h, d = HostTables(batch, n_pages, P, width, stack), DeviceTables(batch, n_pages, P, width, stack, in_place, stride=width + 3)
    for call in range(7):
        if call in (3, 5):
            done = [int(rng.random() < 0.4) * rng.choice([1, -1, 77]) for _ in range(batch)]
            h.free(done)
            d.free(done)
        else:
            one = call in (2, 6)
            cu = [rng.choice([0, 0, 2])]
            for _ in range(batch):
                cu.append(cu[-1] + (rng.choice([0, 1, 1]) if one else rng.choice([0, rng.randint(0, most)])))
            slots = [-7] * (cu[-1] + rng.choice([0, 1, 6]) or 1)
            want, got = h.alloc(cu, slots), d.alloc(cu, slots)
            assert got[1] == want[1]
            assert got[0] == want[0]
        same(d, h)
    assert (d.store[:, width:] == -5).all()


def test_tables_refuse_what_cannot_be():
    """Lengths, offsets and page numbers that no program should have: no access outside the arrays, a status, nothing else moves."""
    P, width, n_pages = 16, 4, 40
    stack = [3, 99, -1, 7, 2 ** 30, 5, 11, 12, 13, 14, 15, 16]
    h, d = HostTables(6, n_pages, P, width, stack), DeviceTables(6, n_pages, P, width, stack, True)
    h.lens = [-4, 2 ** 31 - 1, 70, 3, 0, 64]
    d.lens = ints(h.lens)
    for t in (h.table, d.table):
        t[3][0] = 4444                                        # the page sequence 3 goes on in is none of the pool's
    cu = [0, 5, 9, 12, 20, 90, 90]                            # 90: more rows than there are slots and tokens in a row
    assert d.alloc(cu, [-7] * 40) == h.alloc(cu, [-7] * 40)
    same(d, h)
    assert h.lens[3] == 11
    cu = [8, 4, -3, 30, 10, 12, 2 ** 31 - 1]                  # offsets that fall
    slots, status = d.alloc(cu, [-7] * 40)
    assert status == [2, 2, 2, 2, 0, 2]
    h.lens[4] += 2
    assert d.lens.tolist() == h.lens
    cu = [0, 0, 0, 0, 3, 36, 36]                              # page numbers off the stack that are none of the pool's
    d.stack[:12], d.count[0] = ints(stack), 5
    slots, status = d.alloc(cu, [-7] * 40)
    # sequence 3: 11 + 3 tokens, still in the bad page; 4: 2 + 33 tokens, its first page from before, two new ones: 2 ** 30 and 7
    assert status == [2, 2, 2, 0, 0, 0] and slots[:3] == [-1] * 3
    assert slots[17:33] == [-1] * 16 and slots[33:36] == [7 * P, 7 * P + 1, 7 * P + 2]
    for count in (-5, n_pages + 9):                           # a count outside the stack
        d.count[0] = count
        d.lens = torch.zeros(6, **I32)
        d.alloc([0, 1, 1, 1, 1, 1, 1], [-7] * 4)
        assert d.count.tolist() == ([0] if count < 0 else [n_pages - 1])
    d.lens, d.count = ints([2 ** 31 - 1, -9, 64, 999, 0, 1]), ints([n_pages - 3])
    d.free([1, 1, 1, 1, 1, 1])                                # more than the stack can take
    assert d.count.tolist() == [n_pages] and d.lens.tolist() == [0] * 6


# ---- writes -----------------------------------------------------------------------------------------------------------
def pool(n_pages, P, H, D, dt, layout, fill=None, seed=0):
    g = torch.Generator().manual_seed(seed)
    shape = (n_pages, H, P, D) if layout == "head" else (n_pages, P, H, D)
    x = torch.randn(shape, generator=g) if fill is None else torch.full(shape, fill)
    x = x.to(dt).to(DEV)
    return x.transpose(1, 2) if layout == "head" else x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H,D,P,layout,rows", [(1, 32, 8, "head", 1), (3, 32, 16, "token", 37), (32, 128, 16, "head", 90), (8, 64, 64, "token", 300),
                                               (40, 128, 1024, "head", 50), (160, 32, 8, "head", 9), (5, 128, 32, "token", 0)])
def test_rows_into_pages(dtype, H, D, P, layout, rows):
    print("[write]", dtype, H, D, P, layout, rows, flush=True)
    from paper_2605_00789_amd import binding as B
    dt, rng = TORCH[dtype], random.Random(rows * 7 + H)
    n_pages = rows // P + 9
    K, V = (pool(n_pages, P, H, D, dt, layout, seed=s) for s in (1, 2))
    pages = B.Pages(torch.zeros(2, 3, **I32), K=K, V=V, heads=2 * H)
    # keys, values and something else side by side, as one projection leaves them
    qkv = torch.randn(rows + 4, 3, H, D, generator=torch.Generator().manual_seed(5)).to(dt).to(DEV)
    k, v = qkv[:, 1], qkv[:, 2].transpose(0, 1).contiguous().transpose(0, 1)
    slots = rng.sample(range(n_pages * P), rows + 4)
    for i, bad in zip(rng.sample(range(rows + 4), min(4, rows)), (-1, n_pages * P, -2 ** 31, 2 ** 31 - 1)):
        slots[i] = bad
    for use_cu in (True, False):
        for src_k, src_v in ((k, v), (None, v), (k, None)):
            kk, vv = K.clone(), V.clone()
            for store, src in ((kk, src_k), (vv, src_v)):
                for t in range(rows if use_cu else rows + 4):
                    if src is not None and 0 <= slots[t] < n_pages * P:
                        store[slots[t] // P, slots[t] % P] = src[t]
            B.lightkv_page_write(pages, ints(slots), src_k, src_v, cu_new=ints([0, rows // 2, rows]) if use_cu else None)
            assert torch.equal(K, kk) and torch.equal(V, vv)
            K.copy_(pool(n_pages, P, H, D, dt, layout, seed=1)), V.copy_(pool(n_pages, P, H, D, dt, layout, seed=2))


def test_rows_in_front_of_the_first_sequence_stay_out():
    """Offsets that begin behind row 0: the slots in front are of an earlier call and still name other tokens' places."""
    from paper_2605_00789_amd import binding as B
    K, V = (pool(4, 8, 2, 32, torch.float32, "head", fill=1.0) for _ in range(2))
    pages = B.Pages(torch.zeros(2, 2, **I32), K=K, V=V, heads=2)
    rows = torch.full((9, 2, 32), 5.0, device=DEV)
    B.lightkv_page_write(pages, ints(list(range(9))), rows, rows, cu_new=ints([4, 5, 7]))
    want = torch.ones(4, 8, 2, 32, device=DEV)
    want[0, 4:7] = 5.0
    assert torch.equal(K, want) and torch.equal(V, want)
    B.lightkv_page_write(pages, ints(list(range(9))), rows * 2, rows, cu_new=ints([-3, 0, 1]))
    want[0, 0] = 10.0
    assert torch.equal(K, want)


# ---- attention --------------------------------------------------------------------------------------------------------
def scattered(lens, P, n_pages, width, seed):
    """A table whose pages lie anywhere in the pool; entries behind a sequence's last page are stale."""
    rng = random.Random(seed)
    free = rng.sample(range(n_pages), n_pages)
    table = [[rng.randrange(n_pages) for _ in range(width)] for _ in lens]
    for b, n in enumerate(lens):
        for j in range(-(-max(n, 0) // P)):
            table[b][j] = free.pop()
    return table, free


def reference(Q, K, V, table, lens, P, scale, drop=()):
    """Attention in doubles on the host, with what the tolerance needs: mean absolute values under the weights, and the
    largest sum of |q_e k_e|.  drop: (sequence, token) pairs that do not count."""
    Q, K, V = (x.double().cpu() for x in (Q, K, V))
    batch, heads, D = Q.shape
    H = K.shape[2]
    out, mean = torch.zeros(batch, heads, D, dtype=torch.float64), torch.zeros(batch, heads, D, dtype=torch.float64)
    lse, big = torch.full((heads, batch), -math.inf, dtype=torch.float64), torch.zeros(batch, heads, 1, dtype=torch.float64)
    for b, n in enumerate(lens):
        at = [t for t in range(n) if (b, t) not in drop]
        if not at:
            continue
        page, row = torch.tensor([table[b][t // P] for t in at]), torch.tensor([t % P for t in at])
        k, v = K[page, row], V[page, row]                                    # [tokens, H, D]
        q = Q[b].view(H, heads // H, D)
        x = torch.matmul(q, k.permute(1, 2, 0)) * scale
        z = torch.logsumexp(x, -1, keepdim=True)
        w = torch.exp(x - z)
        out[b] = torch.matmul(w, v.transpose(0, 1)).reshape(heads, D)
        mean[b] = torch.matmul(w, v.abs().transpose(0, 1)).reshape(heads, D)
        lse[:, b] = z.view(-1)
        big[b] = torch.matmul(q.abs(), k.abs().permute(1, 2, 0)).amax(-1).reshape(heads, 1) * scale
    return out, lse, mean, big


def check(dtype, out, lse, ref, D, lens):
    """|error| <= what roundings can add up to.  Scores: a sum of D products in fp32, each partial sum off by at most half a step
    of a value below `big`, then the scale (twice) -- (D + 4) 2^-24 big.  A weight exp(s) is off by that relatively, plus
    the exponential's own 2^-22; numerator and denominator both: twice.  Sums over n weights: 2^-24 for each addition of a
    chain, which is n / 4 lanes long at most before it is joined, plus 64 joins.  bf16 inputs: weights enter the product as
    two bf16 numbers, each cut: 2^-7 * 2^-7 below the weight.  Then one rounding of the result."""
    want, z, mean, big = ref
    n = max(max(lens), 1)
    step = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}[dtype]
    rel = 2 * ((D + 4) * 2.0 ** -24 * big + 2.0 ** -22) + 2 * (n / 4 + 64) * 2.0 ** -24 + (2.0 ** -14 if dtype == "bf16" else 0.0)
    tol = rel * mean + step * (want.abs() + rel * mean) + 1e-37
    err = (out.double().cpu() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())
    if lse is not None:
        off = (D + 4) * 2.0 ** -24 * big.squeeze(-1).t() + 2.0 ** -22 + (n / 4 + 64) * 2.0 ** -24 + 2.0 ** -22 * z.abs().nan_to_num(0, 0, 0)
        got = lse.double().cpu()
        empty = torch.isinf(z)
        assert torch.equal(torch.isinf(got) & (got < 0), empty)
        assert (((got - z).abs() <= off) | empty).all()


def attend(B, pages, lens, Q, out, lse=None, ws=None, **kw):
    if ws is None:
        ws = torch.empty(B.lightkv_page_attention_workspace(pages), dtype=torch.uint8, device=DEV).fill_(0xff)   # NaN wherever it is read unwritten
    B.lightkv_page_attention(pages, ints(lens), Q, out, ws, lse=lse, **kw)


SHORT = [0, 1, 2, 7, 8, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300]
LONG = [0, 1, 33, 255, 256, 257, 0, 700, 1023, 1500, 2049, 0]


@pytest.mark.parametrize("hint", [0, 1, 1 << 20], ids=["table", "whole", "split"])
@pytest.mark.parametrize("dtype,H,group,D,P,layout,lens", [
    ("bf16", 1, 1, 128, 16, "head", SHORT), ("bf16", 2, 1, 128, 8, "token", SHORT), ("bf16", 3, 4, 64, 16, "token", SHORT), ("bf16", 2, 8, 32, 32, "head", SHORT),
    ("bf16", 1, 16, 128, 64, "head", SHORT), ("bf16", 1, 17, 64, 16, "head", SHORT), ("bf16", 1, 40, 128, 128, "token", SHORT), ("bf16", 2, 9, 32, 8, "head", SHORT),
    ("f32", 1, 1, 32, 8, "token", SHORT), ("f32", 3, 2, 64, 16, "head", SHORT), ("f32", 2, 16, 128, 32, "token", SHORT), ("f32", 1, 33, 32, 256, "head", SHORT),
    ("bf16", 8, 4, 128, 32, "head", LONG), ("bf16", 4, 1, 64, 1024, "token", LONG), ("f32", 2, 7, 128, 16, "head", LONG), ("f32", 5, 1, 64, 8, "token", LONG),
    ("bf16", 1, 1, 32, 16, "head", [20000]), ("bf16", 2, 5, 128, 16, "head", [1]), ("f32", 1, 1, 128, 64, "head", [9001]), ("bf16", 32, 1, 32, 8, "head", [0, 0, 0])])
def test_attention(dtype, H, group, D, P, layout, lens, hint):
    print("[attend]", dtype, H, group, D, P, layout, len(lens), hint, flush=True)
    from paper_2605_00789_amd import binding as B
    dt, g = TORCH[dtype], torch.Generator().manual_seed(H * 100 + group)
    width = -(-max(max(lens), 1) // P) + 1
    n_pages = sum(-(-n // P) for n in lens) + 3
    K, V = (pool(n_pages, P, H, D, dt, layout, seed=s) for s in (3, 4))
    table, _ = scattered(lens, P, n_pages, width, 1)
    heads = H * group
    # queries as a slice of a wider projection, outputs as a slice of a wider buffer
    Q = (1.7 * torch.randn(len(lens) + 2, 2, heads, D, generator=g)).to(dt).to(DEV)[:len(lens), 1]
    store = torch.full((len(lens) + 2, heads, D + 16), 7.0, dtype=dt, device=DEV)
    out, lse = store[:len(lens), :, 16:], torch.full((heads, len(lens)), 5.0, device=DEV)
    pages = B.Pages(ints(table), K=K, V=V, heads=heads)
    attend(B, pages, lens, Q, out, lse, max_seq_tokens=hint)
    check(dtype, out, lse, reference(Q, K, V, table, lens, P, D ** -0.5), D, lens)
    assert (store[:, :, :16] == 7).all() and (store[len(lens):] == 7).all()
    again, z = torch.empty_like(out), torch.empty_like(lse)
    attend(B, pages, lens, Q, again, z, max_seq_tokens=hint)
    assert torch.equal(again, out) and torch.equal(z, lse)
    attend(B, pages, lens, Q, again, None, max_seq_tokens=hint, softmax_scale=0.37)
    check(dtype, again, None, reference(Q, K, V, table, lens, P, 0.37), D, lens)


@pytest.mark.parametrize("hint", [1, 1 << 20], ids=["whole", "split"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("P", [8, 64])
def test_attention_leaves_out_what_does_not_count(dtype, P, hint):
    """NaN and infinities behind the last token and in pages of others, stale table entries, page numbers that are none of
    the pool's, lengths below zero and beyond the row."""
    print("[masked]", dtype, P, hint, flush=True)
    from paper_2605_00789_amd import binding as B
    H, group, D, dt = 2, 3, 64, TORCH[dtype]
    lens = [1, 5, 40, 0, 129, 77, 130, -3, 1000000, 64]
    width = 256 // P
    held = [max(0, min(n, width * P)) for n in lens]
    n_pages = sum(-(-n // P) for n in held) + 4
    clean = [pool(n_pages, P, H, D, dt, "head", seed=s) for s in (8, 9)]
    table, free = scattered(held, P, n_pages, width, 2)
    live = torch.zeros(n_pages, P, dtype=torch.bool)
    for b, n in enumerate(held):
        for t in range(n):
            live[table[b][t // P], t % P] = True
    live = live.to(DEV)
    K, V = clean[0].clone(), clean[1].clone()
    K[~live], V[~live] = float("nan"), float("inf")
    drop = set()
    for b, j, bad in ((2, 1 if P == 8 else 0, -1), (4, 1, n_pages), (5, 0, 2 ** 31 - 1), (6, 0, -2 ** 31), (6, 1, -7), (6, 2, n_pages + 1)):
        table[b][j] = bad
        drop |= {(b, t) for t in range(j * P, (j + 1) * P)}
    if P == 64:
        assert all((6, t) in drop for t in range(130))       # nothing is left of sequence 6
    for b, row in enumerate(table):                           # entries behind the last page are not looked at
        for j in range(-(-held[b] // P), width):
            row[j] = random.Random(b * 99 + j).choice([-1, n_pages, 2 ** 31 - 1])
    Q = torch.randn(len(lens), H * group, D, generator=torch.Generator().manual_seed(1)).to(dt).to(DEV)
    out, lse = torch.empty_like(Q), torch.empty(H * group, len(lens), device=DEV)
    attend(B, B.Pages(ints(table), K=K, V=V, heads=H * group), lens, Q, out, lse, max_seq_tokens=hint)
    safe = [[min(max(p, 0), n_pages - 1) for p in row] for row in table]
    check(dtype, out, lse, reference(Q, *clean, safe, held, P, D ** -0.5, drop), D, held)
    assert (out[3] == 0).all() and (out[7] == 0).all()


@pytest.mark.parametrize("hint", [1, 1 << 20], ids=["whole", "split"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_extreme_rows(dtype, hint):
    """Scores of thousands with either sign, a single key that takes all the weight, keys of the type's largest values (all scores
    -inf, or +inf), infinite values, NaN in a row that counts."""
    print("[extreme]", dtype, hint, flush=True)
    from paper_2605_00789_amd import binding as B
    D, P, H, dt = 64, 16, 1, TORCH[dtype]
    lens = [200] * 8
    table, _ = scattered(lens, P, 8 * 13, 13, 3)
    K, V = (pool(8 * 13, P, H, D, dt, "token", seed=s) for s in (5, 6))
    Q = torch.randn(8, 2, D, generator=torch.Generator().manual_seed(2)).to(dt).to(DEV)

    def row(b, t):
        return table[b][t // P], t % P

    Q[0] *= 3000                                              # one key wins
    Q[1] *= 1e-4
    K[row(2, 150)] = 40 * Q[2, 0]
    for t in range(200):
        K[row(3, t)] = -3e38 * torch.sign(Q[3, 0])            # head 0: every score is -inf in fp32
        K[row(4, t)] *= 1e-3
    Q[3, 1] = Q[3, 0]
    V[row(4, 199)][0, 5] = float("inf")
    K[row(5, 17)] = float("nan")
    V[row(6, 0)][0, 3] = float("nan")
    K[row(7, 90)] = 3e38 * torch.sign(Q[7, 0])                # a score of +inf: inf - inf
    out, lse = torch.empty_like(Q), torch.empty(2, 8, device=DEV)
    attend(B, B.Pages(ints(table), K=K, V=V, heads=2), lens, Q, out, lse, max_seq_tokens=hint)
    ref = reference(Q, K, V, table, lens, P, D ** -0.5)
    fine = [0, 1, 2]
    check(dtype, out[fine], lse[:, fine], tuple(r[:, fine] if r.shape[0] == 2 else r[fine] for r in ref), D, lens)
    assert (out[3] == 0).all() and (lse[:, 3] == -math.inf).all()
    assert torch.isinf(out[4, :, 5]).all() and torch.isfinite(out[4, :, :5]).all() and torch.isfinite(lse[:, 4]).all()
    assert torch.isnan(out[5]).all() and torch.isnan(lse[:, 5]).all()
    assert torch.isnan(out[6, :, 3]).all() and torch.isfinite(out[6, :, 4:]).all()
    assert torch.isnan(out[7, 0]).all()


@pytest.mark.parametrize("hint", [1, 1 << 20], ids=["whole", "split"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_of_infinite_values_under_round_weights(dtype, hint):
    """A weight of 1, of 1/2, of 1/4: numbers that a bf16 value holds exactly, against rows with infinities."""
    from paper_2605_00789_amd import binding as B
    D, P, dt = 32, 8, TORCH[dtype]
    lens, inf = [1, 2, 4, 4], float("inf")
    K, V = (torch.zeros(4, P, 1, D, dtype=dt, device=DEV) for _ in range(2))
    V[:, :, :, 1] = 3.0
    V[:, 0, :, 0], V[1, 1, :, 2], V[3, 1, :, 0] = inf, -inf, -inf
    Q, out = torch.ones(4, 1, D, dtype=dt, device=DEV), torch.empty(4, 1, D, dtype=dt, device=DEV)
    attend(B, B.Pages(ints([[0], [1], [2], [3]]), K=K, V=V, heads=1), lens, Q, out, max_seq_tokens=hint)
    want = torch.zeros(4, D)
    want[:, 0], want[:, 1], want[1, 2], want[3, 0] = inf, 3.0, -inf, float("nan")
    assert torch.equal(out[:, 0].float().cpu().nan_to_num(nan=77.0, posinf=1e30, neginf=-1e30), want.nan_to_num(nan=77.0, posinf=1e30, neginf=-1e30))


@pytest.mark.parametrize("batch,H,group,D,dtype,lens", [
    (700, 1, 2, 32, "bf16", (0, 90)), (300, 2, 1, 64, "f32", (1, 60)), (4096, 1, 1, 32, "bf16", (0, 20)), (257, 4, 3, 32, "bf16", (60, 64)),
    (1100, 1, 1, 32, "f32", (0, 30)), (65, 8, 1, 64, "bf16", (100, 700))])
def test_attention_of_large_batches(batch, H, group, D, dtype, lens):
    """More sequences than threads that look for a part, a long sequence among short ones, more segments than workgroups fit."""
    print("[batch]", batch, H, group, D, dtype, lens, flush=True)
    from paper_2605_00789_amd import binding as B
    P, rng = 16, random.Random(batch)
    n = [rng.randint(*lens) for _ in range(batch)]
    for long in (None, 3, batch - 1):
        if long is not None:
            n[long] = 3001
        width = -(-max(n) // P)
        n_pages = sum(-(-v // P) for v in n) + 2
        K, V = (pool(n_pages, P, H, D, TORCH[dtype], "head", seed=s) for s in (1, 2))
        table, _ = scattered(n, P, n_pages, width, 5)
        Q = torch.randn(batch, H * group, D, generator=torch.Generator().manual_seed(7)).to(TORCH[dtype]).to(DEV)
        out, lse = torch.empty_like(Q), torch.empty(H * group, batch, device=DEV)
        attend(B, B.Pages(ints(table), K=K, V=V, heads=H * group), n, Q, out, lse, max_seq_tokens=1 << 20)
        check(dtype, out, lse, reference(Q, K, V, table, n, P, D ** -0.5), D, n)


def test_a_captured_split_follows_the_lengths():
    """One graph, replayed while sequences grow from nothing to thousands of tokens and shrink again: the cut is the device's."""
    from paper_2605_00789_amd import binding as B
    H, group, D, P, batch, room = 2, 4, 64, 16, 5, 6000
    n_pages = batch * room // P
    K, V = (pool(n_pages, P, H, D, torch.bfloat16, "head", seed=s) for s in (1, 2))
    table = [random.Random(9).sample(range(n_pages), n_pages)[b::batch] for b in range(batch)]
    pages = B.Pages(ints(table), K=K, V=V, heads=H * group)
    ws = torch.empty(B.lightkv_page_attention_workspace(pages), dtype=torch.uint8, device=DEV).fill_(0xff)
    lens = ints([0] * batch)
    Q = torch.randn(batch, H * group, D, device=DEV).to(torch.bfloat16)
    out, lse = torch.zeros_like(Q), torch.zeros(H * group, batch, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.lightkv_page_attention(pages, lens, Q, out, ws, lse=lse)
    for n in ([0] * 5, [1, 2, 3, 4, 5], [5990, 0, 40, 1000, 1], [2000] * 5, [6000, 6000, 6000, 6000, 0], [0, 0, 700, 0, 0]):
        lens.copy_(ints(n))
        graph.replay()
        check("bf16", out, lse, reference(Q, K, V, table, n, P, D ** -0.5), D, n)
        ws.fill_(0xff)
        graph.replay()
        check("bf16", out, lse, reference(Q, K, V, table, n, P, D ** -0.5), D, n)
        torch.randn(1000, device=DEV).sum().item()


def test_attention_of_a_row_does_not_depend_on_where_its_pages_lie():
    from paper_2605_00789_amd import binding as B
    H, D, P, n = 2, 128, 16, 333
    lens = [n, n]
    rows = torch.randn(n, H, D, generator=torch.Generator().manual_seed(4)).to(torch.bfloat16).to(DEV)
    table = [[2 * j + b for j in range(21)] for b in range(2)]
    K, V = (torch.zeros(42, P, H, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for b in range(2):
        for t in range(n):
            K[table[b][t // P], t % P] = rows[t]
            V[table[b][t // P], t % P] = rows[t] * 2
    Q = torch.randn(1, 4, D, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).to(DEV).expand(2, 4, D)
    out = torch.empty(2, 4, D, dtype=torch.bfloat16, device=DEV)
    attend(B, B.Pages(ints(table), K=K, V=V, heads=4), lens, Q, out, max_seq_tokens=n)
    assert torch.equal(out[0], out[1])


def test_a_cache_beyond_four_gigabytes():
    """Pages whose byte offsets pass 32 bits, and element offsets that do."""
    from paper_2605_00789_amd import binding as B
    H, D, P, n_pages = 32, 128, 64, 9000                      # 4.7 GB a pool
    K, V = (torch.empty(n_pages, H, P, D, dtype=torch.bfloat16, device=DEV).transpose(1, 2) for _ in range(2))
    lens = [150, 64]
    table = [[n_pages - 1, 8200, n_pages - 2], [8999 - 3, 0, 0]]
    g = torch.Generator(device=DEV).manual_seed(1)
    rows = torch.randn(2, 214, H, D, generator=g, device=DEV).to(torch.bfloat16)
    slots = ints([table[0][t // P] * P + t % P for t in range(150)] + [table[1][0] * P + t for t in range(64)])
    pages = B.Pages(ints(table), K=K, V=V, heads=H)
    B.lightkv_page_write(pages, slots, rows[0], rows[1])
    Q = torch.randn(2, H, D, generator=g, device=DEV).to(torch.bfloat16)
    out, lse = torch.empty_like(Q), torch.empty(H, 2, device=DEV)
    near = torch.zeros(4, P, H, D, dtype=torch.bfloat16), torch.zeros(4, P, H, D, dtype=torch.bfloat16)
    small = [[0, 1, 2], [3, 3, 3]]
    for i, store in enumerate(near):
        for b, (first, n) in enumerate(((0, 150), (150, 64))):
            for t in range(n):
                store[small[b][t // P], t % P] = rows[i, first + t].cpu()
    ref = reference(Q, *near, small, lens, P, D ** -0.5)
    for hint in (1, 1 << 20):
        attend(B, pages, lens, Q, out, lse, max_seq_tokens=hint)
        check("bf16", out, lse, ref, D, lens)


# ---- together ---------------------------------------------------------------------------------------------------------
def dense(rows_k, rows_v, Q, scale):
    """Attention over plain rows: reference() on a table of one page per sequence."""
    n = [len(r) for r in rows_k]
    P = max(n)
    H, D = rows_k[0].shape[1:]
    K, V = torch.zeros(len(n), P, H, D), torch.zeros(len(n), P, H, D)
    for b in range(len(n)):
        K[b, :n[b]], V[b, :n[b]] = rows_k[b].float().cpu(), rows_v[b].float().cpu()
    return reference(Q, K, V, [[b] for b in range(len(n))], n, P, scale), n


@pytest.mark.parametrize("match", ["best_per_a", "edge_topk"])
def test_compression_then_decoding(match):
    """What a serving program does: compress, move the rows that are left into pages (how many is known on the device), the
    prompts behind them, then decode in a captured graph while sequences grow, end and make room for others."""
    print("[decode]", match, flush=True)
    import paper_2605_00789_amd as lk
    batch, heads, hd, gh, gw = 3, 4, 64, 12, 12
    d, n = heads * hd, 144
    g = torch.Generator(device=DEV).manual_seed(3)
    bf = torch.bfloat16
    X, K, V = (torch.randn(batch * n, d, generator=g, device=DEV).to(bf) for _ in range(3))
    txt = [5, 17, 9]
    cu_txt = np.concatenate([[0], np.cumsum(txt)]).astype(np.int32)
    Qt, Kt, Vt = (torch.randn(sum(txt), d, generator=g, device=DEV).to(bf) for _ in range(3))
    pos = torch.arange(n, **I32).repeat(batch)
    kw = dict(dtype="bf16", batch=batch, d=d, heads=heads, head_dim=hd, tiles=1, grid_h=gh, grid_w=gw, cu_txt=cu_txt, windows_per_axis=(3, 1))
    if match == "best_per_a":
        st = lk.CompressionPipeline(targets=(107, 80), **kw).run(X, K, V, Qt, pos)
    else:
        sched = lk.EdgeTopKSchedule(rho=(0.36, 0.3), **kw)
        st = sched.run((np.arange(batch + 1) * n).astype(np.int32), X, K, V, Qt, pos)[-1]
    cache = lk.PagedCache(dtype="bf16", batch=batch, heads=2 * heads, kv_heads=heads, head_dim=hd, n_pages=60, max_seq_tokens=256,
                          max_new_tokens=batch * n, page_tokens=8, layers=2)
    status = cache.store_stage(0, st)
    cache.write(1, Kt.new_ones(batch * n, d), Kt.new_zeros(batch * n, d))          # a second layer of the same lengths
    assert status.tolist() == [0] * batch
    cu = st.cu_vis_out.tolist()
    Ko, Vo = (st.K_out, st.V_out) if match == "best_per_a" else (st.K, st.V)
    rows_k = [Ko[cu[b]:cu[b + 1]].view(-1, heads, hd) for b in range(batch)]
    rows_v = [Vo[cu[b]:cu[b + 1]].view(-1, heads, hd) for b in range(batch)]
    cu_t = torch.from_numpy(cu_txt).to(DEV)
    cache.append(cu_t)
    cache.write(0, Kt, Vt)
    for b in range(batch):
        rows_k[b] = torch.cat([rows_k[b], Kt[cu_txt[b]:cu_txt[b + 1]].view(-1, heads, hd)])
        rows_v[b] = torch.cat([rows_v[b], Vt[cu_txt[b]:cu_txt[b + 1]].view(-1, heads, hd)])
    assert cache.seq_lens.tolist() == [len(r) for r in rows_k]
    # one decoding step: room, the token's row, its attention
    q, k, v = torch.zeros(batch, 2 * heads, hd, dtype=bf, device=DEV), *(torch.zeros(batch, heads, hd, dtype=bf, device=DEV) for _ in range(2))
    out, lse = torch.zeros_like(q), torch.zeros(2 * heads, batch, device=DEV)

    def step():
        cache.append()
        cache.write(0, k, v)
        cache.attend(0, q, out, lse=lse)

    def new_token():
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device=DEV))
        for b in range(batch):
            rows_k[b], rows_v[b] = torch.cat([rows_k[b], k[b:b + 1]]), torch.cat([rows_v[b], v[b:b + 1]])

    def compare():
        ref, lens = dense(rows_k, rows_v, q, hd ** -0.5)
        check("bf16", out, lse, ref, hd, lens)
        assert cache.seq_lens.tolist() == lens and (cache.status == 0).all()

    new_token()
    step()
    compare()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(20):                                       # pages open on the way
        new_token()
        if i % 5 == 4:
            step()                                            # an eager step between replays
        else:
            graph.replay()
        compare()
        torch.zeros(1000, device=DEV).sum().item()
    # one request ends, its pages serve another
    left = int(cache.free_count)
    cache.release(ints([0, 1, 0]))
    assert int(cache.free_count) == left + -(-len(rows_k[1]) // 8)
    rows_k[1], rows_v[1] = rows_k[1][:0], rows_v[1][:0]
    cache.append(ints([0, 0, 30, 30]))
    again = torch.randn(30, heads, hd, generator=g, device=DEV).to(bf)
    cache.write(0, again, 2 * again)
    rows_k[1], rows_v[1] = again, 2 * again
    for _ in range(3):
        new_token()
        graph.replay()
        compare()


def test_calls_on_another_stream():
    """The whole chain on a stream that is not the current one, and two calls that share a workspace in its order."""
    import paper_2605_00789_amd as lk
    s = torch.cuda.Stream()
    cache = lk.PagedCache(dtype="f32", batch=2, heads=2, head_dim=32, n_pages=400, max_seq_tokens=1600, max_new_tokens=3100)
    rows = torch.randn(3100, 2, 32, device=DEV)
    Q, outs = torch.randn(2, 2, 2, 32, device=DEV), torch.zeros(2, 2, 2, 32, device=DEV)
    cu = ints([0, 1550, 3100])
    torch.cuda.synchronize()
    cache.append(cu, stream=s)
    cache.write(0, rows, rows * 0.5, stream=s)
    for i in range(2):
        cache.attend(0, Q[i], outs[i], stream=s)
    s.synchronize()
    for i in range(2):
        ref, lens = dense([rows[:1550], rows[1550:]], [rows[:1550] * 0.5, rows[1550:] * 0.5], Q[i], 32 ** -0.5)
        check("f32", outs[i], None, ref, 32, lens)


def test_two_graphs_share_a_workspace():
    from paper_2605_00789_amd import binding as B
    H, D, P = 4, 128, 16
    lens = [2500, 700]
    table, _ = scattered(lens, P, 210, 160, 4)
    K, V = (pool(210, P, H, D, torch.bfloat16, "head", seed=s) for s in (1, 2))
    pages = B.Pages(ints(table), K=K, V=V, heads=8)
    ws = torch.empty(B.lightkv_page_attention_workspace(pages), dtype=torch.uint8, device=DEV)
    Q = torch.randn(2, 2, 8, D, device=DEV).to(torch.bfloat16)
    out, want = torch.zeros_like(Q), torch.zeros_like(Q)
    dl = ints(lens)
    for i in range(2):
        B.lightkv_page_attention(pages, dl, Q[i], want[i], ws)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            B.lightkv_page_attention(pages, dl, Q[i], out[i], ws)
        graphs.append(g)
    for turn in range(4):
        out.zero_()
        for g in (graphs if turn % 2 else reversed(graphs)):
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_binding_checks_sizes_and_types():
    from paper_2605_00789_amd import binding as B
    K, V = (torch.zeros(4, 16, 2, 32, device=DEV) for _ in range(2))
    pages = B.Pages(torch.zeros(3, 2, **I32), K=K, V=V, heads=4)
    Q, out = torch.zeros(3, 4, 32, device=DEV), torch.zeros(3, 4, 32, device=DEV)
    ws = torch.empty(B.lightkv_page_attention_workspace(pages), dtype=torch.uint8, device=DEV)
    lens = torch.zeros(3, **I32)
    bad = [lambda: B.lightkv_page_attention(pages, lens[:2], Q, out, ws), lambda: B.lightkv_page_attention(pages, lens.long(), Q, out, ws),
           lambda: B.lightkv_page_attention(pages, lens, Q[:, :3], out, ws), lambda: B.lightkv_page_attention(pages, lens, Q.bfloat16(), out, ws),
           lambda: B.lightkv_page_attention(pages, lens, Q, out[:2], ws), lambda: B.lightkv_page_attention(pages, lens, Q, out, ws, lse=torch.zeros(3, 3, device=DEV)),
           lambda: B.lightkv_page_attention(pages, lens, Q.cpu(), out, ws),
           lambda: B.lightkv_page_write(pages, torch.zeros(3, dtype=torch.int64, device=DEV), Q[:, :2], None),
           lambda: B.lightkv_page_write(pages, lens, Q, None),
           lambda: B.lightkv_page_alloc(pages, lens, lens, lens, lens, lens, lens, lens),
           lambda: B.Pages(torch.zeros(3, 2, **I32), K=K, V=V.bfloat16(), heads=4), lambda: B.Pages(torch.zeros(3, 2, **I32), K=K[0], V=V[0], heads=4),
           lambda: B.Pages(torch.zeros(2, 3, **I32).t(), K=K, V=V, heads=4)]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    with pytest.raises(B.LightKVError):
        B.lightkv_page_attention(pages, lens, Q, out, ws[:-256])
    with pytest.raises(B.LightKVError):
        B.Pages(torch.zeros(3, 2, **I32), K=K, V=V, heads=3) and B.lightkv_page_attention(B.Pages(torch.zeros(3, 2, **I32), K=K, V=V, heads=3), lens, Q[:, :3].contiguous(), out[:, :3].contiguous(), ws)
