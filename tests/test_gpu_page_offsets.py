"""lightkv_page_alloc where the offsets of the new tokens fall: what is granted, the slots and the table agree, and a write of the same
offsets reaches every row that got a slot."""
import random

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_pages import DEV, DeviceTables, HostTables, I32, ints, same  # noqa: E402


class AnyOffsets(HostTables):
    """HostTables for offsets in any order: a row has one owner, the first sequence with possible rows that it belongs to."""

    def alloc(self, cu, slots):
        asked, had, status, slots, rows = 0, self.count, [], list(slots), len(slots)
        falls, claimed, before = any(a > b for a, b in zip(cu, cu[1:])), cu[0], list(self.lens)
        for b in range(len(self.lens)):
            n, L = cu[b + 1] - cu[b], self.lens[b]
            bad = cu[b] < 0 or n < 0 or cu[b + 1] > rows or L < 0 or L + n > self.width * self.P
            if bad or falls and (cu[b] < claimed or cu[b + 1] > cu[-1]):
                status.append(2)
                continue
            claimed = cu[b + 1]
            need = self.pages(L + n) - self.pages(L)
            asked += need
            status.append(1 if need and asked > had else 0)
            if status[-1] == 0:
                for j in range(self.pages(L), self.pages(L + n)):
                    self.count -= 1
                    self.table[b][j] = self.stack[self.count]
                self.lens[b] = L + n
        for t in range(max(cu[0], 0), min(cu[-1], rows)):
            slots[t] = -1
            for b, s in enumerate(status):
                if s == 0 and cu[b] <= t < cu[b + 1]:
                    pos = before[b] + t - cu[b]
                    slots[t] = self.table[b][pos // self.P] * self.P + pos % self.P
        return slots, status


def check(h, d, cu, slots):
    want, got = h.alloc(cu, slots), d.alloc(cu, slots)
    assert got[1] == want[1], cu
    assert got[0] == want[0], cu
    same(d, h)
    # every token a sequence holds has a page that nobody else has, and that is off the stack
    held = [p for b, n in enumerate(h.lens) for p in h.table[b][:h.pages(n)]]
    assert len(set(held)) == len(held) and not set(held) & set(h.stack[:h.count]) and all(0 <= p < h.n_pages for p in held)
    return want[1]


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("rows", [40, 700, 3000])
@pytest.mark.parametrize("P,cu,status", [
    (8, [0, 10, 5, 20], [0, 2, 2]),            # rows 5 to 9 twice: they stay the first sequence's
    (16, [0, 16, 32, 0], [2, 2, 2]),           # a write of these offsets covers no row
    (16, [0, 16, 32, 20], [0, 2, 2]),          # rows 16 to 31 end behind cu[batch]
    (8, [4, 2, 9, 30], [2, 2, 0]),             # rows 2 to 8 begin in front of cu[0]
    (8, [8, 4, -3, 30, 10, 12, 38], [2, 2, 2, 2, 0, 0]),
    (8, [0, 9, 9, 3, 3, 9, 20], [0, 0, 2, 2, 2, 0]),
])
def test_offsets_that_fall(P, cu, status, rows, in_place):
    print("[falling]", P, cu, rows, in_place, flush=True)
    batch, n_pages = len(cu) - 1, 60
    stack = random.Random(3).sample(range(n_pages), 50)
    h, d = AnyOffsets(batch, n_pages, P, 8, stack), DeviceTables(batch, n_pages, P, 8, stack, in_place)
    assert check(h, d, cu, [-7] * rows) == status
    for _ in range(2):                          # what was granted goes on as it should
        assert check(h, d, list(range(0, 3 * batch + 1, 3)), [-7] * rows) == [0] * batch


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("batch,P,most,spare", [(3, 8, 9, 12), (40, 16, 60, 90), (300, 8, 12, 500), (1000, 32, 8, 900)])
def test_offsets_in_any_order(batch, P, most, spare, in_place):
    """Ascending offsets with some of them moved, or put where no row is; pools that run short among them."""
    print("[any order]", batch, P, most, spare, in_place, flush=True)
    rng = random.Random(batch)
    n_pages = spare + 3
    stack = rng.sample(range(n_pages), spare)
    h, d = AnyOffsets(batch, n_pages, P, 6, stack), DeviceTables(batch, n_pages, P, 6, stack, in_place, stride=9)
    for call in range(6):
        cu = [rng.choice([0, 2])]
        for _ in range(batch):
            cu.append(cu[-1] + rng.choice([0, 1, rng.randint(0, most)]))
        rows = max(cu[-1] + rng.choice([0, 5]), 1)
        for _ in range(rng.choice([0, 1, 2, batch // 3])):
            i = rng.randrange(batch + 1)
            cu[i] = rng.choice([max(cu[i] - rng.randint(1, most), 0), min(cu[i] + rng.randint(1, most), 2 ** 31 - 1), rng.randint(0, rows), -3, rows + 9, 2 ** 31 - 1, -2 ** 31])
        check(h, d, cu, [-7] * rows)
        done = [int(rng.random() < 0.3) for _ in range(batch)]
        h.free(done)
        d.free(done)
        same(d, h)
    assert (d.store[:, 6:] == -5).all()


def test_a_write_reaches_every_row_that_was_granted():
    from paper_2605_00789_amd import binding as B
    P, cu = 8, [4, 1, 20, 12, 18, 30, 23]       # rows 12 to 17 and 18 to 22: sequence 3 is granted, 4 ends behind cu[batch]
    h, d = AnyOffsets(6, 20, P, 3, list(range(20))), DeviceTables(6, 20, P, 3, list(range(20)), True)
    slots, status = h.alloc(cu, [5] * 40)       # (5: a slot of an earlier call)
    got = ints([5] * 40)
    st = torch.zeros(6, **I32)
    B.lightkv_page_alloc(d.pages, ints(cu), d.lens, d.stack, d.count, d.lens, d.count, got, status=st)
    assert got.tolist() == slots and st.tolist() == status == [2, 2, 2, 0, 2, 2]
    K, V = (torch.zeros(20, P, 1, 32, device=DEV) for _ in range(2))
    rows = torch.arange(1, 41, device=DEV).float().view(40, 1, 1).expand(40, 1, 32).contiguous()
    B.lightkv_page_write(B.Pages(d.table, K=K, V=V, heads=1), got, rows, 2 * rows, cu_new=ints(cu))
    want = torch.zeros(20, P)
    for pos in range(6):
        want[d.table[3, 0].item(), pos] = 12 + pos + 1
    assert torch.equal(K[:, :, 0, 7].cpu(), want) and torch.equal(V[:, :, 0, 7].cpu(), 2 * want)
