"""Measured cases of the paged cache that decoding reads: page tables, page writes and the attention of one new token.

The compression step leaves every sequence with fewer K/V rows than it had tokens, and how many is known on the device
(`cu_vis_out`).  What follows it in a serving program is a cache in pages: pages are handed to the sequences on the device
(`lightkv_page_alloc`), the packed rows are written into them (`lightkv_page_write`), every decoded token attends to them
(`lightkv_page_attention`), and finished sequences give them back (`lightkv_page_free`).

A case is a dict of plain values.  `kind` says which operator it goes through: alloc, free, write or attend.  Lengths come
from a generator seeded with `lens`, uniform between their bounds; a share `idle` of the sequences has none.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
MAX_KV_BYTES = 700 << 20     # the keys and values that one drawn pass reads or writes at most


def listed():
    def attend(name, **kw):
        return dict(dict(name=name, kind="attend", dtype="bf16", batch=1, heads=32, kv_heads=32, head_dim=128, page=16,
                         layout="head", idle=0.0, lens=1), **kw)

    def write(name, **kw):
        return dict(dict(name=name, kind="write", dtype="bf16", batch=16, kv_heads=32, head_dim=128, page=16, layout="head",
                         old_min=0, old_max=0, idle=0.0, lens=1), **kw)

    def alloc(name, **kw):
        return dict(dict(name=name, kind="alloc", page=16, old_min=0, old_max=0, idle=0.0, short=False, lens=1), **kw)

    def free(name, **kw):
        return dict(dict(name=name, kind="free", page=16, idle=0.0, lens=1), **kw)

    return [
        # smallest call: a tiny fp32 model, three sequences after compression to 36 tokens and a prompt -- launches and host work
        attend("attend_tiny_f32", dtype="f32", batch=4, heads=4, kv_heads=4, head_dim=32, page=8, layout="token", len_min=36,
               len_max=60, idle=0.25),
        # one image of a 7B-shaped model: 317 vision tokens are left of 576, and 64 of the prompt
        attend("attend_image_7b", len_min=381, len_max=381),
        # the same model, sixteen requests with ragged prompts
        attend("attend_batch_7b", batch=16, len_min=349, len_max=573),
        # 13B-shaped heads, five image tiles (1584 of 2880 tokens are left), rows of all heads side by side as a cache is often kept
        attend("attend_tiles_13b", batch=6, heads=40, kv_heads=40, page=64, layout="token", len_min=1600, len_max=2100),
        # a serving batch under grouped queries: some rows of the captured batch are padding, lengths from one token to thousands
        attend("attend_serving_gqa", batch=64, heads=64, kv_heads=8, page=32, len_min=1, len_max=8192, idle=0.1),
        # one request with a long document: few rows, the length alone has to fill the chip
        attend("attend_long_gqa", heads=32, kv_heads=8, page=64, len_min=131000, len_max=131000),
        # a decode step: one token for each sequence, some of the batch idle
        write("write_decode", batch=64, kv_heads=8, page=32, new_min=1, new_max=1, old_min=40, old_max=700, idle=0.1),
        # rows of a compressed prefill batch with their prompts, 7B-shaped
        write("write_prefill_7b", new_min=349, new_max=573),
        # a decode step's tables: one token each, every sixteenth sequence opens a page
        alloc("alloc_decode", batch=64, new_min=1, new_max=1, old_min=1, old_max=4000, idle=0.1),
        # a large prefill wave whose pool runs short: the last sequences are refused
        alloc("alloc_wave", batch=700, new_min=200, new_max=5000, idle=0.02, short=True),
        # two requests of a small batch end
        free("free_some", batch=24, old_min=300, old_max=2500, done=0.1),
        # a large batch ends together
        free("free_wave", batch=900, page=8, old_min=100, old_max=9000, done=0.9),
    ]


def draw(rng: random.Random):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["attend"] * 6 + ["write"] * 2 + ["alloc"] * 2 + ["free"])
    c = dict(kind=kind, page=rng.choice([8, 16, 16, 32, 64, 128]), idle=rng.choice([0.0, 0.0, 0.1, 0.3]),
             lens=rng.randint(1, 1 << 20))
    if kind in ("attend", "write"):
        c["dtype"] = rng.choice(["bf16", "bf16", "bf16", "f32"])
        c["head_dim"] = rng.choice([32, 64, 128, 128])
        c["layout"] = rng.choice(["head", "token"])
        c["kv_heads"] = max(1, log(128, 5120) // c["head_dim"])
        row = 2 * c["kv_heads"] * c["head_dim"] * BYTES[c["dtype"]]
        if kind == "attend":
            c["heads"] = c["kv_heads"] * rng.choice([1, 1, 2, 4, 5, 7, 8, 16])
            c["batch"] = log(1, 96)
            top = min(131072, MAX_KV_BYTES // (row * c["batch"]))
            c["len_max"] = log(16, max(17, top))
            c["len_min"] = rng.choice([1, max(1, c["len_max"] // 2), c["len_max"]])
        else:
            c["batch"] = log(1, 96)
            c["new_max"] = log(1, max(2, min(4096, MAX_KV_BYTES // 5 // (row * c["batch"]))))
            c["new_min"] = rng.choice([1, max(1, c["new_max"] // 2)])
            c["old_max"] = rng.choice([0, 5, 77])
            c["old_min"] = 0
    elif kind == "alloc":
        c["batch"] = log(1, 1000)
        c["new_max"] = log(1, max(2, min(8000, 1700000 // c["batch"])))
        c["new_min"] = rng.choice([1, max(1, c["new_max"] // 2)])
        c["old_max"] = rng.choice([0, 30, 2000])
        c["old_min"] = rng.randint(0, c["old_max"])
        c["short"] = rng.random() < 0.3
    else:
        c["batch"] = log(1, 1000)
        c["old_max"] = log(10, 9000)
        c["old_min"] = rng.randint(0, c["old_max"] // 2)
        c["done"] = round(rng.uniform(0.05, 1.0), 2)
    return c


# ---- sizes ------------------------------------------------------------------------------------------------------------
def _lengths(c):
    """(tokens cached before the call, tokens that are new) of every sequence; one of the two lists is empty for some kinds."""
    r = random.Random(c["lens"])
    old, new = [], []
    for _ in range(c["batch"]):
        idle = r.random() < c["idle"]
        if c["kind"] == "attend":
            n = r.randint(c["len_min"], c["len_max"])
            old.append(0 if idle else n)
        else:
            n = r.randint(c["old_min"], c["old_max"])
            old.append(0 if idle and c["kind"] == "free" else n)
            if c["kind"] != "free":
                k = r.randint(c["new_min"], c["new_max"])
                new.append(0 if idle else k)
    if c["kind"] == "attend" and not any(old):
        old[0] = c["len_max"]
    return old, new


def _pages(n, page):
    return (n + page - 1) // page


def _layout(c):
    """Sizes that prepare(), exact() and work() agree on."""
    old, new = _lengths(c)
    total = [a + b for a, b in zip(old, new or [0] * len(old))]
    page = c["page"]
    held = [_pages(n, page) for n in (old if c["kind"] in ("alloc", "free") else total)]
    width = max([_pages(n, page) for n in total] + [1]) + 2
    used = sum(held)
    if c["kind"] == "alloc":
        need = sum(_pages(a + b, page) - _pages(a, page) for a, b in zip(old, new))
        spare = need * 4 // 5 if c["short"] else need + 5
    else:
        spare = 7
    return dict(old=old, new=new, total=total, held=held, width=width, used=used, spare=spare, n_pages=used + spare)


# ---- inputs -----------------------------------------------------------------------------------------------------------
def _rows(shape, g, dtype, outliers):
    """Gaussian rows; a share of the tokens (axis 0 or the page's token axis, folded) is four times as large."""
    x = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g)
    if outliers:
        big = torch.rand(shape[:-1], generator=g, device="cuda") < 0.05
        x.mul_(torch.where(big, 4.0, 1.0).unsqueeze(-1))
    return x.to(dtype)


def _pool(c, z, g, outliers):
    """Key and value pages, as [page, token, head, element] views of the layout that is stored."""
    P, H, D = c["page"], c["kv_heads"], c["head_dim"]
    dt = DTYPES[c["dtype"]]
    if c["layout"] == "head":
        return tuple(_rows((z["n_pages"], H, P, D), g, dt, o).transpose(1, 2) for o in outliers)
    return tuple(_rows((z["n_pages"], P, H, D), g, dt, o) for o in outliers)


def prepare(c, seed):
    z = _layout(c)
    g = torch.Generator(device="cuda").manual_seed(seed)
    i32 = dict(dtype=torch.int32, device="cuda")
    batch, page, width = c["batch"], c["page"], z["width"]
    # pages are scattered over the pool, as after hours of serving; a row's entries behind its last page are stale
    order = torch.randperm(z["n_pages"], generator=g, device="cuda").to(torch.int32)
    table = torch.randint(0, z["n_pages"], (batch, width), generator=g, **i32)
    held = torch.tensor(z["held"], device="cuda")
    table[torch.arange(width, device="cuda") < held.unsqueeze(1)] = order[:z["used"]]
    s = dict(case=c, table=table)
    if c["kind"] == "attend":
        s["K"], s["V"] = _pool(c, z, g, (True, False))
        s["seq_lens"] = torch.tensor(z["old"], **i32)
        s["Q"] = _rows((batch, c["heads"], c["head_dim"]), g, DTYPES[c["dtype"]], False)
        s["out"] = torch.empty_like(s["Q"])
        s["lse"] = torch.empty(c["heads"], batch, dtype=torch.float32, device="cuda")
    elif c["kind"] == "write":
        s["K"], s["V"] = _pool(c, z, g, (False, False))
        cu = [0]
        for n in z["new"]:
            cu.append(cu[-1] + n)
        s["cu_new"] = torch.tensor(cu, **i32)
        # the slots as lightkv_page_alloc leaves them; the row buffers are longer than what this step fills
        rows = max(cu[-1], 1) + 3
        seq = torch.repeat_interleave(torch.arange(batch), torch.tensor(z["new"]))
        at = torch.arange(cu[-1]) - torch.tensor(cu)[seq] + torch.tensor(z["old"])[seq]
        slots = torch.full((rows,), -7, dtype=torch.int32)
        slots[:cu[-1]] = table.cpu()[seq, at // page] * page + (at % page).to(torch.int32)
        s["slots"] = slots.cuda()
        s["K_rows"], s["V_rows"] = (_rows((rows, c["kv_heads"], c["head_dim"]), g, DTYPES[c["dtype"]], False) for _ in range(2))
    else:
        s["seq_lens"] = torch.tensor(z["old"], **i32)
        s["seq_lens_out"] = torch.zeros(batch, **i32)
        s["free_count"] = torch.tensor([z["spare"]], **i32)
        s["free_count_out"] = torch.zeros(1, **i32)
        s["free_pages"] = torch.full((z["n_pages"],), -1, **i32)
        s["free_pages"][:z["spare"]] = order[z["used"]:]
        if c["kind"] == "alloc":
            cu = [0]
            for n in z["new"]:
                cu.append(cu[-1] + n)
            s["cu_new"] = torch.tensor(cu, **i32)
            s["slots"] = torch.full((max(cu[-1], 1) + 5,), -7, **i32)
            s["status"] = torch.zeros(batch, **i32)
        else:
            s["done"] = (torch.rand(batch, generator=g, device="cuda") < c["done"]).to(torch.int32)
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------
def _alloc_plain(s):
    P, lens = s["case"]["page"], s["seq_lens"].long()
    cu, table, free, count = s["cu_new"].long(), s["table"], s["free_pages"], s["free_count"].long()
    batch, width = table.shape
    new = cu[1:] - cu[:-1]
    first, last = (lens + P - 1) // P, (lens + new + P - 1) // P
    over = (lens + new > width * P) | (cu[1:] > s["slots"].numel())
    need = torch.where(over, 0, last - first)
    incl = torch.cumsum(need, 0)
    ok = ~over & ((need == 0) | (incl <= count))
    j = torch.arange(width, device="cuda").unsqueeze(0)
    fresh = ok.unsqueeze(1) & (j >= first.unsqueeze(1)) & (j < (first + need).unsqueeze(1))
    at = count - 1 - ((incl - need).unsqueeze(1) + j - first.unsqueeze(1))
    table.copy_(torch.where(fresh, free[at.clamp(0, free.numel() - 1)], table))
    t = torch.arange(s["slots"].numel(), device="cuda")
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=batch - 1)
    pos = lens[b] + t - cu[b]
    slot = table[b, (pos // P).clamp(0, width - 1)].long() * P + pos % P
    slot = torch.where(ok[b], slot, -1).to(torch.int32)
    s["slots"].copy_(torch.where(t < cu[-1], slot, s["slots"]))
    s["status"].copy_(torch.where(over, 2, torch.where(ok, 0, 1)))
    s["seq_lens_out"].copy_(torch.where(ok, lens + new, lens))
    s["free_count_out"].copy_(count - torch.where(ok & (need > 0), incl, 0).amax())


def _free_plain(s):
    P, lens, table, count = s["case"]["page"], s["seq_lens"].long(), s["table"], s["free_count"].long()
    done = s["done"] != 0
    held = torch.where(done, (lens + P - 1) // P, 0)
    incl = torch.cumsum(held, 0)
    j = torch.arange(table.shape[1], device="cuda").unsqueeze(0)
    mine = j < held.unsqueeze(1)
    at = count + (incl - held).unsqueeze(1) + j
    s["free_pages"][at[mine]] = table[mine]
    s["seq_lens_out"].copy_(torch.where(done, 0, lens))
    s["free_count_out"].copy_(count + incl[-1])


def _write_plain(s):
    P = s["case"]["page"]
    slots = s["slots"].long()
    t = torch.arange(slots.numel(), device="cuda")
    put = (t < s["cu_new"][-1]) & (slots >= 0)
    at = slots[put]
    s["K"][at // P, at % P] = s["K_rows"][put]
    s["V"][at // P, at % P] = s["V_rows"][put]


def _attend_plain(s):
    K, V, table, Q = s["K"], s["V"], s["table"].long(), s["Q"]
    batch, heads, D = Q.shape
    P, H = K.shape[1], K.shape[2]
    lens = s["seq_lens"].long()
    top = s["case"]["len_max"]
    t = torch.arange(top, device="cuda")
    page, at = table[:, t // P], (t % P).unsqueeze(0)
    k = K[page, at].float().permute(0, 2, 3, 1)                                   # [batch, kv head, element, token]
    q = Q.float().view(batch, H, heads // H, D)
    x = torch.matmul(q, k) / math.sqrt(D)
    del k
    live = (t < lens.unsqueeze(1)).view(batch, 1, 1, top)
    x = torch.where(live, x, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(m == -math.inf, 0.0, m))
    l = p.sum(-1, keepdim=True)
    v = V[page, at].float().permute(0, 2, 1, 3)
    o = torch.matmul(p, v) / torch.where(l == 0, 1.0, l)
    s["out"].copy_(o.view(batch, heads, D))
    s["lse"].copy_((m + torch.log(l)).view(batch, heads).t())


def _own_handle(s):
    """The descriptor and workspace that a program makes once for its cache."""
    import paper_2605_00789_amd as lk
    if "pages" not in s:
        c = s["case"]
        if "K" in s:
            s["pages"] = lk.Pages(s["table"], K=s["K"], V=s["V"], heads=c.get("heads", c["kv_heads"]))
        else:
            s["pages"] = lk.Pages(s["table"], n_pages=s["free_pages"].numel(), page_tokens=c["page"])
        if c["kind"] == "attend":
            s["ws"] = torch.empty(lk.lightkv_page_attention_workspace(s["pages"]), dtype=torch.uint8, device="cuda")
    return lk, s["pages"]


def run(s):
    kind = s["case"]["kind"]
    if kind == "alloc":
        if own:
            lk, pages = _own_handle(s)
            lk.lightkv_page_alloc(pages, s["cu_new"], s["seq_lens"], s["free_pages"], s["free_count"], s["seq_lens_out"],
                                  s["free_count_out"], s["slots"], status=s["status"])
        else:
            _alloc_plain(s)
        return {k: s[k] for k in ("table", "slots", "seq_lens_out", "free_count_out", "status")}
    if kind == "free":
        if own:
            lk, pages = _own_handle(s)
            lk.lightkv_page_free(pages, s["done"], s["seq_lens"], s["free_pages"], s["free_count"], s["seq_lens_out"],
                                 s["free_count_out"])
        else:
            _free_plain(s)
        return {k: s[k] for k in ("free_pages", "seq_lens_out", "free_count_out")}
    if kind == "write":
        if own:
            lk, pages = _own_handle(s)
            lk.lightkv_page_write(pages, s["slots"], s["K_rows"], s["V_rows"], cu_new=s["cu_new"])
        else:
            _write_plain(s)
        return {"K": s["K"], "V": s["V"]}
    if own:
        lk, pages = _own_handle(s)
        lk.lightkv_page_attention(pages, s["seq_lens"], s["Q"], s["out"], s["ws"], lse=s["lse"])
    else:
        _attend_plain(s)
    return {"out": s["out"], "lse": s["lse"]}


# ---- what a pass cannot do without ------------------------------------------------------------------------------------
def work(c):
    z = _layout(c)
    tokens, batch = sum(z["old"]), c["batch"]
    if c["kind"] == "attend":
        e, D = BYTES[c["dtype"]], c["head_dim"]
        kv = 2 * tokens * c["kv_heads"] * D * e
        q = 2 * batch * c["heads"] * D * e + 4 * batch * c["heads"]
        return {"bytes": kv + q + 4 * (z["used"] + batch), "flops": 4 * tokens * c["heads"] * D}
    if c["kind"] == "write":
        rows = sum(z["new"])
        return {"bytes": 4 * rows * c["kv_heads"] * c["head_dim"] * BYTES[c["dtype"]] + 4 * (rows + 1), "flops": 0}
    if c["kind"] == "alloc":
        rows = sum(z["new"])
        need = min(z["spare"], sum(_pages(n, c["page"]) for n in z["total"]) - z["used"])
        return {"bytes": 4 * (rows + 2 * need + 4 * batch + 3), "flops": 0}
    moved = int(round(sum(z["held"]) * c["done"]))
    return {"bytes": 4 * (2 * moved + 3 * batch + 2), "flops": 0}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------
def exact(c, seed):
    s = prepare(c, seed)
    page = c["page"]
    if c["kind"] == "attend":
        # sequence by sequence, the pages of its row one behind the other, everything in doubles
        lens = s["seq_lens"].tolist()
        H = c["kv_heads"]
        share = c["heads"] // H
        out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            if n == 0:
                continue
            rows = s["table"][b, :_pages(n, page)].long()
            for h in range(H):
                k = s["K"][rows, :, h].reshape(-1, c["head_dim"])[:n].double()
                v = s["V"][rows, :, h].reshape(-1, c["head_dim"])[:n].double()
                q = s["Q"][b, h * share:(h + 1) * share].double()
                x = (q.unsqueeze(1) * k.unsqueeze(0)).sum(-1) * c["head_dim"] ** -0.5 if n * share < 20000 else q @ k.t() * c["head_dim"] ** -0.5
                z = torch.logsumexp(x, 1)
                out[b, h * share:(h + 1) * share] = torch.exp(x - z.unsqueeze(1)) @ v
                lse[h * share:(h + 1) * share, b] = z
        return {"out": out, "lse": lse}
    if c["kind"] == "write":
        # row by row: a copy has no rounding
        K, V = (s[k].cpu().double() for k in ("K", "V"))
        rows_k, rows_v = (s[k].cpu().double() for k in ("K_rows", "V_rows"))
        for t, slot in enumerate(s["slots"].tolist()[:int(s["cu_new"][-1])]):
            if slot >= 0:
                K[slot // page, slot % page] = rows_k[t]
                V[slot // page, slot % page] = rows_v[t]
        return {"K": K, "V": V}
    # tables: one sequence after the other, with a stack of pages on the host
    table, lens = s["table"].tolist(), s["seq_lens"].tolist()
    stack = s["free_pages"].tolist()
    count = int(s["free_count"])
    ints = lambda v: torch.tensor(v, dtype=torch.int32)
    if c["kind"] == "free":
        for b, d in enumerate(s["done"].tolist()):
            if d:
                n = _pages(lens[b], page)
                stack[count:count + n] = table[b][:n]
                count += n
                lens[b] = 0
        return {"free_pages": ints(stack), "seq_lens_out": ints(lens), "free_count_out": ints([count])}
    cu, slots, status = s["cu_new"].tolist(), s["slots"].tolist(), [0] * c["batch"]
    width, asked = s["table"].shape[1], 0
    have = count
    for b in range(c["batch"]):
        new, old = cu[b + 1] - cu[b], lens[b]
        need = _pages(old + new, page) - _pages(old, page)
        if old + new > width * page:
            status[b] = 2
        else:
            asked += need                      # a refused sequence keeps its place in the queue
            if need and asked > count:
                status[b] = 1
        if status[b]:
            slots[cu[b]:cu[b + 1]] = [-1] * new
            continue
        for k in range(need):
            have -= 1
            table[b][_pages(old, page) + k] = stack[have]
        slots[cu[b]:cu[b + 1]] = [table[b][p // page] * page + p % page for p in range(old, old + new)]
        lens[b] = old + new
    return {"table": ints(table), "slots": ints(slots), "seq_lens_out": ints(lens), "free_count_out": ints([have]),
            "status": ints(status)}
