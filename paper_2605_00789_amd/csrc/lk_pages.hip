// Tables of a paged K/V cache, built on the device from sequence lengths, and the rows that go into its pages.
//
// Pages and slots (lightkv_page_alloc).  With L = seq_lens, n = new tokens, P = page_tokens:
//   need_b = ceil((L_b + n_b) / P) - ceil(L_b / P),  queue_b = sum_{b' < b} need_b',
//   page j of sequence b, j >= ceil(L_b / P), is free_pages[count - 1 - (queue_b + j - ceil(L_b / P))],
//   slot of the token at position x = table[b][x / P] * P + x % P.
// The only dependence between sequences is the running sum over at most 4096 small numbers.  It is taken again by every
// workgroup, in LDS: one trip to memory and one scan, where a launch that leaves it in memory for a second one would cost
// the second launch and the same trip.  A page that is handed out begins with a new token, so the thread that makes that token's
// slot also writes the table entry and nothing has to be scattered separately.  The time is that chain -- lengths, sum, search,
// page, store -- 4.0 us in a graph for a token each of 64 sequences, 8.9 a call for 1.8 M slots of 700 (7 MB).  Lengths in place and more
// than one workgroup: a second launch, 5.8 us for 64 sequences and 1024 slots, 7.4 for 16 and 9216.
#include "lk_common.h"
#include "lk_pages.h"

namespace lk {

constexpr int PG_THREADS = 256;
constexpr int PG_SLOTS_PER_THREAD = 4;     // one 16-byte store, mostly one page to look up
// Up to so many, one workgroup and a slot a thread: decoded tokens have a page each to look up.  us, a slot / four slots a thread: 64
// sequences of a token 4.2 / 6.2, 256 4.5 / 6.5, 4 of 100 tokens 4.6 / 5.3; 8 of 120 6.2 / 5.5, 1000 of a token 9.8 / 8.2.
constexpr int PG_FEW_SLOTS = 512;
// Workgroups of a launch at most: each takes the running sum again, and fewer leave the slots to too few waves.  1.8 M slots of 700
// sequences with 512 / 1024 / 1536: 14.8 / 10.6 / 9.9 us, 1.25 M of 1000 13.3 / 10.9 / 9.6.
constexpr int PG_MAX_WGS = 1536;
constexpr int PG_SAT = 1 << 29;            // sums of impossible lengths stop here: above any number of pages

struct AllocArgs {
  const int32_t *cu_new, *seq_lens, *free_pages, *free_count;
  int32_t *table, *seq_lens_out, *free_count_out, *slots, *status, *cu_copy;
  int64_t table_stride, slot_rows;
  int batch, max_pages, n_pages, lg, skip_empty;
  int what;   // 1: slots and table, 2: lengths, count, status and the copy of the offsets
};

__device__ __forceinline__ int sat_add(int a, int b) { const int s = a + b; return s < PG_SAT ? s : PG_SAT; }

// Exclusive running sum (saturating) of one number per thread over the workgroup; *total is the sum of all.
__device__ __forceinline__ int wg_exclusive_sum(int v, int *scratch, int *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int incl = wave_running(v, sat_add);
  if (lane == 63) scratch[wave] = incl;
  __syncthreads();
  int base = 0, sum = 0;
#pragma unroll
  for (int w = 0; w < PG_THREADS / 64; ++w) {
    if (w < wave) base = sat_add(base, scratch[w]);
    sum = sat_add(sum, scratch[w]);
  }
  *total = sum;
  return sat_add(base, __builtin_amdgcn_update_dpp(0, incl, 0x138, 0xf, 0xf, false));   // wave_shr 1
}

// Last index i in [0, n) with list[i] <= v (list ascending, list[0] <= v).
__device__ __forceinline__ int last_not_above(const int *list, int n, int v) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (list[mid] <= v) lo = mid;
    else hi = mid;
  }
  return lo;
}

// n ints into LDS by the whole workgroup, four loads of a thread at a time.
__device__ __forceinline__ void pg_fetch(const int32_t *from, int *to, int n) {
  for (int i0 = threadIdx.x; i0 < n; i0 += 4 * PG_THREADS) {
    int v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = i0 + u * PG_THREADS < n ? from[i0 + u * PG_THREADS] : 0;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * PG_THREADS < n) to[i0 + u * PG_THREADS] = v[u];
  }
}

// n + 1 offsets and n lengths, all of a thread's loads on their way at once.
__device__ __forceinline__ void pg_fetch_both(const int32_t *cu, int *to_cu, const int32_t *len, int *to_len, int n) {
  for (int i0 = threadIdx.x; i0 <= n; i0 += 2 * PG_THREADS) {
    int c[2], l[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = i0 + u * PG_THREADS;
      c[u] = i <= n ? cu[i] : 0;
      l[u] = i < n ? len[i] : 0;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = i0 + u * PG_THREADS;
      if (i <= n) to_cu[i] = c[u];
      if (i < n) to_len[i] = l[u];
    }
  }
}

__device__ __forceinline__ int clamped_count(const int32_t *count, int n_pages) {
  const int c = count[0];
  return c < 0 ? 0 : (c > n_pages ? n_pages : c);
}

// LDS: cu [batch + 1], length [batch], queue place [batch], or minus the status
template <int SLOTS>
__global__ __launch_bounds__(PG_THREADS) void page_alloc_kernel(AllocArgs g) {
  fetch_args<AllocArgs>();
  extern __shared__ int pg_lds[];
  __shared__ int scratch[PG_THREADS / 64];
  __shared__ int popped;
  int *cu = pg_lds, *len = cu + g.batch + 1, *place = len + g.batch;
  const int tid = threadIdx.x, count = clamped_count(g.free_count, g.n_pages);
  const int room = g.max_pages << g.lg, P = 1 << g.lg;
  const int per = (g.batch + PG_THREADS - 1) / PG_THREADS, b0 = tid * per, b1 = b0 + per < g.batch ? b0 + per : g.batch;
  if (tid == 0) popped = 0;
  pg_fetch_both(g.cu_new, cu, g.seq_lens, len, g.batch);
  __syncthreads();
  // pages that a sequence asks for; -2: its lengths or offsets are impossible, -3: it is left out
  auto need_of = [&](int b, bool &falls) {
    const int first = cu[b], end = cu[b + 1], L = len[b];
    const unsigned n = (unsigned)end - (unsigned)first;
    falls = end < first;
    const bool bad = ((first | L) < 0) | falls | (end > (int)g.slot_rows) | ((unsigned)L + n > (unsigned)room);
    const int need = (int)(((unsigned)L + n + P - 1) >> g.lg) - (int)(((unsigned)L + P - 1) >> g.lg);
    return bad ? -2 : (g.skip_empty && L == 0 && n != 0 ? -3 : need);
  };
  int mine = 0;
  for (int b = b0; b < b1; ++b) {
    bool falls;
    const int need = need_of(b, falls);
    place[b] = need;
    mine = sat_add(mine, falls ? PG_SAT : (need < 0 ? 0 : need));   // offsets that fall: a sum that no pool has
  }
  int total;
  int at = wg_exclusive_sum(mine, scratch, &total), served = 0;
  const bool slow = total == PG_SAT;   // (the same in all threads; ascending offsets below 2^31 take 2^28 pages and one each at most)
  if (!slow) {
    for (int b = b0; b < b1; ++b) {
      const int need = place[b];
      if (need < 0) continue;
      const bool ok = need == 0 || sat_add(at, need) <= count;
      place[b] = ok ? at : -1;
      at = sat_add(at, need);
      if (ok && need > 0) served = at;
    }
  } else if (tid == 0) {
    // Offsets that fall: no program should have them, so one thread decides, sequence by sequence.  A row has one owner, inside the
    // range that a write of these offsets covers: a sequence is refused if its rows begin in front of cu[0] or of the end of
    // one that was not, or end behind cu[batch].
    int claimed = cu[0];
    at = 0;
    for (int b = 0; b < g.batch; ++b) {
      bool falls;
      int need = need_of(b, falls);
      if (need != -2 && (cu[b] < claimed || cu[b + 1] > cu[g.batch])) need = -2;
      place[b] = need;
      if (need == -2) continue;
      claimed = cu[b + 1];
      if (need < 0) continue;
      const bool ok = need == 0 || sat_add(at, need) <= count;
      place[b] = ok ? at : -1;
      at = sat_add(at, need);
      if (ok && need > 0) served = at;
    }
  }
  if ((g.what & 2) && blockIdx.x == 0) {
    served = wave_running_max(served);
    if ((tid & 63) == 63) atomicMax(&popped, served);
  }
  __syncthreads();
  if ((g.what & 2) && blockIdx.x == 0) {
    for (int b = tid; b < g.batch; b += PG_THREADS) {
      const int p = place[b];
      g.seq_lens_out[b] = p >= 0 ? len[b] + (cu[b + 1] - cu[b]) : len[b];
      if (g.status) g.status[b] = p >= 0 ? 0 : -p;
    }
    if (g.cu_copy)
      for (int i = tid; i <= g.batch; i += PG_THREADS) g.cu_copy[i] = cu[i];
    if (tid == 0) g.free_count_out[0] = count - popped;
  }
  if (!(g.what & 1)) return;
  const int64_t end = cu[g.batch] < g.slot_rows ? cu[g.batch] : g.slot_rows;
  if (slow) {   // a slot at a time, its owner among all sequences
    for (int64_t t = (int64_t)blockIdx.x * PG_THREADS + tid; t < end; t += (int64_t)gridDim.x * PG_THREADS) {
      if (t < cu[0]) continue;
      int b = 0, page = -1;
      while (b < g.batch && (place[b] == -2 || t < cu[b] || t >= cu[b + 1])) ++b;
      const int pos = b < g.batch && place[b] >= 0 ? len[b] + (int)(t - cu[b]) : -1;
      if (pos >= 0) {
        const int j = pos >> g.lg, old = (len[b] + P - 1) >> g.lg;
        page = j < old ? g.table[(int64_t)b * g.table_stride + j] : g.free_pages[count - 1 - (place[b] + j - old)];
        if (j >= old && (pos & (P - 1)) == 0) g.table[(int64_t)b * g.table_stride + j] = page;
      }
      g.slots[t] = (unsigned)page < (unsigned)g.n_pages ? (page << g.lg) + (pos & (P - 1)) : -1;
    }
    return;
  }
  const int64_t step = (int64_t)gridDim.x * PG_THREADS * SLOTS;
  const bool wide = (reinterpret_cast<uintptr_t>(g.slots) & 15) == 0;
  for (int64_t t0 = ((int64_t)blockIdx.x * PG_THREADS + tid) * SLOTS; t0 < end; t0 += step) {
    int b = 0, page = -1, page_j = -1, page_b = -1, out[SLOTS];
    unsigned have = 0;
    if (cu[0] <= t0) b = last_not_above(cu, g.batch, (int)t0);
#pragma unroll
    for (int i = 0; i < SLOTS; ++i) {
      const int64_t t = t0 + i;
      out[i] = -1;
      if (t >= end) continue;
      while (b + 1 < g.batch && t >= cu[b + 1]) ++b;
      if (t < cu[b] || t >= cu[b + 1]) continue;   // a row no sequence owns
      have |= 1u << i;
      if (place[b] < 0) continue;
      const int L = len[b], pos = L + (int)(t - cu[b]), j = pos >> g.lg, old = (L + P - 1) >> g.lg;
      if (j != page_j || b != page_b) {   // (mostly one page for the slots of a thread: one trip to memory)
        page = j < old ? g.table[(int64_t)b * g.table_stride + j] : g.free_pages[count - 1 - (place[b] + j - old)];
        page_j = j;
        page_b = b;
      }
      if (j >= old && (pos & (P - 1)) == 0) g.table[(int64_t)b * g.table_stride + j] = page;
      if ((unsigned)page < (unsigned)g.n_pages) out[i] = (page << g.lg) + (pos & (P - 1));
    }
    if (SLOTS == 4 && wide && have == (1u << SLOTS) - 1) {
      *reinterpret_cast<int4 *>(g.slots + t0) = int4{out[0], out[1 % SLOTS], out[2 % SLOTS], out[3 % SLOTS]};
    } else {
#pragma unroll
      for (int i = 0; i < SLOTS; ++i)
        if (have & (1u << i)) g.slots[t0 + i] = out[i];
    }
  }
}

struct FreeArgs {
  const int32_t *done, *seq_lens, *free_count, *table;
  int32_t *free_pages, *seq_lens_out, *free_count_out;
  int64_t table_stride;
  int batch, max_pages, n_pages, lg;
  int what;   // 1: the stack, 2: lengths and count
};

// LDS: flag, then pages pushed before sequence b [batch]; length [batch]
__global__ __launch_bounds__(PG_THREADS) void page_free_kernel(FreeArgs g) {
  fetch_args<FreeArgs>();
  extern __shared__ int pg_lds[];
  __shared__ int scratch[PG_THREADS / 64];
  int *before = pg_lds;
  const int tid = threadIdx.x, count = clamped_count(g.free_count, g.n_pages), P = 1 << g.lg;
  const int per = (g.batch + PG_THREADS - 1) / PG_THREADS, b0 = tid * per, b1 = b0 + per < g.batch ? b0 + per : g.batch;
  int *len = before + g.batch;
  pg_fetch(g.seq_lens, len, g.batch);
  pg_fetch(g.done, before, g.batch);
  __syncthreads();
  int mine = 0;
  for (int b = b0; b < b1; ++b) {
    const int L = len[b];
    int held = 0;
    if (before[b] != 0 && L > 0) {
      held = (int)(((int64_t)L + P - 1) >> g.lg);
      held = held < g.max_pages ? held : g.max_pages;
    }
    before[b] = held;
    mine = sat_add(mine, held);
  }
  int total;
  int at = wg_exclusive_sum(mine, scratch, &total);
  for (int b = b0; b < b1; ++b) {
    const int held = before[b];
    before[b] = at;
    at = sat_add(at, held);
  }
  __syncthreads();
  const int room = g.n_pages - count, pushed = total < room ? total : room;
  if ((g.what & 2) && blockIdx.x == 0) {
    for (int b = tid; b < g.batch; b += PG_THREADS) g.seq_lens_out[b] = g.done[b] != 0 ? 0 : len[b];
    if (tid == 0) g.free_count_out[0] = count + pushed;
  }
  if (!(g.what & 1)) return;
  for (int k = blockIdx.x * PG_THREADS + tid; k < pushed; k += gridDim.x * PG_THREADS) {
    const int b = last_not_above(before, g.batch, k);
    g.free_pages[count + k] = g.table[(int64_t)b * g.table_stride + (k - before[b])];
  }
}

// Rows into pages: both streams of rows are read and written once, so the time is that of a copy: 242 MB of traffic in 42.0 us, 5.8
// TB/s, what the best copies here reach.  A workgroup takes whole rows of K (blockIdx.y 0) or V (1), 16 bytes a thread and load.
constexpr int PG_WRITE_U = 4;   // loads of a thread on their way at once; 121 MB of rows with one 50.7 us, with four 46.9
// Rows of more than the L2 caches hold pass them by, in and out.  us a call, through the caches / past them: 121 MB of rows 46.9 / 43.0,
// 262 MB 100.2 / 96.3; 19 MB 8.2 / 8.9, 4 MB 3.7 / 4.0.
constexpr uint64_t PG_STREAM_BYTES = 32u << 20;

struct WriteArgs {
  const int32_t *cu_new, *slots;
  const char *src[2];
  char *dst[2];
  int64_t src_tok[2], src_head[2];               // bytes
  int64_t dst_page[2], dst_tok[2], dst_head[2];
  int64_t rows;
  int batch, n_slots, lg, pieces_per_row, lg_pieces;   // pieces of 16 bytes in a row, log2 of those in a head
  int rows_per_wg;
};

template <bool STREAM>
__global__ __launch_bounds__(PG_THREADS) void page_write_kernel(WriteArgs g) {
  fetch_args<WriteArgs>();
  const int y = blockIdx.y;
  int64_t rows = g.rows;
  int begin = 0;
  if (g.cu_new) {
    const int n = g.cu_new[g.batch];
    rows = n < rows ? n : rows;
    begin = g.cu_new[0];
  }
  const int per = g.pieces_per_row, in_head = (1 << g.lg_pieces) - 1;
  for (int64_t r0 = (int64_t)blockIdx.x * g.rows_per_wg; r0 < rows; r0 += (int64_t)gridDim.x * g.rows_per_wg) {
    const int n_rows = rows - r0 < g.rows_per_wg ? (int)(rows - r0) : g.rows_per_wg;
    // all loads of a thread are on their way before the first store
    for (int i0 = threadIdx.x; i0 < n_rows * per; i0 += PG_THREADS * PG_WRITE_U) {
      uint4 v[PG_WRITE_U];
      int slot[PG_WRITE_U], head[PG_WRITE_U], piece[PG_WRITE_U];
#pragma unroll
      for (int u = 0; u < PG_WRITE_U; ++u) {
        const int i = i0 + u * PG_THREADS, r = i / per, k = i - r * per;
        head[u] = k >> g.lg_pieces;
        piece[u] = (k & in_head) * 16;
        slot[u] = -1;
        if (i < n_rows * per && r0 + r >= begin) slot[u] = g.slots[r0 + r];
        v[u] = uint4{0u, 0u, 0u, 0u};
        const char *from = g.src[y] + (r0 + r) * g.src_tok[y] + head[u] * g.src_head[y] + piece[u];
        if (i < n_rows * per) v[u] = STREAM ? ld16_stream(from) : ld16(from);
      }
#pragma unroll
      for (int u = 0; u < PG_WRITE_U; ++u) {
        if ((unsigned)slot[u] >= (unsigned)g.n_slots) continue;
        char *to = g.dst[y] + (int64_t)(slot[u] >> g.lg) * g.dst_page[y] + (int64_t)(slot[u] & ((1 << g.lg) - 1)) * g.dst_tok[y] + head[u] * g.dst_head[y] + piece[u];
        if (STREAM) st16_stream(to, v[u]);
        else *reinterpret_cast<uint4 *>(to) = v[u];
      }
    }
  }
}

}  // namespace lk

using namespace lk;

extern "C" {

lightkv_status lightkv_page_alloc(const lightkv_pages *p, const int32_t *cu_new, const int32_t *seq_lens,
                                  const int32_t *free_pages, const int32_t *free_count, int32_t *seq_lens_out,
                                  int32_t *free_count_out, int32_t *slots, int64_t slot_rows, int32_t *status,
                                  void *stream) {
  const lightkv_status st = check_page_table(p);
  if (st != LIGHTKV_OK) return st;
  if (!cu_new || !seq_lens || !free_pages || !free_count || !seq_lens_out || !free_count_out || !slots) return LIGHTKV_ERR_NULL;
  if (slot_rows < 0) return LIGHTKV_ERR_SHAPE;
  if (slot_rows >= (1ll << 31)) return LIGHTKV_ERR_UNSUPPORTED;
  int32_t *const cu_copy = p->cu_copy == cu_new ? nullptr : p->cu_copy;   // (it has them already)
  const void *all[] = {cu_new, seq_lens, free_pages, free_count, seq_lens_out, free_count_out, slots, status, cu_copy};
  for (const void *q : all)
    if (!aligned_to(q, 4)) return LIGHTKV_ERR_UNSUPPORTED;
  const uint64_t nb = (uint64_t)p->batch * 4, np = (uint64_t)p->n_pages * 4, nt = ((uint64_t)p->table_stride * (p->batch - 1) + p->max_pages) * 4;
  struct Range { const void *at; uint64_t bytes; };
  const Range in[] = {{cu_new, nb + 4}, {seq_lens, nb}, {free_pages, np}, {free_count, 4}};
  const Range out[] = {{p->table, nt}, {slots, (uint64_t)slot_rows * 4}, {seq_lens_out, nb}, {free_count_out, 4}, {status, nb}, {cu_copy, nb + 4}};
  for (int i = 0; i < 6; ++i) {
    for (const Range &r : in) {
      if (r.at == out[i].at && ((r.at == seq_lens && i == 2) || (r.at == free_count && i == 3))) continue;
      if (overlap(r.at, r.bytes, out[i].at, out[i].bytes)) return LIGHTKV_ERR_SHAPE;
    }
    for (int j = 0; j < i; ++j)
      if (overlap(out[j].at, out[j].bytes, out[i].at, out[i].bytes)) return LIGHTKV_ERR_SHAPE;
  }
  AllocArgs g{};
  g.cu_new = cu_new; g.seq_lens = seq_lens; g.free_pages = free_pages; g.free_count = free_count; g.table = p->table;
  g.seq_lens_out = seq_lens_out; g.free_count_out = free_count_out; g.slots = slots; g.status = status;
  g.cu_copy = cu_copy; g.skip_empty = p->skip_empty; g.table_stride = p->table_stride; g.slot_rows = slot_rows; g.batch = p->batch; g.max_pages = p->max_pages;
  g.n_pages = p->n_pages; g.lg = log2_of(p->page_tokens);
  const size_t lds = (3 * (size_t)p->batch + 1) * sizeof(int);
  const bool few = slot_rows <= PG_FEW_SLOTS;
  const int64_t per_wg = PG_THREADS * PG_SLOTS_PER_THREAD, want = few ? 1 : (slot_rows + per_wg - 1) / per_wg;
  const int wgs = (int)(want < 1 ? 1 : (want > PG_MAX_WGS ? PG_MAX_WGS : want));
  // lengths and count may be written in place: then only behind the workgroups that still read them
  const bool in_place = seq_lens_out == seq_lens || free_count_out == free_count;
  g.what = wgs > 1 && in_place ? 1 : 3;
  hipLaunchKernelGGL(few ? page_alloc_kernel<1> : page_alloc_kernel<PG_SLOTS_PER_THREAD>, dim3(wgs), dim3(PG_THREADS), lds, static_cast<hipStream_t>(stream), g);
  if (g.what == 1) {
    if (hipGetLastError() != hipSuccess) return LIGHTKV_ERR_LAUNCH;
    g.what = 2;
    hipLaunchKernelGGL(page_alloc_kernel<PG_SLOTS_PER_THREAD>, dim3(1), dim3(PG_THREADS), lds, static_cast<hipStream_t>(stream), g);
  }
  return hipGetLastError() == hipSuccess ? LIGHTKV_OK : LIGHTKV_ERR_LAUNCH;
}

lightkv_status lightkv_page_free(const lightkv_pages *p, const int32_t *done, const int32_t *seq_lens, int32_t *free_pages,
                                 const int32_t *free_count, int32_t *seq_lens_out, int32_t *free_count_out, void *stream) {
  const lightkv_status st = check_page_table(p);
  if (st != LIGHTKV_OK) return st;
  if (!done || !seq_lens || !free_pages || !free_count || !seq_lens_out || !free_count_out) return LIGHTKV_ERR_NULL;
  const void *all[] = {done, seq_lens, free_pages, free_count, seq_lens_out, free_count_out};
  for (const void *q : all)
    if (!aligned_to(q, 4)) return LIGHTKV_ERR_UNSUPPORTED;
  const uint64_t nb = (uint64_t)p->batch * 4, np = (uint64_t)p->n_pages * 4, nt = ((uint64_t)p->table_stride * (p->batch - 1) + p->max_pages) * 4;
  struct Range { const void *at; uint64_t bytes; };
  const Range in[] = {{done, nb}, {seq_lens, nb}, {free_count, 4}, {p->table, nt}};
  const Range out[] = {{free_pages, np}, {seq_lens_out, nb}, {free_count_out, 4}};
  for (int i = 0; i < 3; ++i) {
    for (const Range &r : in) {
      if (r.at == out[i].at && ((r.at == seq_lens && i == 1) || (r.at == free_count && i == 2))) continue;
      if (overlap(r.at, r.bytes, out[i].at, out[i].bytes)) return LIGHTKV_ERR_SHAPE;
    }
    for (int j = 0; j < i; ++j)
      if (overlap(out[j].at, out[j].bytes, out[i].at, out[i].bytes)) return LIGHTKV_ERR_SHAPE;
  }
  FreeArgs g{};
  g.done = done; g.seq_lens = seq_lens; g.free_pages = free_pages; g.free_count = free_count; g.table = p->table;
  g.seq_lens_out = seq_lens_out; g.free_count_out = free_count_out; g.table_stride = p->table_stride; g.batch = p->batch;
  g.max_pages = p->max_pages; g.n_pages = p->n_pages; g.lg = log2_of(p->page_tokens);
  const size_t lds = 2 * (size_t)p->batch * sizeof(int);
  const int64_t most = (int64_t)p->batch * p->max_pages < p->n_pages ? (int64_t)p->batch * p->max_pages : p->n_pages;
  const int64_t want = (most + PG_THREADS * 2 - 1) / (PG_THREADS * 2);
  const int wgs = (int)(want < 1 ? 1 : (want > PG_MAX_WGS ? PG_MAX_WGS : want));
  const bool in_place = seq_lens_out == seq_lens || free_count_out == free_count;
  g.what = wgs > 1 && in_place ? 1 : 3;
  hipLaunchKernelGGL(page_free_kernel, dim3(wgs), dim3(PG_THREADS), lds, static_cast<hipStream_t>(stream), g);
  if (g.what == 1) {
    if (hipGetLastError() != hipSuccess) return LIGHTKV_ERR_LAUNCH;
    g.what = 2;
    hipLaunchKernelGGL(page_free_kernel, dim3(1), dim3(PG_THREADS), lds, static_cast<hipStream_t>(stream), g);
  }
  return hipGetLastError() == hipSuccess ? LIGHTKV_OK : LIGHTKV_ERR_LAUNCH;
}

lightkv_status lightkv_page_write(const lightkv_pages *p, const int32_t *cu_new, const int32_t *slots, int64_t rows,
                                  const void *K, int64_t k_tok_stride, int64_t k_head_stride,
                                  const void *V, int64_t v_tok_stride, int64_t v_head_stride, void *stream) {
  lightkv_status st = check_page_pools(p, false);
  if (st != LIGHTKV_OK) return st;
  if (!slots || (!K && !V) || (K && !p->K) || (V && !p->V)) return LIGHTKV_ERR_NULL;
  if (rows < 0) return LIGHTKV_ERR_SHAPE;
  if (rows >= (1ll << 31) || !aligned_to(slots, 4) || !aligned_to(cu_new, 4)) return LIGHTKV_ERR_UNSUPPORTED;
  const int eb = page_elem_bytes(p);
  const void *src[2] = {K, V};
  void *dst[2] = {p->K, p->V};
  const int64_t tok[2] = {k_tok_stride, v_tok_stride}, head[2] = {k_head_stride, v_head_stride};
  const int64_t page_s[2] = {p->k_page_stride, p->v_page_stride}, tok_s[2] = {p->k_tok_stride, p->v_tok_stride}, head_s[2] = {p->k_head_stride, p->v_head_stride};
  for (int i = 0; i < 2; ++i) {
    if (!src[i]) continue;
    st = check_strided(src[i], eb, tok[i], rows, head[i], p->kv_heads);
    if (st != LIGHTKV_OK) return st;
    // rows of a pool that is written must not share elements
    const int64_t stride[3] = {page_s[i], tok_s[i], head_s[i]}, count[3] = {p->n_pages, p->page_tokens, p->kv_heads};
    if (!apart(p->head_dim, stride, count, 3)) return LIGHTKV_ERR_SHAPE;
    const uint64_t n = strided_bytes(eb, tok[i], rows, head[i], p->kv_heads, p->head_dim);
    for (int k = 0; k < 2; ++k)
      if (src[k] && overlap(src[i], n, dst[k], pool_bytes(p, page_s[k], tok_s[k], head_s[k]))) return LIGHTKV_ERR_SHAPE;
    // slots and offsets are read while pools are written
    const uint64_t bytes = pool_bytes(p, page_s[i], tok_s[i], head_s[i]);
    if (overlap(slots, (uint64_t)rows * 4, dst[i], bytes) || overlap(cu_new, ((uint64_t)p->batch + 1) * 4, dst[i], bytes)) return LIGHTKV_ERR_SHAPE;
  }
  if (K && V && pools_meet(p)) return LIGHTKV_ERR_SHAPE;   // keys and values would be written over each other
  if (rows == 0) return LIGHTKV_OK;
  WriteArgs g{};
  g.cu_new = cu_new; g.slots = slots; g.rows = rows; g.batch = p->batch; g.n_slots = p->n_pages * p->page_tokens; g.lg = log2_of(p->page_tokens);
  int n = 0;
  for (int i = 0; i < 2; ++i) {
    if (!src[i]) continue;
    g.src[n] = static_cast<const char *>(src[i]); g.dst[n] = static_cast<char *>(dst[i]);
    g.src_tok[n] = (rows > 1 ? tok[i] : 0) * eb; g.src_head[n] = (p->kv_heads > 1 ? head[i] : 0) * eb;
    g.dst_page[n] = (p->n_pages > 1 ? page_s[i] : 0) * eb; g.dst_tok[n] = tok_s[i] * eb; g.dst_head[n] = (p->kv_heads > 1 ? head_s[i] : 0) * eb;
    ++n;
  }
  g.lg_pieces = log2_of(p->head_dim * eb / 16);
  g.pieces_per_row = p->kv_heads << g.lg_pieces;
  g.rows_per_wg = g.pieces_per_row < 1024 ? 1024 / g.pieces_per_row : 1;
  const int64_t want = (rows + g.rows_per_wg - 1) / g.rows_per_wg, wgs = want < (1 << 20) ? want : (1 << 20);
  const bool stream_through = (uint64_t)rows * g.pieces_per_row * 16 * n >= PG_STREAM_BYTES;
  const auto kernel = stream_through ? page_write_kernel<true> : page_write_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)wgs, (unsigned)n), dim3(PG_THREADS), 0, static_cast<hipStream_t>(stream), g);
  return hipGetLastError() == hipSuccess ? LIGHTKV_OK : LIGHTKV_ERR_LAUNCH;
}

}  // extern "C"
