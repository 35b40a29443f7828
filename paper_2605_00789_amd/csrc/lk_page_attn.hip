// Attention of one new token per sequence over a paged K/V cache (lightkv_page_attention).
//
//   s_t = q.k_t * scale,   m = max s_t,   l = sum exp(s_t - m),   out = sum exp(s_t - m) v_t / l,   lse = m + log l
//
// One pass over K and V with the running maximum and sum of a softmax; parts of a sequence (waves, workgroups) keep (m, l, o)
// of their own and are joined as l = sum l_i exp(m_i - m), o alike.  4 flops for each element that is read: the bytes of K and
// V bound it, at any number of query heads a K/V head serves.  So the matrix instructions are there to keep the vector units
// out of the way: up to 16 query heads of a K/V head are the columns of one 16 x 16 block, and fewer cost the same.
//
// A tile is 32 tokens (16 for fp32) of one K/V head.  Lane (m = lane % 16, g = lane / 16) of the wave that works on it
//   - loads K and V as whole rows, the lanes of a row side by side (pa_run),
//   - takes K's rows from LDS, where the wave has put them, as the A operand of S^T = K Q^T: row m of half h is token
//     8 (m / 4) + 4 h + m % 4 (fp32: token m).  S^T then leaves lane (m, g) with the scores of query m against tokens 8 g + j
//     (4 g + j), j = 4 h + i: as they stand the B operand of out^T = V^T P^T,
//   - has loaded elements m * head_dim / 16 .. of V's tokens 8 g + j, all of them: V's operand wants one element of the eight
//     tokens in a lane, a transposition inside the lane, one byte permutation per register (fp32: none).  Output rows come
//     out permuted, element m * head_dim / 16 + t for row m of block t, which the store undoes.
// A product does not care how the things it sums over are numbered as long as both operands agree: that is what all of this uses.
// (K straight from memory in its operand's layout, 64 bytes of 16 rows a load: 6 x 1850 tokens of 40 heads, token-major, 48.9 us
// against 43.3.)
//
// Measured on the kernels alone: 131000 tokens of 8 heads, 537 MB, 83 us = 6.5 TB/s (read sweeps of the same size 6.7 to 6.9); 64
// ragged sequences under 64 query heads, 979 MB, 166 us = 5.9; 6 x 1850 of 40 heads, 230 MB, 40.6 = 5.7; 16 x 461 of 32 heads, 120 MB,
// 22.0 = 5.4; one sequence of 381 tokens, 6.3 MB, 6.1 us: the rate of 32 CUs.  Matrix units busy 7 % of the time at most.
#include "lk_common.h"
#include "lk_pages.h"

namespace lk {

constexpr int PA_MAX_Q = 16;     // query heads per block
constexpr float PA_LOG2E = 1.4426950408889634f, PA_LN2 = 0.6931471805599453f;

struct PageAttnArgs {
  const char *K, *V, *Q;
  char *out;
  float *lse, *stats, *part;      // records of partial results: (m, l) and unscaled sums
  int4 *cuts;                     // how many cut segments there are; (sequence, segment, first record, records) of each
  const int32_t *table, *seq_lens;
  int64_t table_stride;
  int64_t k_page, k_tok, k_head, v_page, v_tok, v_head, q_tok, q_head, o_tok, o_head;   // bytes
  int batch, kv_heads, group, q_blocks;   // query heads per K/V head, blocks of at most 16 of them
  int n_pages, lg, room;          // room: tokens a table row can hold
  float scale2;                   // softmax scale * log2(e)
};

template <typename T, int HD> struct PaGeo {
  static constexpr int EB = Elem<T>::BYTES;
  static constexpr int TILE = EB == 2 ? 32 : 16;   // tokens
  static constexpr int NH = TILE / 16;             // 16-token halves
  static constexpr int C = HD * EB / 16;           // 16-byte chunks of a row
  static constexpr int KL = C / 4;                 // ... of it in one lane's operand
  static constexpr int KI = TILE * C / 64;         // loads of K per lane and tile
  static constexpr int K_BYTES = TILE * C * 16;
  static constexpr int NK = TILE / 4;              // V rows per lane
  static constexpr int VT = HD / 16;               // elements per lane and V row, = output blocks
  static constexpr int VW = VT * EB / 4;           // ... in words
};

template <typename T, int HD> struct PaTile {
  using G = PaGeo<T, HD>;
  uint4 k[G::KI];
  uint32_t v[G::NK][G::VW];
  uint32_t live;                                   // bit t: token t of the tile counts
};

// ONCE: K and V are read by one workgroup each and are larger than the caches: loads that do not stay there leave the memory more
// of its rate.  131000 tokens x 8 heads, 537 MB: 97 -> 86 us; 64 ragged sequences, 979 MB: 195 -> 181.  Blocks of a larger
// group of query heads find each other's rows in the caches: 4 x 30000 tokens, 128 heads over one, 51.0 us past them and 35.8
// through them; 16 x 8192, 128 over 4, 93.6 and 88.3.
template <bool ONCE> __device__ __forceinline__ uint4 pa_ld16(const char *p) { return ONCE ? ld16_stream(p) : ld16(p); }
template <int W, bool ONCE> __device__ __forceinline__ void pa_load_words(uint32_t (&d)[W], const char *p) {
  if constexpr (W % 4 == 0) {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const uint4 v = pa_ld16<ONCE>(p + i * 4);
      d[i] = v.x; d[i + 1] = v.y; d[i + 2] = v.z; d[i + 3] = v.w;
    }
  } else if constexpr (W == 2) {
    const uint64_t *q = reinterpret_cast<const uint64_t *>(p);
    const uint64_t v = ONCE ? __builtin_nontemporal_load(q) : *q;
    d[0] = (uint32_t)v; d[1] = (uint32_t)(v >> 32);
  } else {
    const uint32_t *q = reinterpret_cast<const uint32_t *>(p);
    d[0] = ONCE ? __builtin_nontemporal_load(q) : *q;
  }
}

// Row of the first product's A operand <-> token of the tile, and where a token's chunk lies in LDS: chunks are swapped by the
// row number so that the 16 rows of an operand load lie in 16 different places of the 256 bytes a bank cycle covers.
template <typename T, int HD> __device__ __forceinline__ int pa_token_of(int h, int m) { return PaGeo<T, HD>::NH == 2 ? (m >> 2) * 8 + h * 4 + (m & 3) : m; }
template <typename T, int HD> __device__ __forceinline__ int pa_place(int token, int chunk) {
  constexpr int C = PaGeo<T, HD>::C, SHIFT = C >= 16 ? 0 : (C == 8 ? 1 : 2);
  const int m = PaGeo<T, HD>::NH == 2 ? (token >> 3) * 4 + (token & 3) : token;
  return (token * C + (chunk ^ ((m >> SHIFT) & (C - 1)))) * 16;
}

// One wave's share of a segment: (m, l, o) of up to 16 queries.  m belongs to query lane % 16 in all four lane groups, l holds
// the lane's own tokens until it is summed at the end.
template <typename T, int HD> struct PaState {
  using G = PaGeo<T, HD>;
  float m, l;
  f32x4 o[G::VT];
};

template <typename T, int HD>
__device__ __forceinline__ void pa_accumulate(PaState<T, HD> &st, PaTile<T, HD> &tile, const uint4 (&q)[PaGeo<T, HD>::KL], float scale2, char *lds) {
  using G = PaGeo<T, HD>;
  const int lane = threadIdx.x & 63, m = lane & 15, g = lane >> 4;
  // (the wave's own piece of LDS, and a wave's LDS operations are done in order: nothing to wait for in between)
#pragma unroll
  for (int i = 0; i < G::KI; ++i) *reinterpret_cast<uint4 *>(lds + pa_place<T, HD>((lane / G::C) * G::KI + i, lane % G::C)) = tile.k[i];
  float s[G::NH][4];
#pragma unroll
  for (int h = 0; h < G::NH; ++h) {
    f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < G::KL; ++i) {
      const uint4 k = *reinterpret_cast<const uint4 *>(lds + pa_place<T, HD>(pa_token_of<T, HD>(h, m), i * 4 + g));
      if constexpr (G::EB == 2) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[i]), c, 0, 0, 0);
      } else {
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k.x), __uint_as_float(q[i].x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k.y), __uint_as_float(q[i].y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k.z), __uint_as_float(q[i].z), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k.w), __uint_as_float(q[i].w), c, 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[h][i] = c[i] * scale2;
  }
  constexpr uint32_t ALL = G::TILE == 32 ? 0xffffffffu : 0xffffu;
  if (tile.live != ALL) {   // (the same in all lanes)
#pragma unroll
    for (int h = 0; h < G::NH; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool dead = !((tile.live >> (g * G::NK + h * 4 + i)) & 1u);
        if (dead) s[h][i] = -INFINITY;
        // a weight of zero does not silence a NaN or an infinity: the row itself becomes zero
#pragma unroll
        for (int w = 0; w < G::VW; ++w) tile.v[h * 4 + i][w] = dead ? 0u : tile.v[h * 4 + i][w];
      }
  }
  float mx = s[0][0];
#pragma unroll
  for (int h = 0; h < G::NH; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[h][i]);
  // the maximum moves about log(tiles) times: only then do lanes compare and sums get rescaled
  if (__ballot(mx > st.m)) {
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m = fmaxf(st.m, mx);
    const float a = m == st.m ? 1.f : __builtin_amdgcn_exp2f(st.m - m);
    st.m = m;
    st.l *= a;
#pragma unroll
    for (int t = 0; t < G::VT; ++t) st.o[t] *= a;
  }
  const float ref = st.m == -INFINITY ? 0.f : st.m;
  float p[G::NH][4];
#pragma unroll
  for (int h = 0; h < G::NH; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      p[h][i] = __builtin_amdgcn_exp2f(s[h][i] - ref);
      st.l += p[h][i];
    }
  if constexpr (G::EB == 2) {
    // weights as hi + lo, two bf16 numbers: what is cut off lies 2^-15 below the weight, so the product is as good as an
    // fp32 one; the second matrix instruction is free beside the loads (one bf16 number per weight: 2^-8)
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a = __float_as_uint(p[j >> 1][(j & 1) * 2]), b = __float_as_uint(p[j >> 1][(j & 1) * 2 + 1]);
      hi[j] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      // (never zero where the weight is not: a weight that one bf16 number holds must not meet an infinity with a zero.  At least
      // the smallest bf16 number, 2^-133, then, which the matrix instruction keeps; at most the weight)
      const float ra = __builtin_amdgcn_fmed3f(__uint_as_float(a) - __uint_as_float(a & 0xffff0000u), 0x1p-133f, __uint_as_float(a));
      const float rb = __builtin_amdgcn_fmed3f(__uint_as_float(b) - __uint_as_float(b & 0xffff0000u), 0x1p-133f, __uint_as_float(b));
      lo[j] = __builtin_amdgcn_perm(__float_as_uint(rb), __float_as_uint(ra), 0x07060302u);
    }
    const bf16x8 ph = __builtin_bit_cast(bf16x8, uint4{hi[0], hi[1], hi[2], hi[3]}), pl = __builtin_bit_cast(bf16x8, uint4{lo[0], lo[1], lo[2], lo[3]});
#pragma unroll
    for (int t = 0; t < G::VT; ++t) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(tile.v[2 * j + 1][t >> 1], tile.v[2 * j][t >> 1], (t & 1) ? 0x07060302u : 0x05040100u);
      const bf16x8 vt = __builtin_bit_cast(bf16x8, uint4{w[0], w[1], w[2], w[3]});
      st.o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, ph, st.o[t], 0, 0, 0);
      st.o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, pl, st.o[t], 0, 0, 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < G::VT; ++t)
        st.o[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(tile.v[i][t]), p[0][i], st.o[t], 0, 0, 0);
  }
}

// Tiles t0 + wave, t0 + wave + WAVES, .. < t1 of sequence b, K/V head h, query heads h0 .. h0 + gq - 1.  While a tile is
// worked on the next one of the wave is on its way, and the page numbers of the one behind that.
template <typename T, int HD, int WAVES, bool ONCE>
__device__ __forceinline__ void pa_run(const PageAttnArgs &a, int b, int len, int h, int h0, int gq, int t0, int t1, char *lds, PaState<T, HD> &st) {
  using G = PaGeo<T, HD>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  st.m = -INFINITY;
  st.l = 0.f;
#pragma unroll
  for (int t = 0; t < G::VT; ++t) st.o[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  int t = t0 + wave;
  const int32_t *row = a.table + (int64_t)b * a.table_stride;
  const int in_page = (1 << a.lg) - 1;
  // table entry of token lane % TILE of a tile, and from it the token's page; -1: does not count
  auto key_of = [&](int tile) { return tile * G::TILE + (lane & (G::TILE - 1)); };
  auto entry_of = [&](int tile) { return key_of(tile) < a.room ? row[key_of(tile) >> a.lg] : -1; };
  auto page_of = [&](int entry, int tile) { return key_of(tile) < len && (unsigned)entry < (unsigned)a.n_pages ? entry : -1; };
  // queries and the first entries do not wait for the length
  int next = entry_of(t);
  uint4 q[G::KL];
#pragma unroll
  for (int i = 0; i < G::KL; ++i) q[i] = uint4{0u, 0u, 0u, 0u};
  if (m < gq) {
    const char *p = a.Q + (int64_t)b * a.q_tok + (int64_t)(h0 + m) * a.q_head + g * 16;
#pragma unroll
    for (int i = 0; i < G::KL; ++i) q[i] = ld16(p + i * 64);
  }
  if (t >= t1) return;
  // K: the lanes of a row side by side, KI tokens one behind the other for each; V: 16 lanes a row, NK tokens.  Either number
  // divides the smallest page, so the tokens of a lane share one.
  const int kr = lane / G::C;
  const char *kh = a.K + (int64_t)h * a.k_head + (lane % G::C) * 16, *vh = a.V + (int64_t)h * a.v_head + m * (G::VW * 4);
  // rows that do not count are read from page 0 (any row of the pool will do) and masked
  auto load = [&](PaTile<T, HD> &d, int tile, int pg) {
    d.live = (uint32_t)__ballot(pg >= 0) & (G::TILE == 32 ? 0xffffffffu : 0xffffu);
    const int key0 = tile * G::TILE, safe = pg < 0 ? 0 : pg;
    const int kp = __shfl(safe, kr * G::KI, 64), vp = __shfl(safe, g * G::NK, 64);
    const char *p = kh + (int64_t)kp * a.k_page + (int64_t)((key0 + kr * G::KI) & in_page) * a.k_tok;
#pragma unroll
    for (int i = 0; i < G::KI; ++i) d.k[i] = pa_ld16<ONCE>(p + i * a.k_tok);
    p = vh + (int64_t)vp * a.v_page + (int64_t)((key0 + g * G::NK) & in_page) * a.v_tok;
#pragma unroll
    for (int i = 0; i < G::NK; ++i) pa_load_words<G::VW, ONCE>(d.v[i], p + i * a.v_tok);
  };
  PaTile<T, HD> x, y;
  load(x, t, page_of(next, t));
  next = t + WAVES < t1 ? entry_of(t + WAVES) : -1;
  for (;;) {
    if (t + WAVES < t1) {
      load(y, t + WAVES, page_of(next, t + WAVES));
      next = t + 2 * WAVES < t1 ? entry_of(t + 2 * WAVES) : -1;
    }
    pa_accumulate<T, HD>(st, x, q, a.scale2, lds);
    t += WAVES;
    if (t >= t1) break;
    if (t + WAVES < t1) {
      load(x, t + WAVES, page_of(next, t + WAVES));
      next = t + 2 * WAVES < t1 ? entry_of(t + 2 * WAVES) : -1;
    }
    pa_accumulate<T, HD>(st, y, q, a.scale2, lds);
    t += WAVES;
    if (t >= t1) break;
  }
}

template <typename T> __device__ __forceinline__ void pa_store(char *p, float v);
template <> __device__ __forceinline__ void pa_store<float>(char *p, float v) { *reinterpret_cast<float *>(p) = v; }
template <> __device__ __forceinline__ void pa_store<bf16_t>(char *p, float v) { *reinterpret_cast<uint16_t *>(p) = (uint16_t)f32_to_bf16_rne(v); }

// Result of one query element: o / l, zero where nothing counted (l = 0; a NaN goes through).
template <typename T>
__device__ __forceinline__ void pa_finish(const PageAttnArgs &a, int b, int head, int d, float m, float l, float o) {
  pa_store<T>(a.out + (int64_t)b * a.o_tok + (int64_t)head * a.o_head + d * Elem<T>::BYTES, l == 0.f ? 0.f : o / l);
  if (d == 0 && a.lse) a.lse[(int64_t)head * a.batch + b] = l == 0.f ? -INFINITY : (m + log2f(l)) * PA_LN2;
}

// LDS of a wave: K of a tile, later its part of the result, [gq][HD + PA_PAD] sums and [gq] (m, l).
constexpr int PA_PAD = 4;   // words between the rows of two queries
template <typename T, int HD> __host__ __device__ constexpr int pa_wave_bytes(int gq) {
  return gq * (HD + PA_PAD + 2) * 4 > PaGeo<T, HD>::K_BYTES ? (gq * (HD + PA_PAD + 2) * 4 + 15) / 16 * 16 : PaGeo<T, HD>::K_BYTES;
}

// The waves' parts joined in LDS; record < 0: the result, otherwise a record of partial sums.
template <typename T, int HD, int WAVES>
__device__ __forceinline__ void pa_join(const PageAttnArgs &a, char *lds, int wave_bytes, PaState<T, HD> &st, int b, int h0, int gq, int record) {
  using G = PaGeo<T, HD>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  auto so = [&](int w, int n) { return reinterpret_cast<float *>(lds + w * wave_bytes) + n * (HD + PA_PAD); };
  auto ss = [&](int w, int n) { return reinterpret_cast<float *>(lds + w * wave_bytes) + gq * (HD + PA_PAD) + n * 2; };
  float l = st.l;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (m < gq) {
    float *to = so(wave, m);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < G::VT; ++t) to[(g * 4 + i) * G::VT + t] = st.o[t][i];
    if (g == 0) { ss(wave, m)[0] = st.m; ss(wave, m)[1] = l; }
  }
  __syncthreads();
  const int rows = a.group < PA_MAX_Q ? a.group : PA_MAX_Q;   // of a record
  for (int i = threadIdx.x; i < gq * HD; i += WAVES * 64) {
    const int n = i / HD, d = i % HD;
    float top = -INFINITY, sum = 0.f, o = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ss(w, n)[0]);
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float mw = ss(w, n)[0], f = mw == top ? 1.f : __builtin_amdgcn_exp2f(mw - ref);
      sum += f * ss(w, n)[1];
      o += f * so(w, n)[d];
    }
    if (record < 0) {
      pa_finish<T>(a, b, h0 + n, d, top, sum, o);
    } else {
      const int64_t r = (int64_t)record * rows + n;
      a.part[r * HD + d] = o;
      if (d == 0) { a.stats[r * 2] = top; a.stats[r * 2 + 1] = sum; }
    }
  }
}

__device__ __forceinline__ int pa_len(const PageAttnArgs &a, int b) {
  const int n = a.seq_lens[b];
  return n < 0 ? 0 : (n < a.room ? n : a.room);
}

// One workgroup per (sequence, block of query heads): the whole length, no second launch.
template <typename T, int HD, int WAVES, bool ONCE>
__global__ __launch_bounds__(WAVES * 64, 2) void page_attn_whole_kernel(PageAttnArgs a) {
  fetch_args<PageAttnArgs>();
  extern __shared__ __align__(16) char pa_lds[];
  const int rows = a.group < PA_MAX_Q ? a.group : PA_MAX_Q, wave_bytes = pa_wave_bytes<T, HD>(rows);
  char *own = pa_lds + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * wave_bytes;
  const int segs = a.kv_heads * a.q_blocks, b = blockIdx.x / segs, seg = blockIdx.x - b * segs;
  const int h = a.q_blocks == 1 ? seg : seg / a.q_blocks, qb = seg - h * a.q_blocks;
  const int gq = a.group - qb * PA_MAX_Q < PA_MAX_Q ? a.group - qb * PA_MAX_Q : PA_MAX_Q, h0 = h * a.group + qb * PA_MAX_Q;
  const int len = pa_len(a, b);
  PaState<T, HD> st;
  pa_run<T, HD, WAVES, ONCE>(a, b, len, h, h0, gq, 0, (len + PaGeo<T, HD>::TILE - 1) / PaGeo<T, HD>::TILE, own, st);
  pa_join<T, HD, WAVES>(a, pa_lds, wave_bytes, st, b, h0, gq, -1);
}

// Split launches.  A segment (a sequence's K/V head and block of query heads) is cut into parts of at most c tiles, a
// workgroup each, with c chosen from the lengths on the device so that there are about PA_PARTS parts in all: the cut goes by
// what there is to do and needs nothing from the host.  More parts than fit the card at once, so that some begin (a chain of
// loads: lengths, page numbers, rows) while others are in the middle of theirs.  Parts of a segment that is not whole leave
// records, in the order of their tokens, which a second launch joins.
constexpr int PA_SPLIT_WAVES = 4, PA_JOIN_THREADS = 256;
// Parts of a call.  Sequences about as long as each other (the longest at most 3/2 of their mean), or few segments: no more than
// fit the card, two workgroups of 256 registers a CU.  Otherwise twice as many, so that what is left at the end is small.
// us a call with 512 / 1024, 8 K/V heads unless named: 131000 tokens 94.3 / 97.6, 16 x 1100 tokens of 32 heads 52.1 / 56.7, 16 x 8192 of 4
// heads 55.4 / 61.9, 3 x (1 to 8000) of 32 heads 39.6 / 43.0; 64 x (1 to 8192) 193.9 / 176.2, 16 x (50 to 2000) of 32 heads
// 66.4 / 54.1, 64 x (1 to 4096) 104.4 / 93.5, 24 x (1 to 16000) 134.8 / 128.6.  Alike segments that are more than half of what fits
// are not cut, and a last round that is not full costs: 4096 tokens of 512 segments 171 us, 6.3 TB/s; of 520 204, 5.3; of 800 288, 5.8.
constexpr int PA_PARTS = 1024, PA_FEW_SEGS = 192;
// More workgroups than two a CU would fit for smaller heads; it pays for 32 elements only.  With 512 / 768: 2 x 4554 tokens of 23 heads of 32
// 18.9 / 15.9, 10 x (3624 to 7249) of 4 16.8 / 15.5, fp32 8 x 8192 of 32 96.1 / 93.7; heads of 64, 2 x 4554 18.1 / 17.9, 100000 of 8 41.5 / 42.4.
template <int HD> constexpr int PA_SLOTS = HD == 32 ? 768 : 512;
constexpr uint32_t PA_MIN_TILES = PA_SPLIT_WAVES;   // a tile for each wave; 1 x 2048 tokens with 16 / 8 / 4: 13.8 / 12.2 / 10.9 us

// Quotient of numbers that are small in all but impossible calls: a 64-bit division is 130 instructions.
__device__ __forceinline__ int64_t pa_quotient(int64_t n, int64_t d) {
  return ((n | d) >> 32) == 0 ? (int64_t)((uint32_t)n / (uint32_t)d) : n / d;
}

// What a workgroup of a split launch has to do: part `part` of `parts` of segment `seg` of sequence b.
struct PaPart { int b, len, seg, part, parts, record, cut; };

struct PaCutLds { int sums[2][PA_SPLIT_WAVES], used[PA_SPLIT_WAVES], longest[PA_SPLIT_WAVES], parts[PA_SPLIT_WAVES], records[PA_SPLIT_WAVES], cuts[PA_SPLIT_WAVES]; PaPart mine; };

// Finds part `which` of the call (false: there are fewer).  Every thread takes a run of sequences; the one that owns the part
// says so.  Parts of cut segments come first, whole segments, which are no longer than those, fill in behind them.
// all_cuts: cut segments of the call.
template <int TILE, int SLOTS>
__device__ __forceinline__ bool pa_find_part(const PageAttnArgs &a, int segs, int64_t which, PaCutLds &lds, PaPart &out, int &all_cuts) {
  constexpr int THREADS = PA_SPLIT_WAVES * 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int per = (a.batch + THREADS - 1) / THREADS, b0 = tid * per, b1 = b0 + per < a.batch ? b0 + per : a.batch;
  auto sum_of_all = [&](int v, int *scratch) {
    const int s = wave_running_sum(v);
    if (lane == 63) scratch[wave] = s;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < PA_SPLIT_WAVES; ++w) all += scratch[w];
    return all;
  };
  auto tiles_of = [&](int len) { return (uint32_t)(len + TILE - 1) / TILE; };
  // a sequence without tokens is one part, too: it writes what such a sequence gets
  auto parts_of = [&](int len, uint32_t c) { const uint32_t nt = tiles_of(len); return nt <= c ? 1 : (int)((nt + c - 1) / c); };
  if (tid == 0) lds.mine.b = -1;
  int tiles = 0, used = 0, longest = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = (int)tiles_of(pa_len(a, b));
    tiles += n;
    used += n > 0;
    longest = n > longest ? n : longest;
  }
  const int wave_tiles = wave_running_sum(tiles), wave_used = wave_running_sum(used), wave_longest = wave_running_max(longest);
  if (lane == 63) { lds.sums[0][wave] = wave_tiles; lds.used[wave] = wave_used; lds.longest[wave] = wave_longest; }
  __syncthreads();
  tiles = used = longest = 0;
#pragma unroll
  for (int w = 0; w < PA_SPLIT_WAVES; ++w) {
    tiles += lds.sums[0][w];
    used += lds.used[w];
    longest = lds.longest[w] > longest ? lds.longest[w] : longest;
  }
  const int64_t n_segs = (int64_t)used * segs, all_tiles = (int64_t)tiles * segs;
  const bool alike = (int64_t)longest * used * 2 <= (int64_t)tiles * 3;
  uint32_t c;
  if (alike) {
    // k parts of each segment fit the card at once
    const uint32_t k = n_segs < SLOTS ? SLOTS / (uint32_t)(n_segs ? n_segs : 1) : 1;
    c = ((uint32_t)longest + k - 1) / k;
    c = c < PA_MIN_TILES ? PA_MIN_TILES : c;
  } else {
    const int target = n_segs < PA_FEW_SEGS ? SLOTS : PA_PARTS;
    const int64_t want = pa_quotient(all_tiles + target - 1, target);
    c = want < PA_MIN_TILES ? PA_MIN_TILES : (uint32_t)want;
    // rounded up segment by segment they are more than that: longer ones, then
    int n = 0;
    for (int b = b0; b < b1; ++b) n += parts_of(pa_len(a, b), c);
    int64_t all = (int64_t)sum_of_all(n, lds.sums[1]) * segs;
    all = all < 2 * target ? all : 2 * target;
    if (all > target) c = (uint32_t)pa_quotient((int64_t)c * all + target - 1, target);
  }
  int parts = 0;
  int records = 0, cuts = 0;
  for (int b = b0; b < b1; ++b) {
    const int n = parts_of(pa_len(a, b), c);
    if (n > 1) { records += n; ++cuts; }
    else ++parts;
  }
  const int sum_parts = wave_running_sum(parts), sum_records = wave_running_sum(records), sum_cuts = wave_running_sum(cuts);
  if (lane == 63) { lds.parts[wave] = sum_parts; lds.records[wave] = sum_records; lds.cuts[wave] = sum_cuts; }
  __syncthreads();
  int at = sum_parts - parts, rec = sum_records - records, cut = sum_cuts - cuts, all_records = 0;
  all_cuts = 0;
#pragma unroll
  for (int w = 0; w < PA_SPLIT_WAVES; ++w) {
    if (w < wave) { at += lds.parts[w]; rec += lds.records[w]; cut += lds.cuts[w]; }
    all_cuts += lds.cuts[w];
    all_records += lds.records[w];
  }
  all_cuts *= segs;
  const bool whole = which >= (int64_t)all_records * segs;
  const int64_t place = whole ? which - (int64_t)all_records * segs : which;   // among its kind
  const int mine = whole ? at : rec, count = whole ? parts : records;
  if (place >= (int64_t)mine * segs && place < (int64_t)(mine + count) * segs) {
    for (int b = b0; b < b1; ++b) {
      const int len = pa_len(a, b), n = parts_of(len, c);
      if ((n == 1) != whole) continue;
      const int before = whole ? at : rec;
      if (place < (int64_t)(before + n) * segs) {
        const uint32_t local = (uint32_t)(place - (int64_t)before * segs), seg = n == 1 ? local : local / (uint32_t)n;
        lds.mine = PaPart{b, len, (int)seg, (int)(local - seg * n), n, (int)place - (int)(local - seg * n), cut * segs + (int)seg};
        break;
      }
      if (whole) ++at;
      else { rec += n; ++cut; }
    }
  }
  __syncthreads();
  out = lds.mine;
  return out.b >= 0;
}

template <typename T, int HD, bool ONCE>
__global__ __launch_bounds__(PA_SPLIT_WAVES * 64, 2) void page_attn_split_kernel(PageAttnArgs a) {
  fetch_args<PageAttnArgs>();
  extern __shared__ __align__(16) char pa_lds[];
  __shared__ PaCutLds cut_lds;
  const int rows = a.group < PA_MAX_Q ? a.group : PA_MAX_Q, segs = a.kv_heads * a.q_blocks, wave_bytes = pa_wave_bytes<T, HD>(rows);
  char *own = pa_lds + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * wave_bytes;
  PaPart found;
  int cuts;
  const bool any = pa_find_part<PaGeo<T, HD>::TILE, PA_SLOTS<HD>>(a, segs, blockIdx.x, cut_lds, found, cuts);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.cuts[0] = int4{cuts, 0, 0, 0};
  if (!any) return;
  // (uniform, but read from LDS)
  const int b = __builtin_amdgcn_readfirstlane(found.b), len = __builtin_amdgcn_readfirstlane(found.len), seg = __builtin_amdgcn_readfirstlane(found.seg);
  const int part = __builtin_amdgcn_readfirstlane(found.part), parts = __builtin_amdgcn_readfirstlane(found.parts), record = __builtin_amdgcn_readfirstlane(found.record);
  const int h = a.q_blocks == 1 ? seg : seg / a.q_blocks, qb = seg - h * a.q_blocks;
  const int gq = a.group - qb * PA_MAX_Q < PA_MAX_Q ? a.group - qb * PA_MAX_Q : PA_MAX_Q, h0 = h * a.group + qb * PA_MAX_Q;
  const int nt = (len + PaGeo<T, HD>::TILE - 1) / PaGeo<T, HD>::TILE;
  int t0 = 0, t1 = nt;
  if (parts > 1) {   // parts differ by a tile at most
    const int base = nt / parts, more = nt - base * parts;
    t0 = part * base + (part < more ? part : more);
    t1 = t0 + base + (part < more ? 1 : 0);
    if (part == 0 && threadIdx.x == 0) a.cuts[1 + found.cut] = int4{b, seg, record, parts};   // (the record of part 0)
  }
  PaState<T, HD> st;
  pa_run<T, HD, PA_SPLIT_WAVES, ONCE>(a, b, len, h, h0, gq, t0, t1, own, st);
  pa_join<T, HD, PA_SPLIT_WAVES>(a, pa_lds, wave_bytes, st, b, h0, gq, parts > 1 ? record + part : -1);
}

// Joins the records of a cut segment, a workgroup per query head, always in the records' order.
constexpr int PA_FEW = 4;   // records that a thread loads at once, weights and sums, in one trip to memory

template <typename T, int HD>
__global__ __launch_bounds__(PA_JOIN_THREADS) void page_attn_join_kernel(PageAttnArgs a) {
  fetch_args<PageAttnArgs>();
  extern __shared__ __align__(16) char pa_lds[];
  __shared__ float all_top, all_sum;
  const int tid = threadIdx.x, lane = tid & 63;
  const int rows = a.group < PA_MAX_Q ? a.group : PA_MAX_Q;
  const int n_cuts = a.cuts[0].x;
  const int4 cut = a.cuts[1 + blockIdx.x];
  if ((int)blockIdx.x >= n_cuts) return;
  const int b = cut.x, seg = cut.y, n_rec = cut.w;
  const int h = seg / a.q_blocks, qb = seg - h * a.q_blocks, head = h * a.group + qb * PA_MAX_Q + (int)blockIdx.y;
  if (head >= (h + 1) * a.group) return;   // a block of fewer heads
  constexpr int V = HD / 4, GROUPS = PA_JOIN_THREADS / V;   // four elements a thread, and every GROUPS-th record
  const int grp = tid / V, d = (tid - grp * V) * 4;
  auto record = [&](int r) { return (int64_t)(cut.z + r) * rows + blockIdx.y; };
  auto weight_of = [](float m, float top) { return m == top ? 1.f : __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top)); };
  auto finish = [&](float top, float sum, const float4 &o) {
    const float e[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) pa_finish<T>(a, b, head, d + k, top, sum, e[k]);
  };
  if (n_rec <= PA_FEW) {
    if (grp != 0) return;
    float2 s[PA_FEW];
    float4 v[PA_FEW];
#pragma unroll
    for (int r = 0; r < PA_FEW; ++r) {
      const int64_t k = record(r < n_rec ? r : 0);
      s[r] = *reinterpret_cast<const float2 *>(a.stats + k * 2);
      v[r] = *reinterpret_cast<const float4 *>(a.part + k * HD + d);
    }
    float top = s[0].x, sum = 0.f;
#pragma unroll
    for (int r = 1; r < PA_FEW; ++r) top = fmaxf(top, s[r].x);
    float4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < PA_FEW; ++r) {
      if (r >= n_rec) continue;
      const float f = weight_of(s[r].x, top);
      sum += f * s[r].y;
      o.x += f * v[r].x; o.y += f * v[r].y; o.z += f * v[r].z; o.w += f * v[r].w;
    }
    finish(top, sum, o);
    return;
  }
  float *weight = reinterpret_cast<float *>(pa_lds);    // [n_rec]
  if (tid < 64) {
    float top = -INFINITY, sum = 0.f;
    for (int r = lane; r < n_rec; r += 64) top = fmaxf(top, a.stats[record(r) * 2]);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    for (int r = lane; r < n_rec; r += 64) {
      const float2 s = *reinterpret_cast<const float2 *>(a.stats + record(r) * 2);
      weight[r] = weight_of(s.x, top);
      sum += weight[r] * s.y;
    }
    sum = wave_sum_butterfly(sum);
    if (lane == 0) { all_top = top; all_sum = sum; }
  }
  __syncthreads();
  float4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int r = grp; r < n_rec; r += GROUPS) {
    const float4 v = *reinterpret_cast<const float4 *>(a.part + record(r) * HD + d);
    const float f = weight[r];
    o.x += f * v.x; o.y += f * v.y; o.z += f * v.z; o.w += f * v.w;
  }
  float4 *part_sum = reinterpret_cast<float4 *>(weight + ((n_rec + 3) & ~3));   // [GROUPS][V]
  part_sum[tid] = o;
  __syncthreads();
  if (grp != 0) return;
  for (int k = 1; k < GROUPS; ++k) {
    const float4 v = part_sum[k * V + tid];
    o.x += v.x; o.y += v.y; o.z += v.z; o.w += v.w;
  }
  finish(all_top, all_sum, o);
}

// Launches of one workgroup per segment, or split ones?  The host knows a bound on the lengths, not the lengths.  us a call, whole
// / split, 32 heads of 128 with 32 or 8 K/V heads, all sequences at the bound: 8 segments of 512 tokens 7.6 / 10.3, of 1100 14.9 /
// 12.7; 32 of 512 9.7 / 12.0, of 1024 15.9 / 12.7; 128 of 512 12.0 / 14.5, of 1024 19.4 / 19.5, of 2048 32.3 / 30.8; 160 of 2048
// 33.8 / 35.2; 192 36.8 / 42.7; 256 46.5 / 51.6; 512 86.5 / 89.1.  A long sequence among short ones is where whole segments lose,
// 10 ns a token of the longest one at worst: 512 of 50 to 2000 tokens 57.7 / 54.7, 256 of 100 to 4000 60.1 / 61.0, 192 of 1 to 16000
// 181 / 129.  The higher line guards against the latter only: sequences at the bound lose nothing as whole segments behind it either (240 of
// 1600 to 2100 tokens, token-major, 42.7 / 44.8; of 4096 80.2 / 85.9; 480 of 3000 115.5 / 118.6, of 4096 156.1 / 159.4; 512 of 4096
// 168.5 / 172.4), and of 1 to 4096 tokens 240 take 56.0 / 56.5, 480 90.4 / 87.6, 512 93.0 / 96.1.
constexpr int PA_WHOLE_TOKENS = 768;
// Eight waves a segment where each has a CU of its own, four where two share one.  us, eight / four: 32 segments of 381 tokens 6.5 / 7.5,
// 240 of 1850 41.5 / 42.7, 2048 of 256 55.1 / 47.7.  (More than eight query heads: the join of eight waves would not fit the LDS.)
constexpr unsigned PA_WIDE_SEGS = 256;
constexpr unsigned PA_MANY_SEGS = 160;
constexpr int PA_WHOLE_TOKENS_MANY = 2048;

// a segment of n parts has more than n - 1 times the tiles of a whole part, and n > 1: at most twice PA_PARTS records, of at most
// PA_PARTS segments
constexpr int PA_RECORDS = 2 * PA_PARTS;

inline int pa_rows(const lightkv_pages *p) { const int g = p->heads / p->kv_heads; return g < PA_MAX_Q ? g : PA_MAX_Q; }
inline size_t pa_stat_bytes(const lightkv_pages *p) { return ((size_t)PA_RECORDS * pa_rows(p) * 2 * sizeof(float) + 255) / 256 * 256; }
inline size_t pa_part_bytes(const lightkv_pages *p) { return (size_t)PA_RECORDS * pa_rows(p) * p->head_dim * sizeof(float); }
inline size_t pa_bytes(const lightkv_pages *p) { return pa_stat_bytes(p) + pa_part_bytes(p) + (PA_PARTS + 1) * sizeof(int4); }

template <typename T, int HD>
static hipError_t pa_launch(const PageAttnArgs &a, bool whole, hipStream_t stream) {
  const int rows = a.group < PA_MAX_Q ? a.group : PA_MAX_Q;
  const size_t wave_bytes = pa_wave_bytes<T, HD>(rows);
  const unsigned segs = (unsigned)a.batch * (unsigned)(a.kv_heads * a.q_blocks);
  if (whole) {
    if (rows <= 8 && segs <= PA_WIDE_SEGS) hipLaunchKernelGGL((page_attn_whole_kernel<T, HD, 8, true>), dim3(segs), dim3(512), 8 * wave_bytes, stream, a);
    else if (a.q_blocks == 1) hipLaunchKernelGGL((page_attn_whole_kernel<T, HD, 4, true>), dim3(segs), dim3(256), 4 * wave_bytes, stream, a);
    else hipLaunchKernelGGL((page_attn_whole_kernel<T, HD, 4, false>), dim3(segs), dim3(256), 4 * wave_bytes, stream, a);
    return hipGetLastError();
  }
  // parts: as many as a table row's tokens allow, PA_PARTS and one more per segment at most
  const int64_t tile = PaGeo<T, HD>::TILE, longest = ((int64_t)a.room + tile * PA_MIN_TILES - 1) / (tile * PA_MIN_TILES);
  const int64_t all = (int64_t)segs * longest < (int64_t)PA_PARTS + segs ? (int64_t)segs * longest : (int64_t)PA_PARTS + segs;
  const auto split = a.q_blocks == 1 ? page_attn_split_kernel<T, HD, true> : page_attn_split_kernel<T, HD, false>;
  hipLaunchKernelGGL(split, dim3((unsigned)all), dim3(PA_SPLIT_WAVES * 64), PA_SPLIT_WAVES * wave_bytes, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const unsigned cuts = segs < (unsigned)PA_PARTS ? segs : (unsigned)PA_PARTS;
  // records of a segment: those of a sequence's segments are as many, so PA_PARTS / (their number) + 1 at most
  const size_t most = PA_PARTS / (size_t)(a.kv_heads * a.q_blocks) + 1;
  const size_t join = ((most + 3) / 4 * 4 + 4 * PA_JOIN_THREADS) * sizeof(float);
  hipLaunchKernelGGL((page_attn_join_kernel<T, HD>), dim3(cuts, rows), dim3(PA_JOIN_THREADS), join, stream, a);
  return hipGetLastError();
}

}  // namespace lk

using namespace lk;

namespace {
lightkv_status check_page_attention(const lightkv_pages *p) {
  const lightkv_status st = check_page_pools(p, true);
  if (st != LIGHTKV_OK) return st;
  // tiles are counted in 32 bits, workgroups and their threads too
  if ((int64_t)p->batch * (((int64_t)p->max_pages * p->page_tokens + 15) / 16) >= (1ll << 31)) return LIGHTKV_ERR_UNSUPPORTED;
  if ((int64_t)p->batch * p->heads >= (1ll << 22)) return LIGHTKV_ERR_UNSUPPORTED;
  return LIGHTKV_OK;
}
}  // namespace

extern "C" {

lightkv_status lightkv_page_attention_workspace(const lightkv_pages *p, size_t *bytes) {
  if (!bytes) return LIGHTKV_ERR_NULL;
  const lightkv_status st = check_page_attention(p);
  if (st == LIGHTKV_OK) *bytes = pa_bytes(p);
  return st;
}

lightkv_status lightkv_page_attention(const lightkv_pages *p, const int32_t *seq_lens, int32_t max_seq_tokens,
                                      const void *Q, int64_t q_tok_stride, int64_t q_head_stride, float softmax_scale,
                                      void *out, int64_t o_tok_stride, int64_t o_head_stride, float *lse,
                                      void *ws, size_t ws_bytes, void *stream) {
  lightkv_status st = check_page_attention(p);
  if (st != LIGHTKV_OK) return st;
  if (!seq_lens || !Q || !out) return LIGHTKV_ERR_NULL;
  // (NaN too; scores are taken times scale * log2(e), which has to be a number)
  if (!(softmax_scale >= 0.f && softmax_scale * PA_LOG2E <= 3.4028234e38f) || max_seq_tokens < 0) return LIGHTKV_ERR_SHAPE;
  if (!aligned_to(seq_lens, 4) || !aligned_to(lse, 4)) return LIGHTKV_ERR_UNSUPPORTED;
  const int eb = page_elem_bytes(p);
  st = check_strided(Q, eb, q_tok_stride, p->batch, q_head_stride, p->heads);
  if (st == LIGHTKV_OK) st = check_strided(out, eb, o_tok_stride, p->batch, o_head_stride, p->heads);
  if (st != LIGHTKV_OK) return st;
  // nothing that is written may lie in what is read, or in each other
  struct Range { const void *at; uint64_t bytes; };
  const Range in[] = {{Q, strided_bytes(eb, q_tok_stride, p->batch, q_head_stride, p->heads, p->head_dim)}, {seq_lens, (uint64_t)p->batch * 4},
                      {p->table, ((uint64_t)p->table_stride * (p->batch - 1) + p->max_pages) * 4},
                      {p->K, pool_bytes(p, p->k_page_stride, p->k_tok_stride, p->k_head_stride)}, {p->V, pool_bytes(p, p->v_page_stride, p->v_tok_stride, p->v_head_stride)}};
  const Range written[] = {{out, strided_bytes(eb, o_tok_stride, p->batch, o_head_stride, p->heads, p->head_dim)}, {lse, (uint64_t)p->heads * p->batch * 4}, {ws, pa_bytes(p)}};
  for (int i = 0; i < 3; ++i) {
    for (const Range &r : in)
      if (overlap(r.at, r.bytes, written[i].at, written[i].bytes)) return LIGHTKV_ERR_SHAPE;
    for (int j = 0; j < i; ++j)
      if (overlap(written[j].at, written[j].bytes, written[i].at, written[i].bytes)) return LIGHTKV_ERR_SHAPE;
  }
  // rows of the output must not share elements
  const int64_t o_stride[2] = {o_tok_stride, o_head_stride}, o_count[2] = {p->batch, p->heads};
  if (!apart(p->head_dim, o_stride, o_count, 2)) return LIGHTKV_ERR_SHAPE;
  const size_t stat = pa_stat_bytes(p);
  if (!ws || !aligned_to(ws, 256) || ws_bytes < pa_bytes(p)) return LIGHTKV_ERR_WORKSPACE;
  PageAttnArgs a{};
  a.K = static_cast<const char *>(p->K); a.V = static_cast<const char *>(p->V);
  a.Q = static_cast<const char *>(Q); a.out = static_cast<char *>(out); a.lse = lse;
  a.stats = static_cast<float *>(ws); a.part = reinterpret_cast<float *>(static_cast<char *>(ws) + stat);
  a.cuts = reinterpret_cast<int4 *>(static_cast<char *>(ws) + stat + pa_part_bytes(p));
  a.table = p->table; a.seq_lens = seq_lens; a.table_stride = p->table_stride;
  // an axis of one entry has no stride
  a.k_page = p->n_pages > 1 ? p->k_page_stride * eb : 0; a.k_tok = p->k_tok_stride * eb; a.k_head = p->kv_heads > 1 ? p->k_head_stride * eb : 0;
  a.v_page = p->n_pages > 1 ? p->v_page_stride * eb : 0; a.v_tok = p->v_tok_stride * eb; a.v_head = p->kv_heads > 1 ? p->v_head_stride * eb : 0;
  a.q_tok = p->batch > 1 ? q_tok_stride * eb : 0; a.q_head = p->heads > 1 ? q_head_stride * eb : 0;
  a.o_tok = p->batch > 1 ? o_tok_stride * eb : 0; a.o_head = p->heads > 1 ? o_head_stride * eb : 0;
  a.batch = p->batch; a.kv_heads = p->kv_heads; a.group = p->heads / p->kv_heads; a.q_blocks = (a.group + PA_MAX_Q - 1) / PA_MAX_Q;
  a.n_pages = p->n_pages; a.lg = log2_of(p->page_tokens); a.room = p->max_pages * p->page_tokens;
  a.scale2 = (softmax_scale > 0.f ? softmax_scale : 1.f / sqrtf((float)p->head_dim)) * PA_LOG2E;
  const int bound = max_seq_tokens > 0 && max_seq_tokens < a.room ? max_seq_tokens : a.room;
  const bool whole = bound <= ((unsigned)(a.batch * a.kv_heads * a.q_blocks) < PA_MANY_SEGS ? PA_WHOLE_TOKENS : PA_WHOLE_TOKENS_MANY);
  const hipStream_t s = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (p->dtype == LIGHTKV_BF16)
    e = p->head_dim == 128 ? pa_launch<bf16_t, 128>(a, whole, s) : p->head_dim == 64 ? pa_launch<bf16_t, 64>(a, whole, s) : pa_launch<bf16_t, 32>(a, whole, s);
  else
    e = p->head_dim == 128 ? pa_launch<float, 128>(a, whole, s) : p->head_dim == 64 ? pa_launch<float, 64>(a, whole, s) : pa_launch<float, 32>(a, whole, s);
  return e == hipSuccess ? LIGHTKV_OK : LIGHTKV_ERR_LAUNCH;
}

}  // extern "C"
