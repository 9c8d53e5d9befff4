// Attention over the 4-bit key/value cache (layout: kv.cuh).
//
// For a query row, with K_t = zk_t + sk_t ck_t and V_t = zv_t + sv_t cv_t per plane of 64 channels (codes c = 0 .. 15):
//   s_t = scale (sk_t (q . ck_t) + zk_t sum(q));    o = [sum_t (p_t sv_t) cv_t + sum_t p_t zv_t] / sum_t p_t,   p_t = 2^(s_t log2(e) - m)
// so the codes enter the tensor cores as they are and every scale is applied to a score, not to 64 elements.  Both products
// are warp MMAs (m16n8k16, fp16 operands, fp32 sums) with the codes as A, 16 tokens x 16 channels or their transpose, and
// 8 query rows as the columns of B: the g query heads of a kv head fill them.  A code is put into the low mantissa bits of an
// fp16 by one AND: c 2^-24, a subnormal that tensor cores multiply exactly.  The upper nibble of a byte gives 16 c 2^-24: its query
// channels are divided by 16.  The values' upper nibbles stay beside the lower ones, c + 16 c', and the sums over c, which the same lane
// holds, are taken off at the end.  Queries are bf16 times a power of two per row that
// brings them into the middle of fp16: exact.  The weights p sv are the only operand that is rounded, to fp16 (2^-11
// relative); their sums p are not.  To keep them inside fp16 whatever the scales are, m follows the maximum of s_t +
// log2(sv_t): a weight is at most 2^15, and precise to 2^-35 of the row's largest (2^-25 at 2^10).  m lags (a row is rescaled when a
// weight would exceed 2^15, to 2^10), so most tiles need no reduction over the warp.  A wide head's second plane has values, and so
// scales, of its own: its weights are p sv 2^d with a d per row, so that they too are at most 2^15 and precise to 2^-35 of that
// plane's largest.  (With one maximum for both, 64 wide requests, now 49.2 us, took 1.8 less, but of a plane 2^-24 and
// less of the other only sum p zv was left.)
//
// Sums over many tokens are made by fp32 additions that round, not in the accumulator of the MMA, which truncates: codes are
// positive, so the sum grows with every token while what is left of it after sum p zv shrinks with their number (131072 tokens
// in chains of 2048 MMAs: results 2 % off; like this 0.17 %, the rounding of the output).
//
// Scores come out as [token x row] with a lane holding two rows of two tokens; the second product wants weights as [token x
// row] with tokens along a lane's registers: one movmatrix per 8 x 8 block turns them.
#include <float.h>

#include <type_traits>

#include "kv.cuh"
#include "ptx.cuh"

namespace moin {

constexpr int kKvAttWarps = 4;
constexpr int kKvMaxWorkers = 1024;  // CTAs that share the work, at most
constexpr int kKvStages = 3;         // steps of a warp in shared memory
constexpr int kKvItemCost = 8;       // what beginning an item costs, in tiles
constexpr float kKvTop = 10.f;       // log2 of the largest weight after a rescale
constexpr float kKvMost = 15.f;      // log2 of the largest weight at all
constexpr float kKvApart = 100.f;    // d at most: planes further apart lose from the smaller one

// Who takes what: a CTA an item; warps equal shares of all items; or, of one request, each of gridDim.x CTAs its part of each item.
enum { KV_WHOLE = 0, KV_SHARES = 1, KV_CUT = 2 };
struct KvAttParams {
  KvView kv;
  const int *table, *rows, *cu_q, *kv_len;
  int n_rows, max_pages;
  int R, T, max_q, max_kv, G, n_heads;
  uint32_t inv_g;          // row / G = row inv_g >> 32
  uint32_t page_bytes;     // of all heads
  int tpp_log2;            // tiles of a page
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  long long q_stride, out_stride;
  const float2* rope;      // [rope_len, D / 2] or nullptr
  float scale_log2;
  int split;               // KV_WHOLE, KV_SHARES, KV_CUT
  float* part;             // [worker][2][row][64 P + 4]: sums of items that several workers share
  int4* desc;              // [CTA][2]: the item that it begins without ending it (head, first row, first token, CTAs behind), its rows
};

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint64_t twice_f32(float v) { return pair_f32(v, v); }
__device__ __forceinline__ float kv_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float kv_log2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A sum of p taken against one maximum, against another that is d = old - new away.  Weights p sv are near 2^10 at the most, p
// alone is up to 2^79 where a value's scale is tiny: there d may be below what 2^d can say and the sum still count.
__device__ __forceinline__ float kv_rescale_sum(float l, float d) {
  const float f = kv_exp2(0.5f * d);
  return l * f * f;
}

__device__ __forceinline__ int kv_div_g(const KvAttParams& p, int row) { return p.G == 1 ? row : (int)__umulhi((uint32_t)row, p.inv_g); }

// What a warp works on: the rows [row0, row0 + 8 NT) of request `req` and kv head `head`; row = (query token) * G + head of the group.
struct KvItem {
  int req, head, row0;
  int t0, q_len, kv_len;      // first query row of the request in q, its tokens, its cached tokens (0: nothing to see)
  const int* table;
};

__device__ __forceinline__ KvItem kv_item(const KvAttParams& p, int req, int head, int row0) {
  KvItem it;
  it.req = req; it.head = head; it.row0 = row0;
  it.t0 = min(max(p.cu_q[req], 0), p.T);
  it.q_len = min(max(p.cu_q[req + 1], it.t0), p.T) - it.t0;
  it.kv_len = p.kv_len[req];
  const int row = p.rows ? p.rows[req] : req;
  if (it.kv_len < 0 || it.kv_len > p.max_kv || it.q_len > p.max_q || row < 0 || row >= p.n_rows) it.kv_len = 0;
  it.q_len = min(it.q_len, p.max_q);   // (bounds that do not hold: nothing behind them is touched)
  it.table = p.table + (size_t)(it.kv_len ? row : 0) * p.max_pages;
  return it;
}

template <int P, int NT>
struct KvState {            // a warp's share of an item: 8 NT rows, 64 P channels; pairs are rows 2 t, 2 t + 1 of an n-tile
  uint64_t o[NT][P][4][2];  // [channel block of 16][g, g + 8]
  uint64_t m[NT], l[NT], z[P][NT];   // m: negated
  uint64_t d[NT];           // (P = 2) log2 of what the second plane's weights are multiplied with
  uint32_t fresh;           // bit 2 n + c: the row has seen no key yet (its m is 0 and means nothing)
};

// Query rows as B fragments: b[n][plane][k-step][half], and per row (2 t, 2 t + 1 of an n-tile) the factor and the sum.
template <int P, int NT>
struct KvQuery {
  uint32_t b[NT][P][4][2];
  uint64_t fac[NT], sum[P][NT];
  int last[NT][2];          // last key the row sees
  int all;                  // keys below this are seen by every row
  bool large;               // one of the warp's queries is
};
// A score is acc (sums of codes 2^-24 by queries near 2^9) times fac ks, and fac has 2^24 and the row's power in it: beyond 2^115 it
// left fp32, and times signed sums gave NaN.  A warp with a query of 2^kKvLarge or more takes 2^24 into acc instead and holds
// scores, factors and sums 2^-16 smaller until the score is complete: powers of two, so other rows' bits stay.  (Steps of their own:
// the others pay nothing.)
// These steps also take over where a row's maximum passes kKvCoarse: fp32 has no room for log2(sv) beside it then, so m is the
// largest score alone, and the first plane's weights are p sv 2^e, as the second plane's are p sv 2^d.  And where a row's scores rise
// by more than kKvGone: what it has is nothing beside 2^kKvGone, and the new scores, taken less the old maximum, may have lost
// theirs to its size, so the row begins anew with them.
constexpr int kKvLarge = 16;
constexpr float kKvCoarse = 0x1p20f, kKvGone = 512.f;

template <int P, int NT>
__device__ __forceinline__ void kv_load_query(const KvAttParams& p, const KvItem& it, int lane, KvQuery<P, NT>& q) {
  const int g = lane >> 2, t = lane & 3;
  const int n_rows = it.q_len * p.G, past = it.kv_len - it.q_len;
  q.large = false;
  q.all = it.kv_len;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = it.row0 + 8 * n + g;
    const int qi = kv_div_g(p, row);
    const bool live = row < n_rows && past + qi >= 0;
    float x[P][16];
#pragma unroll
    for (int pl = 0; pl < P; ++pl)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[pl][i] = 0.f;
    if (live) {
      const __nv_bfloat16* src = p.q + (long long)(it.t0 + qi) * p.q_stride + (it.head * p.G + row - qi * p.G) * 64 * P;
#pragma unroll
      for (int pl = 0; pl < P; ++pl)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(src + 64 * pl + 16 * (i >> 2) + 8 * ((i >> 1) & 1) + 2 * t));
          x[pl][i] = bf16_lo(w);
          x[pl][i + 1] = bf16_hi(w);
        }
      if (p.rope != nullptr) {
        const float2* cs = p.rope + (size_t)(past + qi) * (32 * P);
        constexpr int half = 8 * P;   // pairs of this lane: x[i], x[i + half] over the planes laid end to end
#pragma unroll
        for (int i = 0; i < half; ++i) {
          const float2 c = __ldg(cs + 16 * (i >> 2) + 8 * ((i >> 1) & 1) + 2 * t + (i & 1));
          float& a = x[0][i];
          float& b = P == 1 ? x[0][(i + 8) & 15] : x[P - 1][i];
          const float lo = round_bf16(kv_rot_lo(a, b, c)), hi = round_bf16(kv_rot_hi(a, b, c));
          a = lo;
          b = hi;
        }
      }
    }
    float top = 0.f;
#pragma unroll
    for (int pl = 0; pl < P; ++pl)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[pl][i]));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // 2^(9 - exponent of the largest element); a row of zeros, subnormals or infinities stays as it is
    const int e = (int)(__float_as_uint(top) >> 23) - 127;
    const bool scaled = e > -118 && e < 128;
    const float f = scaled ? __uint_as_float((uint32_t)(9 - e + 127) << 23) : 1.f;
    const float inv = scaled ? __uint_as_float((uint32_t)(e - 9 + 127) << 23) : 1.f;
    // to the lanes that hold these rows' scores: rows 2 t, 2 t + 1 of the n-tile
    q.fac[n] = pair_f32(__shfl_sync(0xffffffffu, inv, 8 * t), __shfl_sync(0xffffffffu, inv, 8 * t + 4));
    q.large = q.large || (scaled && e >= kKvLarge);
#pragma unroll
    for (int pl = 0; pl < P; ++pl) {
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float y[4] = {x[pl][4 * j] * f, x[pl][4 * j + 1] * f, x[pl][4 * j + 2] * f, x[pl][4 * j + 3] * f};
        sum += (y[0] + y[1]) + (y[2] + y[3]);
        q.b[n][pl][j][0] = pack_f16(y[0], y[1]);
        q.b[n][pl][j][1] = pack_f16(y[2] * 0.0625f, y[3] * 0.0625f);
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      q.sum[pl][n] = pair_f32(__shfl_sync(0xffffffffu, sum, 8 * t), __shfl_sync(0xffffffffu, sum, 8 * t + 4));
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = it.row0 + 8 * n + 2 * t + c;
      // rows that are not there compute something that is not stored, and mask nothing
      q.last[n][c] = r < n_rows ? past + kv_div_g(p, r) : it.kv_len - 1;
      q.all = min(q.all, q.last[n][c] + 1);
    }
  }
  q.all = min(q.all, __shfl_xor_sync(0xffffffffu, q.all, 1));
  q.all = min(q.all, __shfl_xor_sync(0xffffffffu, q.all, 2));
  q.large = __any_sync(0xffffffffu, q.large);
  const uint64_t up = twice_f32(p.scale_log2 * (q.large ? 0x1p-16f : 0x1p24f)), less = twice_f32(q.large ? 0x1p-16f : 1.f);
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int pl = 0; pl < P; ++pl) q.sum[pl][n] = mul2(mul2(q.sum[pl][n], mul2(q.fac[n], less)), twice_f32(p.scale_log2));
    q.fac[n] = mul2(q.fac[n], up);
  }
}

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// U tiles of 16 tokens from shared memory, the first at key0; bit u of `there`: tile u is part of the warp's work.  `whole`: every
// row sees every token.  `large`: of a warp with large queries or scores; without it false is returned, and nothing is done, where it
// has to be made with it, and with it where it has to be made again.
template <bool whole, bool large, int P, int NT, int U>
__device__ __forceinline__ bool kv_step(const uint8_t* tiles, uint32_t there, int key0, int kv_len, const KvQuery<P, NT>& q, int lane, KvState<P, NT>& st,
                                        uint64_t (&e)[NT]) {
  constexpr uint32_t kLo = 0x000F000Fu, kHi = 0x00F000F0u;
  const int g = lane >> 2;
  uint64_t s[U][NT][2];    // [token g, g + 8]: scores in powers of two, less the row's m
  uint32_t pv[U][P][2];
  float lg[U][P][2];
#pragma unroll
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int pl = 0; pl < P; ++pl) {
      const uint8_t* at = tiles + (u * P + pl) * kKvTileBytes;
      const uint4 k4 = *reinterpret_cast<const uint4*>(at + 16 * lane);
      const uint4 pr = *reinterpret_cast<const uint4*>(at + kKvPairs + 16 * g);
      uint32_t pk[2] = {pr.x, pr.y};
      pv[u][pl][0] = pr.z;
      pv[u][pl][1] = pr.w;
      if (!whole) {   // what lies behind the last token, or in a tile that was not fetched, may be anything
#pragma unroll
        for (int h = 0; h < 2; ++h)
          if (!(there >> u & 1u) || key0 + u * kKvTile + g + 8 * h >= kv_len) pk[h] = pv[u][pl][h] = 0;
      }
      const uint32_t kw[4] = {k4.x, k4.y, k4.z, k4.w};
      float acc[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w = kw[j], w8 = w >> 8;
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_f16_16816(acc[n], w & kLo, w8 & kLo, w & kHi, w8 & kHi, q.b[n][pl][j][0], q.b[n][pl][j][1]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint64_t ks = twice_f32(kv_scale(pk[h])), kz = twice_f32(kv_zero(pk[h]));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          uint64_t codes = pair_f32(acc[n][2 * h], acc[n][2 * h + 1]), before = pl == 0 ? st.m[n] : s[u][n][h];
          if (large) {
            codes = mul2(codes, twice_f32(0x1p24f));
            if (pl == 0) before = mul2(before, twice_f32(0x1p-16f));
          }
          s[u][n][h] = fma2(codes, mul2(q.fac[n], ks), fma2(q.sum[pl][n], kz, before));
          if (large && pl == P - 1) s[u][n][h] = mul2(s[u][n][h], twice_f32(0x1p16f));
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int pl = 0; pl < P; ++pl) lg[u][pl][h] = fmaxf(kv_log2(kv_scale(pv[u][pl][h])), -64.f);
    if (!whole) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = key0 + u * kKvTile + g + 8 * h;
          float a, b;
          unpair_f32(s[u][n][h], a, b);
          if (!(there >> u & 1u) || key > q.last[n][0]) a = -INFINITY;
          if (!(there >> u & 1u) || key > q.last[n][1]) b = -INFINITY;
          s[u][n][h] = pair_f32(a, b);
        }
    }
  }
  float top[NT][P][2];     // log2 of the rows' largest weights here
  bool grow = st.fresh != 0;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int pl = 0; pl < P; ++pl) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float a0, b0, a1, b1;
        unpair_f32(s[u][n][0], a0, b0);
        unpair_f32(s[u][n][1], a1, b1);
        a0 += lg[u][pl][0]; b0 += lg[u][pl][0]; a1 += lg[u][pl][1]; b1 += lg[u][pl][1];
        top[n][pl][0] = u == 0 ? fmaxf(a0, a1) : fmax3(top[n][pl][0], a0, a1);
        top[n][pl][1] = u == 0 ? fmaxf(b0, b1) : fmax3(top[n][pl][1], b0, b1);
      }
      if (pl == 1 || large) {
        float d0, d1;
        unpair_f32(pl == 1 ? st.d[n] : e[n], d0, d1);
        top[n][pl][0] += d0;
        top[n][pl][1] += d1;
      }
      grow = grow || fmaxf(top[n][pl][0], top[n][pl][1]) > kKvMost;
    }
  }
  if (__any_sync(0xffffffffu, grow)) {
    if (!large) {
      bool coarse = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float m[2];
        unpair_f32(st.m[n], m[0], m[1]);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float t = top[n][0][c];
          coarse = coarse || (t > -INFINITY && fabsf(t - m[c]) > kKvCoarse) || (t > kKvGone && !(st.fresh >> (2 * n + c) & 1u));
        }
      }
      if (__any_sync(0xffffffffu, coarse)) return false;
    } else {
      bool anew = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float most[2] = {-INFINITY, -INFINITY}, m[2], d[2], was[2], keep[2];
        unpair_f32(st.m[n], m[0], m[1]);
        unpair_f32(e[n], was[0], was[1]);
        if (P == 2) unpair_f32(st.d[n], d[0], d[1]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float x, y;
            unpair_f32(s[u][n][h], x, y);
            most[0] = fmaxf(most[0], x);
            most[1] = fmaxf(most[1], y);
          }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) most[c] = fmaxf(most[c], __shfl_xor_sync(0xffffffffu, most[c], o));
          const uint32_t bit = 1u << (2 * n + c);
          const bool gone = most[c] > kKvGone && !(st.fresh & bit);
          anew = anew || gone;
          if (gone) {
            st.fresh |= bit;
            m[c] = d[c] = was[c] = 0.f;
          }
          keep[c] = gone ? 0.f : 1.f;   // (times the sums: a NaN stays)
        }
        const uint64_t f = pair_f32(keep[0], keep[1]);
        st.m[n] = pair_f32(m[0], m[1]);
        e[n] = pair_f32(was[0], was[1]);
        if (P == 2) st.d[n] = pair_f32(d[0], d[1]);
        st.l[n] = mul2(st.l[n], f);
#pragma unroll
        for (int pl = 0; pl < P; ++pl) {
          st.z[pl][n] = mul2(st.z[pl][n], f);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            st.o[n][pl][j][0] = mul2(st.o[n][pl][j][0], f);
            st.o[n][pl][j][1] = mul2(st.o[n][pl][j][1], f);
          }
        }
      }
      if (__any_sync(0xffffffffu, anew)) return false;
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float up[P][2], corr[P][2], zc[2];   // by so much smaller are a plane's weights to become, in log2; the factor of its sums, of sums of p zv
      float l[2], d[2];
      unpair_f32(st.l[n], l[0], l[1]);
      if (P == 2) unpair_f32(st.d[n], d[0], d[1]);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint32_t bit = 1u << (2 * n + c);
        const bool fresh = st.fresh & bit;      // (its sums are 0, or NaN for good)
        bool seen = false;
#pragma unroll
        for (int pl = 0; pl < P; ++pl) {
          float mx = top[n][pl][c];
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          const bool more = mx > (fresh ? -INFINITY : kKvMost);
          up[pl][c] = more ? mx - kKvTop : 0.f;
          seen = seen || more;
        }
        if (P == 2) {   // p becomes smaller by up[0], what it is multiplied with for the second plane takes the rest
          const float apart = d[c] + up[0][c] - up[P - 1][c];
          if (apart > kKvApart) up[P - 1][c] += apart - kKvApart;
          if (apart < -kKvApart) up[0][c] += -kKvApart - apart;
          d[c] = fminf(fmaxf(apart, -kKvApart), kKvApart);
        }
#pragma unroll
        for (int pl = 0; pl < P; ++pl) corr[pl][c] = fresh ? 1.f : kv_exp2(-up[pl][c]);
        if (large) {
          float m[2], was[2][2];
          unpair_f32(st.m[n], m[0], m[1]);
          unpair_f32(e[n], was[0][0], was[0][1]);
          if (P == 2) unpair_f32(st.d[n], was[1][0], was[1][1]);
          float most = -INFINITY, t[P];   // the row's largest score so far, largest weights here against it
          auto score = [&](int u, int h) {
            float x[2];
            unpair_f32(s[u][n][h], x[0], x[1]);
            return x[c];
          };
#pragma unroll
          for (int u = 0; u < U; ++u) most = fmax3(most, score(u, 0), score(u, 1));
#pragma unroll
          for (int o = 4; o < 32; o <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
          if (!fresh) most = fmaxf(most, 0.f);
#pragma unroll
          for (int pl = 0; pl < P; ++pl) {
            t[pl] = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) t[pl] = fmax3(t[pl], score(u, 0) - most + lg[u][pl][0], score(u, 1) - most + lg[u][pl][1]);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) t[pl] = fmaxf(t[pl], __shfl_xor_sync(0xffffffffu, t[pl], o));
          }
          const bool coarse = fabsf(most - m[c]) > kKvCoarse;
          if (seen && (coarse || was[0][c] != 0.f)) {
            up[0][c] = coarse ? most : most + (t[0] - kKvTop);
            float now[P];
#pragma unroll
            for (int pl = 0; pl < P; ++pl) {
              now[pl] = fminf(fmaxf((coarse ? kKvTop : t[0]) - t[pl], -kKvApart), kKvApart);
              if (!fresh) corr[pl][c] = kv_exp2(now[pl] - was[pl][c] - up[0][c]);
            }
            e[n] = c == 0 ? pair_f32(now[0], was[0][1]) : pair_f32(was[0][0], now[0]);
            if (P == 2) d[c] = now[P - 1];
          }
        }
        zc[c] = !large ? corr[0][c] : fresh ? 1.f : kv_exp2(-up[0][c]);
        if (!fresh) l[c] = kv_rescale_sum(l[c], -up[0][c]);
        if (seen) st.fresh &= ~bit;
      }
      const uint64_t less = pair_f32(-up[0][0], -up[0][1]), f = pair_f32(zc[0], zc[1]);
      st.m[n] = add2(st.m[n], less);
      st.l[n] = pair_f32(l[0], l[1]);
      if (P == 2) st.d[n] = pair_f32(d[0], d[1]);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        s[u][n][0] = add2(s[u][n][0], less);
        s[u][n][1] = add2(s[u][n][1], less);
      }
#pragma unroll
      for (int pl = 0; pl < P; ++pl) {
        st.z[pl][n] = mul2(st.z[pl][n], f);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint64_t fo = pair_f32(corr[pl][0], corr[pl][1]);
          st.o[n][pl][j][0] = mul2(st.o[n][pl][j][0], fo);
          st.o[n][pl][j][1] = mul2(st.o[n][pl][j][1], fo);
        }
      }
    }
  }
  uint64_t apart[P][NT];
#pragma unroll
  for (int pl = large ? 0 : 1; pl < P; ++pl)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float x, y;
      unpair_f32(pl == 1 ? st.d[n] : e[n], x, y);
      apart[pl][n] = pair_f32(kv_exp2(x), kv_exp2(y));
    }
  uint32_t b[U][NT][P][2];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint64_t pr[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float x, y;
        unpair_f32(s[u][n][h], x, y);
        pr[n] = pair_f32(kv_exp2(x), kv_exp2(y));
        st.l[n] = add2(st.l[n], pr[n]);
      }
#pragma unroll
      for (int pl = 0; pl < P; ++pl) {
        const uint64_t sv = twice_f32(kv_scale(pv[u][pl][h])), zv = twice_f32(kv_zero(pv[u][pl][h]));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float x, y;
          const uint64_t w = mul2(pl == 1 || large ? mul2(pr[n], apart[pl][n]) : pr[n], sv);
          if (whole) {
            st.z[pl][n] = fma2(pr[n], zv, st.z[pl][n]);
            unpair_f32(w, x, y);
          } else {   // a value that a row must not see may be NaN
            const int key = key0 + u * kKvTile + g + 8 * h;
            const bool out0 = !(there >> u & 1u) || key > q.last[n][0], out1 = !(there >> u & 1u) || key > q.last[n][1];
            float zx, zy;
            unpair_f32(mul2(pr[n], zv), zx, zy);
            unpair_f32(w, x, y);
            x = out0 ? 0.f : x;
            y = out1 ? 0.f : y;
            st.z[pl][n] = add2(st.z[pl][n], pair_f32(out0 ? 0.f : zx, out1 ? 0.f : zy));
          }
          b[u][n][pl][h] = movmatrix_trans(pack_f16(x, y));
        }
      }
    }
#pragma unroll
  for (int pl = 0; pl < P; ++pl) {
    uint4 v4[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v4[u] = *reinterpret_cast<const uint4*>(tiles + (u * P + pl) * kKvTileBytes + 512 + 16 * lane);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float d[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) d[n][0] = d[n][1] = d[n][2] = d[n][3] = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t w = j == 0 ? v4[u].x : j == 1 ? v4[u].y : j == 2 ? v4[u].z : v4[u].w;
        const uint32_t even = w & 0x00FF00FFu, odd = __byte_perm(w, 0u, 0x4341);
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_f16_16816(d[n], w & kLo, even, odd & kLo, odd, b[u][n][pl][0], b[u][n][pl][1]);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        st.o[n][pl][j][0] = add2(st.o[n][pl][j][0], pair_f32(d[n][0], d[n][1]));
        st.o[n][pl][j][1] = add2(st.o[n][pl][j][1], pair_f32(d[n][2], d[n][3]));
      }
    }
  }
  return true;
}

// What a request counts for an item: its tiles and the cost of beginning.  Items without tiles are there too: their rows are written.
__device__ __forceinline__ int kv_count(int kv_len, int max_kv) {
  return kKvItemCost + (kv_len < 1 || kv_len > max_kv ? 1 : (kv_len + kKvTile - 1) / kKvTile);
}
__device__ __forceinline__ long long kv_cost(const KvAttParams& p, int req, int rows) {
  const int t0 = min(max(p.cu_q[req], 0), p.T), t1 = min(max(p.cu_q[req + 1], t0), p.T);
  const int blocks = (int)(((long long)min(t1 - t0, p.max_q) * p.G + rows - 1) / rows);
  return (long long)blocks * p.kv.H * kv_count(p.kv_len[req], p.max_kv);
}

// All items stand in one line (request, row block, head), each as long as it counts, and every warp takes an equal run of it.
// Every CTA finds its warps' places: each thread adds up a run of requests, a scan over the CTA gives the total, and the
// thread whose run holds a place walks it.
struct KvShare { long long at, end, base; int req; };   // base: what the requests before `req` count
__device__ __forceinline__ long long kv_div(long long a, long long b) {   // both positive; 32 bits where they do
  return ((a | b) >> 32) ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}
template <int NT, int U>
__device__ __forceinline__ long long kv_share(const KvAttParams& p, long long* s_sum, KvShare* s_share) {
  constexpr int kThreads = 32 * kKvAttWarps;
  const int tid = threadIdx.x, lane = tid & 31, per = (p.R + kThreads - 1) / kThreads;
  const int r0 = min(tid * per, p.R), r1 = min(r0 + per, p.R);
  long long mine = 0;
  for (int r = r0; r < r1; ++r) mine += kv_cost(p, r, 8 * NT);
  long long inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long a = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += a;
  }
  if (lane == 31) s_sum[tid >> 5] = inc;
  if (tid < kKvAttWarps) s_share[tid] = {0, 0, 0, 0};
  __syncthreads();
  long long total = 0, before = inc - mine;
#pragma unroll
  for (int w = 0; w < kKvAttWarps; ++w) {
    if (w < (tid >> 5)) before += s_sum[w];
    total += s_sum[w];
  }
  const long long warps = (long long)gridDim.x * kKvAttWarps;
  const long long run = max(kv_div(total + warps - 1, warps), (long long)(kKvItemCost + 2 * U));   // (not less than is worth beginning)
  const long long stop = before + mine;
  int r = r0;
  for (int i = 0; i < kKvAttWarps; ++i) {
    const long long at = ((long long)blockIdx.x * kKvAttWarps + i) * run;
    if (at < before || at >= stop) continue;
    for (;;) {
      const long long c = kv_cost(p, r, 8 * NT);
      if (at < before + c) break;
      before += c;
      ++r;
    }
    s_share[i] = {at, min(at + run, total), before, r};
  }
  __syncthreads();
  return run;
}

// Sums of some rows taken against different maxima, four channels of one row: joined one by one, always in the order of the tokens.
struct KvSum {
  float m, l;
  float4 v;
  __device__ __forceinline__ void add(float m2, float l2, const float4& v2) {
    const float top = fmaxf(m, m2), f1 = kv_exp2(m - top), f2 = kv_exp2(m2 - top);
    l = kv_rescale_sum(l, m - top) + kv_rescale_sum(l2, m2 - top);
    v.x = v.x * f1 + v2.x * f2; v.y = v.y * f1 + v2.y * f2; v.z = v.z * f1 + v2.z * f2; v.w = v.w * f1 + v2.w * f2;
    m = top;
  }
  __device__ __forceinline__ uint2 result() const {
    const float inv = l == 0.f ? 0.f : 1.f / l;   // nothing to see: zeros
    return make_uint2(pack_bf16(v.x * inv, v.y * inv), pack_bf16(v.z * inv, v.w * inv));
  }
};
__device__ __forceinline__ __nv_bfloat16* kv_out(const KvAttParams& p, int t0, int head, int r, int ch, int channels) {
  const int qi = kv_div_g(p, r);
  return p.out + (long long)(t0 + qi) * p.out_stride + (head * p.G + r - qi * p.G) * channels + ch;
}

// A piece of an item as its warp leaves it: rows of kPitch floats, 64 P sums and the row's maximum and sum of weights behind them.
// In slot 0 the piece that begins inside its item (the first of a warp, or of a CTA), in slot 1 the one that begins an item without
// ending it (the last).
struct KvPiece { int head, row0, t0, n_rows, left; };   // t0, n_rows of its request; what its item counts behind it; -1: no piece

// A warp's ring, in which its last piece lies too.
template <int P, int NT, int U>
__host__ __device__ constexpr int kv_ring_bytes() {
  return kKvStages * U * P * kKvTileBytes > 8 * NT * (64 * P + 4) * 4 ? kKvStages * U * P * kKvTileBytes : 8 * NT * (64 * P + 4) * 4;
}

// A warp takes pieces of items, tile by tile through a ring of kKvStages steps of U tiles in shared memory, filled by its own
// asynchronous copies of 16 bytes a lane.  Whole items are written at once; pieces of items that the CTA's
// warps share are joined in shared memory, those that several CTAs share by kv_join_kernel.
template <int P, int NT, int U>
__global__ void __launch_bounds__(32 * kKvAttWarps, P * NT == 1 ? 4 : P * NT == 2 ? 3 : 2)
kv_attention_kernel(const KvAttParams p) {
  constexpr int kRows = 8 * NT, kCh = 64 * P, kPitch = kCh + 4, kStep = U * P * kKvTileBytes;
  constexpr int kPiece = kRows * kPitch * 4, kRing = kv_ring_bytes<P, NT, U>();
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long s_sum[kKvAttWarps];
  __shared__ KvShare s_share[kKvAttWarps];
  __shared__ KvPiece s_piece[kKvAttWarps][2];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  uint8_t* ring = smem + warp * (kRing + kPiece);
  const uint32_t ring_addr = smem_u32(ring);
  if (threadIdx.x < 2 * kKvAttWarps) s_piece[threadIdx.x >> 1][threadIdx.x & 1].left = -1;
  pdl_begin();
  __syncthreads();
  const int tpp = 1 << p.tpp_log2;
  KvShare share;
  long long run = 1;
  if (p.split == KV_SHARES) {
    run = kv_share<NT, U>(p, s_sum, s_share);
    share = s_share[warp];
  } else {   // the warp's part of the item
    const int req = p.split == KV_CUT ? 0 : blockIdx.z, warps = p.split == KV_CUT ? kKvAttWarps * gridDim.x : kKvAttWarps;
    const long long n = kv_count(p.kv_len[req], p.max_kv) - kKvItemCost;
    const int w = (p.split == KV_CUT ? blockIdx.x * kKvAttWarps : 0) + warp;
    share = {n * w / warps, n * (w + 1) / warps, 0, req};
  }
  while (share.at < share.end) {
    // ---- the piece: tiles tile0 .. tile1 of an item of n_tiles
    KvItem it;
    int tile0, tile1, left;
    if (p.split == KV_SHARES) {
      long long c = kv_cost(p, share.req, kRows);
      while (share.at >= share.base + c) {
        share.base += c;
        c = kv_cost(p, ++share.req, kRows);
      }
      const int count = kv_count(p.kv_len[share.req], p.max_kv);
      const long long in = share.at - share.base;
      const int item = (int)kv_div(in, count), from = (int)(in - (long long)item * count), to = (int)min((long long)count, from + (share.end - share.at));
      share.at += to - from;
      if (to <= kKvItemCost) continue;   // only the beginning: left to the next warp
      left = count - to;
      tile0 = max(0, from - kKvItemCost);
      tile1 = to - kKvItemCost;
      const int block = item / p.kv.H;
      it = kv_item(p, share.req, item - block * p.kv.H, block * kRows);
    } else {
      const int block = p.split == KV_CUT ? blockIdx.z : blockIdx.x;
      it = kv_item(p, share.req, blockIdx.y, block * kRows);
      tile0 = (int)share.at;
      tile1 = (int)share.end;
      left = kv_count(p.kv_len[share.req], p.max_kv) - kKvItemCost - tile1;
      share.at = share.end;
    }
    const int n_rows = it.q_len * p.G;
    if (it.row0 >= n_rows) break;   // (an item of its own CTA that is not there)
    // keys that the last row of the block sees
    const int see = max(0, min(it.kv_len, it.kv_len - it.q_len + kv_div_g(p, min(it.row0 + kRows - 1, n_rows - 1)) + 1));
    const int stop = min(tile1, (see + kKvTile - 1) / kKvTile);
    const int n_steps = stop <= tile0 ? 0 : (stop - tile0 + U - 1) / U;
    // pages of 32 tiles at a time, a lane each, and of the 32 behind them
    auto pages_of = [&](int w) -> int {
      const int tile = 32 * w + lane;
      return tile < stop ? __ldg(it.table + (tile >> p.tpp_log2)) : -1;
    };
    int window = tile0 >> 5;
    int pages = 0, pages_next = 0;
    if (n_steps > 0) {
      pages = pages_of(window);
      pages_next = pages_of(window + 1);
    }
    const uint8_t* heads = p.kv.pages + (size_t)it.head * tpp * (P * kKvTileBytes) + 16 * lane;
    uint32_t have = 0;             // tiles of the steps in flight, four bits each, the next step's lowest
    uint32_t fill_at = ring_addr + 16 * lane, use_at = 0;
    auto fill = [&](int i) {       // step i of the piece into the ring
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int tile = tile0 + U * i + u;
        if ((tile >> 5) != window) {
          ++window;
          pages = pages_next;
          pages_next = pages_of(window + 1);
        }
        const int page = __shfl_sync(0xffffffffu, pages, tile & 31);
        if (page >= 0 && page < p.kv.n_pages) {   // (the same for the whole warp; -1 behind the piece)
          const uint8_t* src = heads + (size_t)(uint32_t)page * p.page_bytes + (tile & (tpp - 1)) * (P * kKvTileBytes);
#pragma unroll
          for (int pl = 0; pl < P; ++pl) {
            cp_async_16(fill_at + (u * P + pl) * kKvTileBytes, src + pl * kKvTileBytes);
            cp_async_16(fill_at + (u * P + pl) * kKvTileBytes + 512, src + pl * kKvTileBytes + 512);
            if (lane < 8) cp_async_16(fill_at + (u * P + pl) * kKvTileBytes + kKvPairs, src + pl * kKvTileBytes + kKvPairs);
          }
          have |= 1u << (4 * (kKvStages - 1) + u);
        }
      }
      fill_at += kStep;
      if (fill_at == ring_addr + 16 * lane + kKvStages * kStep) fill_at = ring_addr + 16 * lane;
    };
#pragma unroll 1
    for (int i = 0; i < kKvStages - 1; ++i) {
      have >>= 4;
      if (i < n_steps) fill(i);
      cp_async_commit();
    }
    // (under the first copies)
    KvQuery<P, NT> q;
    kv_load_query<P, NT>(p, it, lane, q);
    KvState<P, NT> st;
    st.fresh = (1u << (2 * NT)) - 1;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      st.m[n] = st.l[n] = st.d[n] = 0;
#pragma unroll
      for (int pl = 0; pl < P; ++pl) {
        st.z[pl][n] = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) st.o[n][pl][j][0] = st.o[n][pl][j][1] = 0;
      }
    }
    uint64_t e[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) e[n] = 0;
    auto begin = [&](int i) {
      have >>= 4;
      cp_async_wait<kKvStages - 2>();
      __syncwarp();   // this step's tiles are there for every lane; the stage filled now was read a step ago
      if (i + kKvStages - 1 < n_steps) fill(i + kKvStages - 1);
      cp_async_commit();
    };
    auto step = [&](auto large, int i) -> bool {
      const int key0 = (tile0 + U * i) * kKvTile;
      const uint32_t there = have & ((1u << U) - 1);
      if (there == (1u << U) - 1 && key0 + U * kKvTile <= q.all) {
        if (!kv_step<true, decltype(large)::value, P, NT, U>(ring + use_at, there, key0, it.kv_len, q, lane, st, e)) return false;
      } else {
        if (!kv_step<false, decltype(large)::value, P, NT, U>(ring + use_at, there, key0, it.kv_len, q, lane, st, e)) return false;
      }
      use_at += kStep;
      if (use_at == kKvStages * kStep) use_at = 0;
      return true;
    };
    int i = 0;
    bool begun = false;
    if (!q.large) {
#pragma unroll 1
      for (; i < n_steps; ++i) {
        begin(i);
        if (!step(std::false_type(), i)) {
          begun = true;
          break;
        }
      }
      if (begun) {   // (as kv_load_query leaves them for large queries)
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          q.fac[n] = mul2(q.fac[n], twice_f32(0x1p-40f));
#pragma unroll
          for (int pl = 0; pl < P; ++pl) q.sum[pl][n] = mul2(q.sum[pl][n], twice_f32(0x1p-16f));
        }
      }
    }
#pragma unroll 1
    while (i < n_steps) {
      if (!begun) begin(i);
      begun = !step(std::true_type(), i);   // (again at most once: a row that has begun anew does not)
      i += begun ? 0 : 1;
    }
    // ---- the rows to shared memory: the ring is idle, a piece to be joined with the warp before has its own place
    __syncwarp();
    const bool inside = tile0 > 0, whole = !inside && left == 0 && p.split != KV_CUT;
    float* rows = reinterpret_cast<float*>(ring + (inside ? kRing : 0));
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float l[2], m[2], d[P][2], z[P][2];
      unpair_f32(st.l[n], l[0], l[1]);
      unpair_f32(e[n], d[0][0], d[0][1]);
      if (P == 2) unpair_f32(st.d[n], d[P - 1][0], d[P - 1][1]);
      unpair_f32(st.m[n], m[0], m[1]);
#pragma unroll
      for (int pl = 0; pl < P; ++pl) unpair_f32(st.z[pl][n], z[pl][0], z[pl][1]);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float* row = rows + (8 * n + 2 * t + c) * kPitch;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
          l[c] += __shfl_xor_sync(0xffffffffu, l[c], o);
#pragma unroll
          for (int pl = 0; pl < P; ++pl) z[pl][c] += __shfl_xor_sync(0xffffffffu, z[pl][c], o);
        }
        if (g == 0) *reinterpret_cast<float2*>(row + kCh) = make_float2((st.fresh >> (2 * n + c) & 1u) ? -FLT_MAX : -m[c], l[c]);
#pragma unroll
        for (int pl = 0; pl < P; ++pl) {
          const float back = kv_exp2(-d[pl][c]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float x[2], y[2];
            unpair_f32(st.o[n][pl][j][0], x[0], x[1]);
            unpair_f32(st.o[n][pl][j][1], y[0], y[1]);
            row[64 * pl + 16 * j + g] = fmaf(x[c], back * 0x1p24f, z[pl][c]);
            row[64 * pl + 16 * j + 8 + g] = fmaf(y[c] - x[c], back * 0x1p20f, z[pl][c]);
          }
        }
      }
    }
    __syncwarp();
    if (whole) {
#pragma unroll 1
      for (int i = lane; i < kRows * kCh / 4; i += 32) {
        const int row = i / (kCh / 4), ch = 4 * (i % (kCh / 4)), r = it.row0 + row;
        if (r >= n_rows) break;
        KvSum sum = {0.f, rows[row * kPitch + kCh + 1], *reinterpret_cast<const float4*>(rows + row * kPitch + ch)};
        *reinterpret_cast<uint2*>(kv_out(p, it.t0, it.head, r, ch, kCh)) = sum.result();
      }
      __syncwarp();   // (the ring is filled again)
    } else if (lane == 0) {
      s_piece[warp][inside ? 0 : 1] = {it.head, it.row0, it.t0, n_rows, left};
    }
  }
  __syncthreads();
  // ---- pieces of the CTA's warps, in order, a thread for four channels of a row
  const size_t cta = p.split == KV_CUT ? ((size_t)blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x : blockIdx.x;
  float* part = p.part + cta * 2 * kRows * kPitch;
  int4 open_item = make_int4(0, 0, 0, 0);   // of an item that this CTA begins and does not end: head, first row, t0 | rows, CTAs behind
  int open_rows = 0;
#pragma unroll 1
  for (int i = threadIdx.x; i < kRows * kCh / 4; i += 32 * kKvAttWarps) {
    const int row = i / (kCh / 4), ch = 4 * (i % (kCh / 4));
    KvSum sum = {-FLT_MAX, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
    KvPiece d = {0, 0, 0, 0, -1};
    bool open = false, outside = false;   // the item began in a CTA before
    auto leave = [&](int slot) {
      float* dst = part + (slot * kRows + row) * kPitch;
      *reinterpret_cast<float4*>(dst + ch) = sum.v;
      if (ch == 0) *reinterpret_cast<float2*>(dst + kCh) = make_float2(sum.m, sum.l);
    };
#pragma unroll 1
    for (int k = 0; k < 2 * kKvAttWarps; ++k) {
      const KvPiece e = s_piece[k >> 1][k & 1];
      if (e.left < 0) continue;
      const float* src = reinterpret_cast<const float*>(smem + (k >> 1) * (kRing + kPiece) + ((k & 1) ? 0 : kRing)) + row * kPitch;
      const float2 ml = *reinterpret_cast<const float2*>(src + kCh);
      const float4 v = *reinterpret_cast<const float4*>(src + ch);
      if (p.split == KV_CUT) {   // everything belongs to one item
        sum.add(ml.x, ml.y, v);
        continue;
      }
      if (!open) {
        sum = {ml.x, ml.y, v};
        outside = (k & 1) == 0;
        open = true;
      } else {
        sum.add(ml.x, ml.y, v);
      }
      d = e;
      if (e.left == 0) {
        open = false;
        if (outside) leave(0);
        else if (d.row0 + row < d.n_rows) *reinterpret_cast<uint2*>(kv_out(p, d.t0, d.head, d.row0 + row, ch, kCh)) = sum.result();
      }
    }
    if (p.split == KV_CUT) leave(0);
    if (open) {
      leave(outside ? 0 : 1);
      if (!outside) {
        open_item = make_int4(d.head, d.row0, d.t0, (int)kv_div(d.left + kKvAttWarps * run - 1, kKvAttWarps * run));
        open_rows = d.n_rows;
      }
    }
  }
  if (p.split == KV_SHARES && threadIdx.x == 0) {
    p.desc[blockIdx.x * 2] = open_item;
    p.desc[blockIdx.x * 2 + 1].x = open_rows;
  }
}

// Items that several CTAs share.  KV_SHARES: CTA (w, y) looks at the item that CTA w begins without ending it, and adds up, for ROWS
// of its rows, that piece (slot 1) and those of the CTAs behind (slot 0).  KV_CUT: CTA (head, block, y) adds up the item's `cuts`
// pieces (slot 0).  Bound by latency: the chain item, pieces, result.
// SETS = 1: a thread for four channels of every row walks the pieces (most items have two: a step of 256 requests spends 3 us
// less here than with sets).  Few long items of many pieces: several sets of threads take a run of pieces each.
template <int P, int NT, int ROWS, int SETS>
__global__ void __launch_bounds__(ROWS * 16 * P * SETS)
kv_join_kernel(const KvAttParams p, int cuts) {
  constexpr int kRows = 8 * NT, kCh = 64 * P, kPitch = kCh + 4, kThreads = ROWS * kCh / 4, kAhead = SETS == 1 ? 2 : 6;
  __shared__ float4 s_acc[SETS][SETS == 1 ? 1 : kThreads];
  __shared__ float2 s_ml[SETS][ROWS];
  pdl_begin();
  const int set = SETS == 1 ? 0 : threadIdx.x / kThreads, e = threadIdx.x % kThreads;
  const int row_at = e / (kCh / 4), ch = 4 * (e % (kCh / 4));
  int head, row0, t0, n_rows, n, y;   // of the item; its pieces; which rows
  size_t first;
  if (p.split == KV_CUT) {
    const KvItem it = kv_item(p, 0, blockIdx.x, blockIdx.y * kRows);
    head = it.head; row0 = it.row0; t0 = it.t0; n_rows = it.q_len * p.G; n = cuts; y = blockIdx.z;
    first = ((size_t)blockIdx.y * gridDim.x + blockIdx.x) * cuts;
  } else {
    const int4 d = p.desc[blockIdx.x * 2];
    n_rows = p.desc[blockIdx.x * 2 + 1].x;
    head = d.x; row0 = d.y; t0 = d.z; n = d.w == 0 ? 0 : d.w + 1; y = blockIdx.y;
    first = blockIdx.x;
  }
  if (n == 0 || row0 + y * ROWS >= n_rows) return;
  const int row = y * ROWS + row_at, r = row0 + row;
  // (each set of threads takes a run of pieces: the order of the sums is that of the tokens)
  const int sets = min(n, SETS), i0 = set < sets ? n * set / sets : 0, i1 = set < sets ? n * (set + 1) / sets : 0;
  KvSum sum = {-FLT_MAX, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
  for (int i = i0; i < i1; i += kAhead) {
    float2 ml[kAhead];
    float4 v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k < i1) {
        const float* part = p.part + ((first + i + k) * 2 + (i + k == 0 && p.split == KV_SHARES ? 1 : 0)) * kRows * kPitch + row * kPitch;
        ml[k] = *reinterpret_cast<const float2*>(part + kCh);
        v[k] = *reinterpret_cast<const float4*>(part + ch);
      }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k < i1) sum.add(ml[k].x, ml[k].y, v[k]);
  }
  if (SETS > 1) {
    if (set > 0 && set < sets) {
      s_acc[set][e] = sum.v;
      if (ch == 0) s_ml[set][row_at] = make_float2(sum.m, sum.l);
    }
    __syncthreads();
    if (set != 0) return;
    for (int i = 1; i < sets; ++i) sum.add(s_ml[i][row_at].x, s_ml[i][row_at].y, s_acc[i][e]);
  }
  if (r < n_rows) *reinterpret_cast<uint2*>(kv_out(p, t0, head, r, ch, kCh)) = sum.result();
}

template <int P, int NT, int U>
constexpr size_t kv_att_smem() {
  return (size_t)kKvAttWarps * (kv_ring_bytes<P, NT, U>() + 8 * NT * (64 * P + 4) * sizeof(float));
}
static size_t kv_part_bytes(int planes, int nt) { return (size_t)kKvMaxWorkers * 2 * 8 * nt * (64 * planes + 4) * sizeof(float); }

template <int P, int NT, int U>
static moin_status kv_att_launch(HostState* hs, int optin, KvAttParams& p, cudaStream_t s) {
  const size_t smem = kv_att_smem<P, NT, U>();
  cudaError_t e = ensure_smem_optin(optin, kv_attention_kernel<P, NT, U>, smem);
  if (e != cudaSuccess) return record_cuda(e);
  const long long blocks = ((long long)p.max_q * p.G + 8 * NT - 1) / (8 * NT), items = blocks * p.kv.H * p.R;
  int& per_sm = hs->kv_per_sm[optin - OPTIN_KV_ATTENTION];
  if (per_sm == 0) {
    int n = 0;
    if ((e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kv_attention_kernel<P, NT, U>, 32 * kKvAttWarps, smem)) != cudaSuccess) return record_cuda(e);
    per_sm = n < 1 ? 1 : n;
  }
  long long workers = (long long)per_sm * hs->n_sms;
  // A CTA per item needs neither places nor joins: 3 to 5 us less, until the longest item outlasts that.  One token each for R requests
  // of at most 256, 512, 1024, 1536 tokens, in us, whole items / shares:
  //   heads 32 of 64, 4 kv heads    R = 4    5.8 / 11.7    7.2 / 11.9    9.6 / 11.9   12.3 / 12.3
  //                                 R = 64   6.6 / 12.9    8.3 / 13.3   11.3 / 16.0   14.3 / 17.7
  //                                 R = 256 14.4 / 17.0   19.4 / 20.3   27.7 / 27.7   36.9 / 35.4   (1.7 waves of items)
  //   heads 32 of 128, 8 kv heads   R = 64  16.2 / 19.3   20.7 / 20.7   27.8 / 26.8   37.2 / 34.0   (1.2 waves)
  //                                 R = 256 42.3 / 29.8   60.0 / 43.8   83.2 / 67.2  106.3 / 90.4   (4.6 waves)
  //   one request, whole / cut                5.7 / 6.9     7.0 / 7.0     9.1 / 7.1   11.6 / 7.3
  const int longest = p.R == 1 ? 512 : items <= workers ? 1536 : items <= 2 * workers ? 512 : 0;
  p.split = p.max_kv <= longest && blocks <= 0x7FFFFFFF ? KV_WHOLE : p.R == 1 && blocks <= 65535 ? KV_CUT : KV_SHARES;
  ProfScope prof(MOIN_K_KV_ATTENTION, p.split == KV_WHOLE ? 1 : 2, s);
  if (p.split == KV_WHOLE)
    return record_cuda(launch_pdl(kv_attention_kernel<P, NT, U>, dim3((unsigned)blocks, (unsigned)p.kv.H, (unsigned)p.R), 32 * kKvAttWarps, smem, s, p));
  if (workers > kKvMaxWorkers) workers = kKvMaxWorkers;
  const int tiles = (p.max_kv + kKvTile - 1) / kKvTile;
  if (p.split == KV_CUT && items <= workers) {   // of one request all items are alike: no places to be found, no more joins than items
    long long cuts = workers / items, most = (tiles + kKvAttWarps * U - 1) / (kKvAttWarps * U);
    if (cuts > most) cuts = most;
    e = launch_pdl(kv_attention_kernel<P, NT, U>, dim3((unsigned)cuts, (unsigned)p.kv.H, (unsigned)blocks), 32 * kKvAttWarps, smem, s, p);
    if (e != cudaSuccess) return record_cuda(e);
    return record_cuda(launch_pdl(kv_join_kernel<P, NT, 1, 16 / P>, dim3((unsigned)p.kv.H, (unsigned)blocks, 8 * NT), 256, 0, s, p, (int)cuts));
  }
  p.split = KV_SHARES;
  // no more CTAs than there can be shares
  const long long most = (long long)(tiles + kKvItemCost) * items / (kKvAttWarps * (kKvItemCost + 2 * U)) + 1;
  if (workers > most) workers = most;
  e = launch_pdl(kv_attention_kernel<P, NT, U>, (unsigned)workers, 32 * kKvAttWarps, smem, s, p);
  if (e != cudaSuccess) return record_cuda(e);
  if (workers > 8 * items) e = launch_pdl(kv_join_kernel<P, NT, 2, 8 / P>, dim3((unsigned)workers, 4 * NT), 256, 0, s, p, 0);
  else e = launch_pdl(kv_join_kernel<P, NT, 8 * NT, 1>, (unsigned)workers, 128 * P * NT, 0, s, p, 0);
  return record_cuda(e);
}

__global__ void __launch_bounds__(256)
kv_rope_kernel(float2* __restrict__ table, int n_pos, int half, double base) {
  pdl_begin();
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  if (idx >= (long long)n_pos * half) return;
  const int pos = (int)(idx / half), i = (int)(idx % half);
  const double ang = (double)pos * pow(base, -(double)i / (double)half);
  table[idx] = make_float2((float)cos(ang), (float)sin(ang));
}

}  // namespace moin

using namespace moin;

extern "C" moin_status moin_rope_table(float* table, int32_t n_pos, int32_t head_dim, float base, moin_stream stream) {
  if (n_pos < 0 || !(base > 0.f)) return MOIN_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return MOIN_ERR_BAD_SHAPE;
  if (n_pos == 0) return MOIN_OK;
  if (!table) return MOIN_ERR_INVALID_ARG;
  if (!aligned16(table)) return MOIN_ERR_MISALIGNED;
  HostState* hs;
  moin_status st = host_state(&hs);
  if (st) return st;
  ProfScope prof(MOIN_K_GLUE, 1, (cudaStream_t)stream);
  const long long n = (long long)n_pos * (head_dim / 2);
  return record_cuda(launch_pdl(kv_rope_kernel, (unsigned)((n + 255) / 256), 256, 0, (cudaStream_t)stream, (float2*)table, n_pos, head_dim / 2, (double)base));
}

// Row blocks of 8 NT rows: as many as a request has, up to what the registers hold.
static int kv_nt(long long tall) { return tall <= 8 ? 1 : 2; }

// Long chunks go to the tcgen05 kernel (kv_chunk.cu) where the times that both would take, in us as fitted to measurements, say so:
// here a row of queries passes 0.66 keys per ns and pays for beginning an item; there a CTA of 296 takes 1.9 us for 128 keys of 128 rows
// and twice that to begin and end an item, keys, values and queries are laid out first, and there are three launches.  Measured, here /
// there, for chunks of q tokens behind p:
//   32 heads on 4    R = 1    p 500   q 64 18 / 19     q 128 24 / 21     q 512 40 / 28     p 4000  q 64 30 / 30     q 512 118 / 55
//                    R = 16   p 1     q 64 23 / 26     q 128 37 / 33     q 512 226 / 126   p 4000  q 16 63 / 53     q 512 1634 / 553
//                    R = 64   p 1     q 64 55 / 60     q 128 122 / 118   q 256 341 / 224   p 4000  q 16 200 / 146   q 256 3091 / 1097
//   4 heads on 1     R = 1    p 4000  q 64 14 / 19     q 512 31 / 30     p 16000           q 64 19 / 26     q 512 70 / 43
//   8 heads on 8     R = 4    p 4000  q 64 28 / 40     q 128 40 / 40     q 512 118 / 61
// Over 150 such calls (R 1 to 64, p 1 to 16000, q 16 to 512) the rule's choice takes 1 % more than the better of the two.
static bool kv_use_chunk(int R, int T, int max_q, int max_kv, int n_heads, int n_kv_heads, int head_dim, float scale) {
  const double G = n_heads / n_kv_heads, H = n_kv_heads;
  const int impl = gemm_impl_option();   // 1: the kernel here, 2: the other wherever it can take the call
  if (head_dim != 64 || !(scale > 0.f) || impl == 1 || (impl == 0 && max_q * G < 64)) return false;
  const double tiles = (max_kv + 63) / 64, queries = T < (double)R * max_q ? T : (double)R * max_q;
  double items = (double)(long long)((max_q * G + 127) / 128) * R * H;
  if (items > queries * n_heads / 128 + R * H) items = queries * n_heads / 128 + R * H;
  // (the tensors that are laid out: at most 1 GiB; their blocks and rows, and the work items, within 32 bits; keys that fp16 weights hold)
  if (R * tiles * 64 * H * 264 + (double)T * n_heads * 132 > (1ll << 30) || (max_q * G / 128 + 1) * R * H > (1ll << 30) ||
      max_kv > (1 << 19)) return false;
  if (impl == 2) return true;
  const double keys = max_kv - 0.5 * (max_q < max_kv ? max_q : max_kv), pairs = items * (keys / 128 + 2) / 296;
  const double here = 11 + queries * n_heads * (keys + 240) / 0.66e6;
  return 16 + 1.9 * (pairs > 2 ? pairs : 2) + 1e-4 * R * H * max_kv + 2e-4 * queries * n_heads < here;
}

extern "C" size_t moin_kv_attention_workspace_bytes(int32_t R, int32_t T, int32_t max_q, int32_t max_kv, int32_t n_heads, int32_t n_kv_heads,
                                                    int32_t head_dim) {
  if (R < 1 || T < 1 || max_q < 1 || max_kv < 1 || n_kv_heads < 1 || n_heads < n_kv_heads || (head_dim != 64 && head_dim != 128)) return 256;
  if (max_q > T) max_q = T;
  const int planes = head_dim / 64, nt = kv_nt((long long)max_q * (n_heads / n_kv_heads));
  size_t bytes = kv_part_bytes(planes, nt) + (size_t)kKvMaxWorkers * 2 * sizeof(int4);
  if (kv_use_chunk(R, T, max_q, max_kv, n_heads, n_kv_heads, head_dim, 1.f)) {
    const size_t chunk = kv_chunk_bytes(R, T, max_kv, n_heads, n_kv_heads);
    bytes = chunk > bytes ? chunk : bytes;
  }
  return bytes;
}

extern "C" moin_status moin_kv_attention(const moin_kv* kv, const moin_kv_tables* tables, const int32_t* rows, const int32_t* cu_q,
                                         const int32_t* kv_len, int32_t R, int32_t T, int32_t max_q, int32_t max_kv, const void* q,
                                         int64_t q_stride, int32_t n_heads, float scale, const float* rope, int32_t rope_len,
                                         void* out, int64_t out_stride, void* workspace, size_t workspace_bytes, moin_stream stream) {
  KvAttParams p = {};
  moin_status st = kv_view(kv, &p.kv);
  if (st) return st;
  if (!tables || !tables->block_table || tables->n_rows < 1 || tables->max_pages < 1 || R < 0 || T < 0) return MOIN_ERR_INVALID_ARG;
  if (tables->page_tokens != kv->page_tokens || n_heads < 1 || n_heads % kv->n_kv_heads != 0) return MOIN_ERR_BAD_SHAPE;
  const long long row = (long long)tables->max_pages * kv->page_tokens;
  if (row > (1 << 30) || (!rows && R > tables->n_rows)) return MOIN_ERR_BAD_SHAPE;
  if (R == 0 || T == 0) return MOIN_OK;
  if (!cu_q || !kv_len || !q || !out) return MOIN_ERR_INVALID_ARG;
  if (max_q < 1 || max_q > T) max_q = T;
  if (max_kv < 1 || max_kv > row) max_kv = (int32_t)row;
  if (rope && rope_len < max_kv) return MOIN_ERR_BAD_SHAPE;
  if (!kv_stride_ok(q_stride, n_heads, kv->head_dim) || !kv_stride_ok(out_stride, n_heads, kv->head_dim)) return MOIN_ERR_BAD_SHAPE;
  if (!aligned16(q) || !aligned16(out) || (rope && !aligned16(rope))) return MOIN_ERR_MISALIGNED;
  const long long group = n_heads / kv->n_kv_heads;
  if (R > 65535 || max_q * group * group > 0xFFFFFFFFll) return MOIN_ERR_BAD_SHAPE;
  if (!workspace || !aligned16(workspace) || workspace_bytes < moin_kv_attention_workspace_bytes(R, T, max_q, max_kv, n_heads, kv->n_kv_heads, kv->head_dim))
    return MOIN_ERR_WORKSPACE;
  HostState* hs;
  if ((st = host_state(&hs))) return st;
  p.table = tables->block_table; p.rows = rows; p.cu_q = cu_q; p.kv_len = kv_len;
  p.n_rows = tables->n_rows; p.max_pages = tables->max_pages;
  p.R = R; p.T = T; p.max_q = max_q; p.max_kv = max_kv; p.n_heads = n_heads; p.G = n_heads / kv->n_kv_heads;
  p.q = (const __nv_bfloat16*)q; p.out = (__nv_bfloat16*)out; p.q_stride = q_stride; p.out_stride = out_stride;
  p.rope = (const float2*)rope;
  p.scale_log2 = scale * 1.4426950408889634f;
  cudaStream_t s = (cudaStream_t)stream;
  if (kv_use_chunk(R, T, max_q, max_kv, n_heads, kv->n_kv_heads, kv->head_dim, scale))
  {
    ProfScope prof(MOIN_K_KV_CHUNK, 3, s);
    KvPieces pieces;
    st = launch_kv_chunk(hs, p.kv, p.table, rows, cu_q, kv_len, p.n_rows, p.max_pages, R, T, max_q, max_kv, n_heads, p.q, q_stride, p.out, out_stride,
                         p.rope, p.scale_log2, workspace, &pieces, s);
    if (st) return st;
    p.split = KV_SHARES;
    p.inv_g = (uint32_t)((0x100000000ull + p.G - 1) / p.G);
    p.part = pieces.part;
    p.desc = pieces.desc;
    const unsigned w = (unsigned)pieces.workers;
    const cudaError_t e = pieces.workers > 8 * pieces.items ? launch_pdl(kv_join_kernel<1, 16, 8, 4>, dim3(w, 16), 512, 0, s, p, 0)
                                                            : launch_pdl(kv_join_kernel<1, 16, 16, 1>, dim3(w, 8), 256, 0, s, p, 0);
    return record_cuda(e);
  }
  p.page_bytes = (uint32_t)p.kv.tile_at(1, 0, 0);
  p.tpp_log2 = kv->page_tokens == 16 ? 0 : kv->page_tokens == 32 ? 1 : kv->page_tokens == 64 ? 2 : 3;
  const int nt = kv_nt((long long)max_q * p.G);
  p.inv_g = (uint32_t)((0x100000000ull + p.G - 1) / p.G);   // exact while row * G < 2^32
  p.part = (float*)workspace;
  p.desc = (int4*)((char*)workspace + kv_part_bytes(p.kv.planes, nt));
  if (p.kv.planes == 2) return nt == 1 ? kv_att_launch<2, 1, 2>(hs, OPTIN_KV_ATTENTION, p, s) : kv_att_launch<2, 2, 1>(hs, OPTIN_KV_ATTENTION + 1, p, s);
  return nt == 1 ? kv_att_launch<1, 1, 2>(hs, OPTIN_KV_ATTENTION + 2, p, s) : kv_att_launch<1, 2, 2>(hs, OPTIN_KV_ATTENTION + 3, p, s);
}
