// Attention over the 4-bit key/value cache (layout: kv.cuh).
//
// For a query row, with K_t = zk_t + sk_t ck_t and V_t = zv_t + sv_t cv_t per plane of 64 channels (codes c = 0 .. 15):
//   s_t = scale (sk_t (q . ck_t) + zk_t sum(q));    o = [sum_t (p_t sv_t) cv_t + sum_t p_t zv_t] / sum_t p_t,   p_t = 2^(s_t log2(e) - m)
// so the codes enter the tensor cores as they are and every scale is applied to a score, not to 64 elements.  Both products
// are warp MMAs (m16n8k16, fp16 operands, fp32 sums) with the codes as A, 16 tokens x 16 channels or their transpose, and
// 8 query rows as the columns of B: the g query heads of a kv head fill them.  A code is put into the low mantissa bits of an
// fp16 by one AND: c 2^-24, a subnormal that tensor cores multiply exactly (the upper nibble of a byte gives 16 c 2^-24;
// its query channels are divided by 16, its value channels at the end).  Queries are bf16 times a power of two per row that
// brings them into the middle of fp16: exact.  The weights p sv are the only operand that is rounded, to fp16 (2^-12
// relative); their sums p are not.  To keep them inside fp16 whatever the scales are, m follows the maximum of s_t +
// log2(sv_t): a weight is at most 2^15, and precise to 2^-24 of the row's largest.  m lags (a row is rescaled when a
// weight would exceed 2^15, to 2^10), so most tiles need no reduction over the warp.
//
// Sums over many tokens are made by fp32 additions that round, not in the accumulator of the MMA, which truncates: codes are
// positive, so the sum grows with every token while what is left of it after sum p zv shrinks with their number (131072 tokens
// in chains of 2048 MMAs: results 2 % off; like this 0.17 %, the rounding of the output).
//
// Scores come out as [token x row] with a lane holding two rows of two tokens; the second product wants weights as [token x
// row] with tokens along a lane's registers: one movmatrix per 8 x 8 block turns them.
#include <float.h>

#include "kv.cuh"

namespace moin {

constexpr int kKvAttWarps = 4;
constexpr float kKvTop = 10.f;       // log2 of the largest weight after a rescale
constexpr float kKvMost = 15.f;      // log2 of the largest weight at all

struct KvAttParams {
  KvView kv;
  const int *table, *rows, *cu_q, *kv_len;
  int n_rows, max_pages;
  int R, T, max_q, max_kv, G, n_heads;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  long long q_stride, out_stride;
  const float2* rope;      // [rope_len, D / 2] or nullptr
  float scale_log2;
};

__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
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

// What a CTA works on: the rows [row0, row0 + 8 NT) of request `req` and kv head `head`; row = (query token) * G + head of the group.
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
  it.table = p.table + (size_t)(it.kv_len ? row : 0) * p.max_pages;
  return it;
}

template <int P, int NT>
struct KvState {            // a warp's share of an item: 8 NT rows, 64 P channels
  float o[NT][P][4][4];     // [channel block of 16][(g, row 2 t), (g, row 2 t + 1), (g + 8, ..)]
  float m[NT][2], l[NT][2], z[P][NT][2];
};

// Query rows as B fragments: b[n][plane][k-step][half], and per row (2 t, 2 t + 1 of an n-tile) the factor and the sum.
template <int P, int NT>
struct KvQuery {
  uint32_t b[NT][P][4][2];
  float fac[NT][2], sum[P][NT][2];
  int last[NT][2];          // last key the row sees
  int all;                  // keys below this are seen by every row
};

template <int P, int NT>
__device__ __forceinline__ void kv_load_query(const KvAttParams& p, const KvItem& it, int lane, KvQuery<P, NT>& q) {
  const int g = lane >> 2, t = lane & 3;
  const int n_rows = it.q_len * p.G, past = it.kv_len - it.q_len;
  q.all = it.kv_len;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int row = it.row0 + 8 * n + g;
    const int qi = row / p.G;
    const bool live = row < n_rows && past + qi >= 0;
    float x[P][16];
#pragma unroll
    for (int pl = 0; pl < P; ++pl)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[pl][i] = 0.f;
    if (live) {
      const __nv_bfloat16* src = p.q + (long long)(it.t0 + qi) * p.q_stride + (it.head * p.G + row % p.G) * 64 * P;
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
    const float f = (e > -120 && e < 128) ? __uint_as_float((uint32_t)(9 - e + 127) << 23) : 1.f;
    float sum[P];
#pragma unroll
    for (int pl = 0; pl < P; ++pl) {
      sum[pl] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sum[pl] += (x[pl][4 * j] + x[pl][4 * j + 1]) + (x[pl][4 * j + 2] + x[pl][4 * j + 3]);
        q.b[n][pl][j][0] = pack_f16(x[pl][4 * j] * f, x[pl][4 * j + 1] * f);
        q.b[n][pl][j][1] = pack_f16(x[pl][4 * j + 2] * f * 0.0625f, x[pl][4 * j + 3] * f * 0.0625f);
      }
      sum[pl] += __shfl_xor_sync(0xffffffffu, sum[pl], 1);
      sum[pl] += __shfl_xor_sync(0xffffffffu, sum[pl], 2);
    }
    // to the lanes that hold these rows' scores: rows 2 t, 2 t + 1 of the n-tile
    const float fac = p.scale_log2 * 0x1p24f / f;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int from = 4 * (2 * t + c);
      q.fac[n][c] = __shfl_sync(0xffffffffu, fac, from);
#pragma unroll
      for (int pl = 0; pl < P; ++pl) q.sum[pl][n][c] = __shfl_sync(0xffffffffu, sum[pl], from) * p.scale_log2;
      const int r = it.row0 + 8 * n + 2 * t + c;
      // rows that are not there compute something that is not stored, and mask nothing
      q.last[n][c] = r < n_rows ? past + r / p.G : it.kv_len - 1;
      q.all = min(q.all, q.last[n][c] + 1);
    }
  }
  q.all = min(q.all, __shfl_xor_sync(0xffffffffu, q.all, 1));
  q.all = min(q.all, __shfl_xor_sync(0xffffffffu, q.all, 2));
}

struct KvTileRegs { uint4 k, v, pr; };

template <int P>
__device__ __forceinline__ void kv_load_tile(const uint8_t* at, int lane, KvTileRegs (&r)[P]) {
#pragma unroll
  for (int pl = 0; pl < P; ++pl) {
    r[pl].k = ldg_stream(at + pl * kKvTileBytes + 16 * lane);
    r[pl].v = ldg_stream(at + pl * kKvTileBytes + 512 + 16 * lane);
    r[pl].pr = ldg_stream(at + pl * kKvTileBytes + kKvPairs + 16 * (lane >> 2));
  }
}

// One tile of 16 tokens from `key0` on.
template <int P, int NT>
__device__ __forceinline__ void kv_tile(const KvTileRegs (&r)[P], int key0, int kv_len, const KvQuery<P, NT>& q, int lane, KvState<P, NT>& st) {
  constexpr uint32_t kLo = 0x000F000Fu, kHi = 0x00F000F0u;
  const int g = lane >> 2;
  float s[NT][4];
  uint32_t pk[P][2], pv[P][2];
  const bool whole = key0 + kKvTile <= q.all;
#pragma unroll
  for (int pl = 0; pl < P; ++pl) {
    pk[pl][0] = r[pl].pr.x; pk[pl][1] = r[pl].pr.y; pv[pl][0] = r[pl].pr.z; pv[pl][1] = r[pl].pr.w;
    if (!whole) {   // what lies behind the last token was never written
      if (key0 + g >= kv_len) pk[pl][0] = pv[pl][0] = 0;
      if (key0 + g + 8 >= kv_len) pk[pl][1] = pv[pl][1] = 0;
    }
    const uint32_t kw[4] = {r[pl].k.x, r[pl].k.y, r[pl].k.z, r[pl].k.w};
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
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float zero = pl == 0 ? 0.f : s[n][e];
        s[n][e] = fmaf(acc[n][e], q.fac[n][e & 1] * kv_scale(pk[pl][e >> 1]), fmaf(q.sum[pl][n][e & 1], kv_zero(pk[pl][e >> 1]), zero));
      }
  }
  float lg[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float sv = kv_scale(pv[0][h]);
    if (P == 2) sv = fmaxf(sv, kv_scale(pv[P - 1][h]));
    lg[h] = fmaxf(kv_log2(sv), -64.f);
  }
  if (!whole) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (key0 + g + 8 * (e >> 1) > q.last[n][e & 1]) s[n][e] = -INFINITY;
  }
  bool grow = false;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) grow = grow || s[n][e] + lg[e >> 1] > st.m[n][e & 1] + kKvMost;
  if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float mx = fmaxf(s[n][c] + lg[0], s[n][c + 2] + lg[1]);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        if (mx > st.m[n][c] + kKvMost) {
          const float m = mx - kKvTop, corr = kv_exp2(st.m[n][c] - m);
          st.l[n][c] = kv_rescale_sum(st.l[n][c], st.m[n][c] - m);
          st.m[n][c] = m;
#pragma unroll
          for (int pl = 0; pl < P; ++pl) {
            st.z[pl][n][c] *= corr;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              st.o[n][pl][j][c] *= corr;
              st.o[n][pl][j][c + 2] *= corr;
            }
          }
        }
      }
  }
  uint32_t b[NT][P][2];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float pr[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      pr[e] = kv_exp2(s[n][e] - st.m[n][e & 1]);
      st.l[n][e & 1] += pr[e];
    }
#pragma unroll
    for (int pl = 0; pl < P; ++pl) {
      float w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float zv = kv_zero(pv[pl][e >> 1]);
        w[e] = pr[e] * kv_scale(pv[pl][e >> 1]);
        if (!whole) {   // a value that a row must not see may be anything
          const bool out = key0 + g + 8 * (e >> 1) > q.last[n][e & 1];
          w[e] = out ? 0.f : w[e];
          st.z[pl][n][e & 1] += out ? 0.f : pr[e] * zv;
        } else {
          st.z[pl][n][e & 1] = fmaf(pr[e], zv, st.z[pl][n][e & 1]);
        }
      }
      b[n][pl][0] = movmatrix_trans(pack_f16(w[0], w[1]));
      b[n][pl][1] = movmatrix_trans(pack_f16(w[2], w[3]));
    }
  }
#pragma unroll
  for (int pl = 0; pl < P; ++pl) {
    const uint32_t vw[4] = {r[pl].v.x, r[pl].v.y, r[pl].v.z, r[pl].v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = vw[j], w8 = w >> 8;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float d[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16_16816(d, w & kLo, w & kHi, w8 & kLo, w8 & kHi, b[n][pl][0], b[n][pl][1]);
#pragma unroll
        for (int e = 0; e < 4; ++e) st.o[n][pl][j][e] += d[e];
      }
    }
  }
}

// A CTA takes an item; its warps take the item's tiles in turn and meet in shared memory.
template <int P, int NT>
__global__ void __launch_bounds__(32 * kKvAttWarps)
kv_attention_kernel(const KvAttParams p) {
  constexpr int kRows = 8 * NT, kCh = 64 * P, kPitch = kCh + 4;
  extern __shared__ float smem[];
  float* s_o = smem;                                             // [warp][row][channel]
  float* s_ml = smem + kKvAttWarps * kRows * kPitch;             // [warp][row][m, l, z ..]
  pdl_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const KvItem it = kv_item(p, blockIdx.z, blockIdx.y, blockIdx.x * kRows);
  const int n_rows = it.q_len * p.G;
  if (it.row0 >= n_rows) return;
  KvQuery<P, NT> q;
  kv_load_query<P, NT>(p, it, lane, q);
  KvState<P, NT> st;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      st.m[n][c] = -FLT_MAX;
      st.l[n][c] = 0.f;
#pragma unroll
      for (int pl = 0; pl < P; ++pl) st.z[pl][n][c] = 0.f;
    }
#pragma unroll
    for (int pl = 0; pl < P; ++pl)
#pragma unroll
      for (int j = 0; j < 4; ++j) st.o[n][pl][j][0] = st.o[n][pl][j][1] = st.o[n][pl][j][2] = st.o[n][pl][j][3] = 0.f;
  }
  // keys that the last row of the tile sees
  const int see = max(0, min(it.kv_len, it.kv_len - it.q_len + min(it.row0 + kRows - 1, n_rows - 1) / p.G + 1));
  const int n_tiles = (see + kKvTile - 1) / kKvTile, tpp = p.kv.page_tokens / kKvTile;
  for (int i = warp; i < n_tiles; i += kKvAttWarps) {
    const int page = __ldg(it.table + i / tpp);
    if (page < 0 || page >= p.kv.n_pages) continue;   // (the same for the whole warp)
    KvTileRegs r[P];
    kv_load_tile<P>(p.kv.pages + p.kv.tile_at(page, it.head, i % tpp), lane, r);
    kv_tile<P, NT>(r, i * kKvTile, it.kv_len, q, lane, st);
  }
  // ---- this warp's sums to shared memory
  float* mine = s_o + warp * kRows * kPitch;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int row = 8 * n + 2 * t + c;
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) {
        st.l[n][c] += __shfl_xor_sync(0xffffffffu, st.l[n][c], o);
#pragma unroll
        for (int pl = 0; pl < P; ++pl) st.z[pl][n][c] += __shfl_xor_sync(0xffffffffu, st.z[pl][n][c], o);
      }
      if (g == 0) {
        float* ml = s_ml + (warp * kRows + row) * 4;
        ml[0] = st.m[n][c];
        ml[1] = st.l[n][c];
#pragma unroll
        for (int pl = 0; pl < P; ++pl) ml[2 + pl] = st.z[pl][n][c];
      }
#pragma unroll
      for (int pl = 0; pl < P; ++pl)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          mine[row * kPitch + 64 * pl + 16 * j + g] = st.o[n][pl][j][c] * 0x1p24f;
          mine[row * kPitch + 64 * pl + 16 * j + 8 + g] = st.o[n][pl][j][c + 2] * 0x1p20f;
        }
    }
  __syncthreads();
  // ---- joined: a thread takes two channels of a row
  for (int i = threadIdx.x; i < kRows * kCh / 2; i += 32 * kKvAttWarps) {
    const int row = i / (kCh / 2), ch = 2 * (i % (kCh / 2));
    const int r = it.row0 + row;
    if (r >= n_rows) continue;
    float top = -FLT_MAX;
#pragma unroll
    for (int w = 0; w < kKvAttWarps; ++w) top = fmaxf(top, s_ml[(w * kRows + row) * 4]);
    float l = 0.f, a = 0.f, b = 0.f;
#pragma unroll
    for (int w = 0; w < kKvAttWarps; ++w) {
      const float* ml = s_ml + (w * kRows + row) * 4;
      const float f = kv_exp2(ml[0] - top);
      const float* o = s_o + (w * kRows + row) * kPitch + ch;
      l += kv_rescale_sum(ml[1], ml[0] - top);
      a += (o[0] + ml[2 + ch / 64]) * f;
      b += (o[1] + ml[2 + ch / 64]) * f;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;   // nothing to see: zeros
    *reinterpret_cast<uint32_t*>(p.out + (long long)(it.t0 + r / p.G) * p.out_stride + (it.head * p.G + r % p.G) * kCh + ch) = pack_bf16(a * inv, b * inv);
  }
}

template <int P, int NT>
static cudaError_t kv_att_launch(const KvAttParams& p, cudaStream_t s) {
  const size_t smem = (size_t)kKvAttWarps * 8 * NT * (64 * P + 4 + 4) * sizeof(float);
  const dim3 grid((unsigned)(((long long)p.max_q * p.G + 8 * NT - 1) / (8 * NT)), (unsigned)p.kv.H, (unsigned)p.R);
  return launch_pdl(kv_attention_kernel<P, NT>, grid, 32 * kKvAttWarps, smem, s, p);
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

extern "C" size_t moin_kv_attention_workspace_bytes(int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
  (void)n_heads; (void)n_kv_heads; (void)head_dim;
  return 256;
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
  if (R > 65535 || (long long)max_q * n_heads > 0x7FFFFFFFll) return MOIN_ERR_BAD_SHAPE;
  if (!workspace || !aligned16(workspace) || workspace_bytes < moin_kv_attention_workspace_bytes(n_heads, kv->n_kv_heads, kv->head_dim))
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
  const long long tall = (long long)max_q * p.G;
  ProfScope prof(MOIN_K_KV_ATTENTION, 1, s);
  cudaError_t e;
  if (p.kv.planes == 1) e = tall <= 8 ? kv_att_launch<1, 1>(p, s) : tall <= 16 ? kv_att_launch<1, 2>(p, s) : kv_att_launch<1, 4>(p, s);
  else e = tall <= 8 ? kv_att_launch<2, 1>(p, s) : kv_att_launch<2, 2>(p, s);
  return record_cuda(e);
}
