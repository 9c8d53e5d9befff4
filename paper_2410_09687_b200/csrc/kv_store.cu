// The 4-bit key/value cache: rows stored by slot (rotated, quantised) and read back.  Layout: kv.cuh.
#include "kv.cuh"
#include "ptx.cuh"

namespace moin {

constexpr int kKvStoreWarps = 4;

struct KvStoreParams {
  KvView kv;
  const int* slot;                    // [T]
  const __nv_bfloat16 *k, *v;         // store: [T, H, D] with row strides
  __nv_bfloat16 *k_out, *v_out;       // read
  long long k_stride, v_stride;
  const int* pos;                     // [T], with rope
  const float2* rope;                 // [rope_len, D / 2] or nullptr
  int rope_len, T, window;
};

// Rows t .. t + 15 of a call that lie in one tile, in order, are a group: what one warp handles for a head and plane.  A
// group starts where a row does not continue the row before it, or opens a tile.  Returns whether `t` starts one.
__device__ __forceinline__ bool kv_slot_ok(const KvStoreParams& p, int s) { return s >= 0 && s < p.kv.n_pages * p.kv.page_tokens; }
__device__ __forceinline__ bool kv_group_start(const KvStoreParams& p, int t) {
  const int s = p.slot[t];
  if (!kv_slot_ok(p, s)) return false;
  return t == 0 || (s % kKvTile) == 0 || p.slot[t - 1] != s - 1;
}
struct KvGroup { int t0, i0, n, page, tile; };   // first row, its place in the tile, rows
__device__ __forceinline__ KvGroup kv_group(const KvStoreParams& p, int t0, int lane) {
  KvGroup g;
  const int s0 = p.slot[t0];
  g.t0 = t0;
  g.i0 = s0 % kKvTile;
  const bool in = lane < kKvTile - g.i0 && t0 + lane < p.T && p.slot[t0 + lane] == s0 + lane;
  const uint32_t m = __ballot_sync(0xffffffffu, in);
  g.n = __ffs(~m) - 1;   // (lanes from 16 on are out: the complement is never 0)
  g.page = s0 / p.kv.page_tokens;
  g.tile = (s0 % p.kv.page_tokens) / kKvTile;
  return g;
}

// 64 channels of a row, 16 to a lane, two to a word: x[2 j + h] = channels 16 j + 8 h + 2 t, + 1.
__device__ __forceinline__ void kv_load_row(const __nv_bfloat16* row, int t, uint32_t (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __ldg(reinterpret_cast<const uint32_t*>(row + 8 * i + 2 * t));
}
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {   // NaN if either is
  uint32_t d;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}
__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// Codes of the lane's channels of a row, added into w[j] at bit 8 s: nibbles 0, 1 are x[2 j], x[2 j + 1]; low half first channel.
//   scale = bf16(max((max - min) / 15, |min| 2^-12, 2^-64)), zero = min, code = rint((x - zero) / scale)
// Inputs are bf16, so the zero is exact, and rows that are not constant have a step above |min| 2^-12: the second term
// gives constant rows a step that is not 0 and not out of proportion (attention divides by steps).  2^-64 bounds what
// underflows: values that far below it are stored as their row's minimum.  A row with an element or a span that is not
// finite is stored as NaN.
// The quotient is rounded as a division rounds it, by Markstein's correction of a product with the correctly rounded reciprocal:
// halves of a step are common among bf16 values, and go to the even code.  It is below 15.5 (the scale is at most 2^-8 of itself
// too small), so nothing is clamped.  Adding 1.5 2^23 leaves the integer in the low bits; the rest of those words' bits
// adds up to a constant.
constexpr float kKvMagic = 12582912.f;
__device__ __forceinline__ uint32_t kv_quantise(uint32_t (&x)[8], int s, uint32_t (&w)[4]) {
  uint32_t mn = x[0], mx = x[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    mn = min2_nan(mn, x[i]);
    mx = max2_nan(mx, x[i]);
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    mn = min2_nan(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    mx = max2_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
  }
  mn = min2_nan(mn, __byte_perm(mn, mn, 0x1032));
  mx = max2_nan(mx, __byte_perm(mx, mx, 0x1032));
  float lo = bf16_lo(mn);
  const float span = bf16_lo(mx) - lo;
  const bool bad = !(span < INFINITY);
  if (bad) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = 0u;
    lo = 0.f;
  }
  const float scale = bad ? 1.f : round_bf16(fmaxf(fmaxf(span / 15.f, fabsf(lo) * 0x1p-12f), 0x1p-64f));
  const float inv = __frcp_rn(scale);
  const uint64_t nlo2 = pair_f32(-lo, -lo), inv2 = pair_f32(inv, inv), nsc2 = pair_f32(-scale, -scale), magic2 = pair_f32(kKvMagic, kKvMagic);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint64_t d = add2(pair_f32(bf16_lo(x[i]), bf16_hi(x[i])), nlo2);
    uint64_t q = mul2(d, inv2);
    q = fma2(fma2(q, nsc2, d), inv2, q);
    float a, b;
    unpair_f32(add2(q, magic2), a, b);
    const int sh = 8 * s + 4 * (i & 1);
    w[i >> 1] += (__float_as_uint(a) << sh) + (__float_as_uint(b) << (sh + 16));
  }
  return bad ? 0x7FC07FC0u : (__float_as_uint(scale) >> 16) | (__float_as_uint(lo) & 0xFFFF0000u);
}
__host__ __device__ constexpr uint32_t kv_magic_sum() {
  uint32_t sum = 0;
  for (int sh = 0; sh < 32; sh += 4) sum += 0x4B400000u << sh;
  return sum;
}

__device__ __forceinline__ void kv_rotate_words(uint32_t& a, uint32_t& b, const float4& cs) {   // (cos, sin) of two channels
  const float2 c0 = make_float2(cs.x, cs.y), c1 = make_float2(cs.z, cs.w);
  const float a0 = bf16_lo(a), a1 = bf16_hi(a), b0 = bf16_lo(b), b1 = bf16_hi(b);
  a = pack_bf16(kv_rot_lo(a0, b0, c0), kv_rot_lo(a1, b1, c1));
  b = pack_bf16(kv_rot_hi(a0, b0, c0), kv_rot_hi(a1, b1, c1));
}

// A warp stores the keys or the values of a group, of one head and NP planes of it: its lanes load two token rows (g and g + 8 of
// the tile, 16 channels a plane each), quantise them and hold the tile's words.  Whole tiles are written by 16-byte stores, others
// byte by byte, a token's own bytes only.
// Bound by the chain slot, position, (cos, sin), row, quantised words, store, with few warps to hide it: for prompts issue slots are
// 54 % busy (about 550 instructions a warp, tile and plane) at 35 % of the warps that an SM holds, for single tokens there is nothing
// but the chain.  A wide head's planes in one warp (NP = 2): a key's partner plane is not loaded and rotated twice; 21 thousand tokens of
// 8 heads of 128 take 46 us (110 MB: 2.4 TB/s); when this form took 52, a warp per plane took 71, and for few tokens was 0.9 us
// faster.  Seven CTAs an SM: 2 us less than the six that 80 registers leave.
template <int D, int NP>
__global__ void __launch_bounds__(32 * kKvStoreWarps, 7)
kv_append_kernel(const KvStoreParams p) {
  constexpr int kPer = D / 64 / NP;   // warps of a head's keys
  pdl_begin();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int unit = blockIdx.y * kKvStoreWarps + (threadIdx.x >> 5);
  if (unit >= 2 * p.kv.H * kPer) return;
  const bool value = unit & 1;
  const int hp = unit >> 1, head = hp / kPer, plane0 = hp % kPer;
  const __nv_bfloat16* base = (value ? p.v : p.k) + head * D;
  const long long stride = value ? p.v_stride : p.k_stride;
  const int first = blockIdx.x * p.window;
  uint32_t starts = __ballot_sync(0xffffffffu, lane < p.window && first + lane < p.T && kv_group_start(p, first + lane));
  while (starts) {
    const KvGroup gr = kv_group(p, first + __ffs(starts) - 1, lane);
    starts &= starts - 1;
    uint32_t x[NP][2][8];
    bool live[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      live[s] = g + 8 * s >= gr.i0 && g + 8 * s < gr.i0 + gr.n;
#pragma unroll
      for (int pl = 0; pl < NP; ++pl) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[pl][s][i] = 0u;
        if (live[s]) kv_load_row(base + (gr.t0 + g + 8 * s - gr.i0) * stride + 64 * (plane0 + pl), t, x[pl][s]);
      }
    }
    if (p.rope != nullptr) {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (!live[s]) continue;
        const int row = gr.t0 + g + 8 * s - gr.i0, at = p.pos[row];
        live[s] = at >= 0 && at < p.rope_len;   // (a value is not stored without its key)
        if (value) continue;
        const float* cs = reinterpret_cast<const float*>(p.rope + (size_t)(live[s] ? at : 0) * (D / 2) + 2 * t);
        if (D == 64) {
#pragma unroll
          for (int i = 0; i < 4; ++i) kv_rotate_words(x[0][s][i], x[0][s][i + 4], __ldg(reinterpret_cast<const float4*>(cs + 16 * i)));
        } else if (NP == 2) {
#pragma unroll
          for (int i = 0; i < 8; ++i) kv_rotate_words(x[0][s][i], x[NP - 1][s][i], __ldg(reinterpret_cast<const float4*>(cs + 16 * i)));
        } else {
          uint32_t other[8];
          kv_load_row(base + row * stride + 64 * (1 - plane0), t, other);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 c = __ldg(reinterpret_cast<const float4*>(cs + 16 * i));
            if (plane0 == 0) kv_rotate_words(x[0][s][i], other[i], c);
            else kv_rotate_words(other[i], x[0][s][i], c);
          }
        }
      }
    }
    const uint32_t rows = __ballot_sync(0xffffffffu, live[0]), rows8 = __ballot_sync(0xffffffffu, live[1]);   // bit 4 g: token g
#pragma unroll
    for (int pl = 0; pl < NP; ++pl) {
      uint32_t w[4] = {0u, 0u, 0u, 0u}, pair[2];
#pragma unroll
      for (int s = 0; s < 2; ++s) pair[s] = kv_quantise(x[pl][s], s, w);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        w[j] -= kv_magic_sum();
        if (value) w[j] = movmatrix_trans(w[j]);
      }
      uint8_t* tile = p.kv.pages + p.kv.tile_at(gr.page, head, gr.tile) + (plane0 + pl) * kKvTileBytes;
      uint8_t* words = tile + (value ? 512 : 0) + 16 * lane;
      uint32_t* pairs = reinterpret_cast<uint32_t*>(tile + kKvPairs) + 4 * g + (value ? 2 : 0);
      if ((rows & rows8) == 0xffffffffu) {
        *reinterpret_cast<uint4*>(words) = make_uint4(w[0], w[1], w[2], w[3]);
        if (t == 0) *reinterpret_cast<uint2*>(pairs) = make_uint2(pair[0], pair[1]);
        continue;
      }
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (live[s] && t == 0) pairs[s] = pair[s];
        const uint32_t r = s == 0 ? rows : rows8;
#pragma unroll
        for (int c = 0; c < 2; ++c)   // byte 2 c + s of a word: of keys token g + 8 s, of values token 2 t + c + 8 s
          if (r >> (4 * (value ? 2 * t + c : g)) & 1u) {
#pragma unroll
            for (int j = 0; j < 4; ++j) words[4 * j + 2 * c + s] = (uint8_t)(w[j] >> (16 * c + 8 * s));
          }
      }
    }
  }
}

// The rows of a group back as bf16(zero + scale code); rows without a slot are zeros.  A code becomes a bf16 by two operations on a
// pair (128 + code by its bits, less 128), its value by one fused multiply-add.  A lane's words go through shared memory, so that
// rows are written 16 bytes a lane (pitch 36 words: neither side meets a bank twice).
constexpr int kKvReadPitch = 36;
template <int D>
__global__ void __launch_bounds__(32 * kKvStoreWarps)
kv_read_kernel(const KvStoreParams p) {
  __shared__ __align__(16) uint32_t s_rows[kKvStoreWarps][kKvTile * kKvReadPitch];
  pdl_begin();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int unit = blockIdx.y * kKvStoreWarps + (threadIdx.x >> 5);
  if (unit >= 2 * p.kv.H * (D / 64)) return;
  const bool value = unit & 1;
  const int hp = unit >> 1, head = hp / (D / 64), plane = hp % (D / 64);
  __nv_bfloat16* base = (value ? p.v_out : p.k_out) + head * D + 64 * plane;
  const long long stride = value ? p.v_stride : p.k_stride;
  uint32_t* stage = s_rows[threadIdx.x >> 5];
  const int first = blockIdx.x * p.window;
  const bool mine = lane < p.window && first + lane < p.T;
  uint32_t none = __ballot_sync(0xffffffffu, mine && !kv_slot_ok(p, p.slot[mine ? first + lane : 0]));
  for (; none; none &= none - 1) reinterpret_cast<uint32_t*>(base + (first + __ffs(none) - 1) * stride)[lane] = 0u;
  uint32_t starts = __ballot_sync(0xffffffffu, mine && kv_group_start(p, mine ? first + lane : 0));
  while (starts) {
    const KvGroup gr = kv_group(p, first + __ffs(starts) - 1, lane);
    starts &= starts - 1;
    const uint8_t* tile = p.kv.pages + p.kv.tile_at(gr.page, head, gr.tile) + plane * kKvTileBytes;
    const uint4 c4 = *reinterpret_cast<const uint4*>(tile + (value ? 512 : 0) + 16 * lane);
    const uint2 pr = *reinterpret_cast<const uint2*>(tile + kKvPairs + 16 * g + (value ? 8 : 0));
    uint32_t w[4] = {c4.x, c4.y, c4.z, c4.w};
    if (value) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = movmatrix_trans(w[j]);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint32_t pair = s == 0 ? pr.x : pr.y;
      const uint32_t scale2 = __byte_perm(pair, pair, 0x1010), zero2 = __byte_perm(pair, pair, 0x3232);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t bits = (w[i >> 1] >> (8 * s + 4 * (i & 1)) & 0x000F000Fu) | 0x43004300u;
        uint32_t c, v;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(c) : "r"(bits), "r"(0x43004300u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v) : "r"(c), "r"(scale2), "r"(zero2));
        stage[(g + 8 * s) * kKvReadPitch + 4 * i + t] = v;
      }
    }
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = 4 * k + (lane >> 3);
      if (row >= gr.i0 && row < gr.i0 + gr.n)
        *reinterpret_cast<uint4*>(base + (gr.t0 + row - gr.i0) * stride + 8 * (lane & 7)) =
            *reinterpret_cast<const uint4*>(stage + row * kKvReadPitch + 4 * (lane & 7));
    }
    __syncwarp();
  }
}

// Rows in which a CTA looks for groups.  One while warps are few, so that every token has its own; more beyond, where the groups of
// prompts are whole tiles and most warps of single rows would find nothing.  Stored and read back in us, windows of 1, 4, 8, 32 rows:
//   4 heads of 64    1024 single tokens  13 23 35 72     1024 of a prompt   7.8 7.5 7.2 10     4096 single  40 39 50 124    4096 of prompts  20 11 11 15
//                    16384 of prompts    71 23 19 20
//   8 heads of 128   256 single          15 26 46 108    1024 single        44 45 55 162       1024 of a prompt  23 13 13 22
//                    8192 of prompts     107 40 32 29    16384              209 75 59 52
static int kv_window(const KvStoreParams& p) {
  const long long warps = (long long)p.T * 2 * p.kv.H * p.kv.planes;
  return warps <= 12000 ? 1 : warps <= 66000 ? 4 : warps <= 200000 ? 8 : 32;
}

template <class Fn>
static moin_status kv_store_launch(Fn* fn, KvStoreParams& p, int per_head, cudaStream_t s) {
  p.window = kv_window(p);
  const dim3 grid((unsigned)((p.T + (long long)p.window - 1) / p.window), (unsigned)((2 * p.kv.H * per_head + kKvStoreWarps - 1) / kKvStoreWarps));
  ProfScope prof(MOIN_K_KV_STORE, 1, s);
  return record_cuda(launch_pdl(fn, grid, 32 * kKvStoreWarps, 0, s, p));
}

}  // namespace moin

using namespace moin;

extern "C" size_t moin_kv_bytes(int32_t n_pages, int32_t page_tokens, int32_t n_kv_heads, int32_t head_dim) {
  if (n_pages < 0 || page_tokens < 0 || n_kv_heads < 0 || head_dim < 0) return 0;
  return (size_t)n_pages * n_kv_heads * (page_tokens / kKvTile) * (head_dim / 64) * kKvTileBytes;
}

extern "C" moin_status moin_kv_append(const moin_kv* kv, const int32_t* slot, const void* k, int64_t k_stride, const void* v,
                                      int64_t v_stride, const int32_t* pos, const float* rope, int32_t rope_len, int32_t T,
                                      moin_stream stream) {
  KvStoreParams p = {};
  moin_status st = kv_view(kv, &p.kv);
  if (st) return st;
  if (T < 0 || rope_len < 0) return MOIN_ERR_INVALID_ARG;
  if (T == 0) return MOIN_OK;
  if (!slot || !k || !v || (rope && !pos)) return MOIN_ERR_INVALID_ARG;
  if (!kv_stride_ok(k_stride, kv->n_kv_heads, kv->head_dim) || !kv_stride_ok(v_stride, kv->n_kv_heads, kv->head_dim)) return MOIN_ERR_BAD_SHAPE;
  if (!aligned16(k) || !aligned16(v) || (rope && !aligned16(rope))) return MOIN_ERR_MISALIGNED;
  HostState* hs;
  if ((st = host_state(&hs))) return st;
  p.slot = slot; p.k = (const __nv_bfloat16*)k; p.v = (const __nv_bfloat16*)v;
  p.k_stride = k_stride; p.v_stride = v_stride;
  p.pos = pos; p.rope = (const float2*)rope; p.rope_len = rope_len; p.T = T;
  if (kv->head_dim == 64) return kv_store_launch(kv_append_kernel<64, 1>, p, 1, (cudaStream_t)stream);
  if (kv_window(p) > 1) return kv_store_launch(kv_append_kernel<128, 2>, p, 1, (cudaStream_t)stream);
  return kv_store_launch(kv_append_kernel<128, 1>, p, 2, (cudaStream_t)stream);
}

extern "C" moin_status moin_kv_read(const moin_kv* kv, const int32_t* slot, void* k, int64_t k_stride, void* v, int64_t v_stride,
                                    int32_t T, moin_stream stream) {
  KvStoreParams p = {};
  moin_status st = kv_view(kv, &p.kv);
  if (st) return st;
  if (T < 0) return MOIN_ERR_INVALID_ARG;
  if (T == 0) return MOIN_OK;
  if (!slot || !k || !v) return MOIN_ERR_INVALID_ARG;
  if (!kv_stride_ok(k_stride, kv->n_kv_heads, kv->head_dim) || !kv_stride_ok(v_stride, kv->n_kv_heads, kv->head_dim)) return MOIN_ERR_BAD_SHAPE;
  if (!aligned16(k) || !aligned16(v)) return MOIN_ERR_MISALIGNED;
  HostState* hs;
  if ((st = host_state(&hs))) return st;
  p.slot = slot; p.k_out = (__nv_bfloat16*)k; p.v_out = (__nv_bfloat16*)v;
  p.k_stride = k_stride; p.v_stride = v_stride; p.T = T;
  return kv->head_dim == 64 ? kv_store_launch(kv_read_kernel<64>, p, 1, (cudaStream_t)stream)
                            : kv_store_launch(kv_read_kernel<128>, p, 2, (cudaStream_t)stream);
}
