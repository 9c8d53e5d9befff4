// The 4-bit key/value cache: rows stored by slot (rotated, quantised) and read back.  Layout: kv.cuh.
#include "kv.cuh"

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

// 64 channels of a row, 16 to a lane: x[4 j + 2 half + c] = channel 16 j + 8 half + 2 t + c.
__device__ __forceinline__ void kv_load_row(const __nv_bfloat16* row, int t, float (&x)[16]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(row + 16 * j + 8 * h + 2 * t));
      x[4 * j + 2 * h] = bf16_lo(w);
      x[4 * j + 2 * h + 1] = bf16_hi(w);
    }
}

// Codes of a row, 16 to a lane: word j holds those of x[4 j ..] in nibbles 0, 1 (low half c = 0, high half c = 1).
//   scale = bf16(max((max - min) / 15, |min| 2^-12, 2^-64)), zero = min, code = rint((x - zero) / scale) in 0 .. 15
// Inputs are bf16, so the zero is exact, and rows that are not constant have a step above |min| 2^-12: the second term
// gives constant rows a step that is not 0 and not out of proportion (attention divides by steps).  2^-64 bounds what
// underflows: values that far below it are stored as their row's minimum.  A row with an element or a span that is not
// finite is stored as NaN.
__device__ __forceinline__ uint32_t kv_quantise(const float (&x)[16], uint32_t (&w)[4]) {
  float lo = x[0], hi = x[0], bad = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    bad = fmaf(x[i], 0.f, bad);   // NaN once an element is not finite
  }
#pragma unroll
  for (int o = 1; o < 4; o <<= 1) {
    lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    bad += __shfl_xor_sync(0xffffffffu, bad, o);
  }
  const float span = hi - lo;
  bad = fmaf(span, 0.f, bad);
  const float scale = round_bf16(fmaxf(fmaxf(__fdiv_rn(span, 15.f), fabsf(lo) * 0x1p-12f), 0x1p-64f));
  const bool ok = bad == 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    w[j] = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int c = ok ? min(__float2int_rn(__fdiv_rn(x[4 * j + e] - lo, scale)), 15) : 0;
      w[j] |= (uint32_t)c << (4 * (e >> 1) + 16 * (e & 1));
    }
  }
  return ok ? (__float_as_uint(scale) >> 16) | (__float_as_uint(lo) & 0xFFFF0000u) : 0x7FC07FC0u;
}

// A warp stores a group of one head and plane: its lanes load two token rows (g and g + 8 of the tile, 16 channels each),
// quantise them and hold the tile's words.  Whole tiles are written by 16-byte stores, others byte by byte, a token's own
// bytes only.
template <int D>
__global__ void __launch_bounds__(32 * kKvStoreWarps)
kv_append_kernel(const KvStoreParams p) {
  pdl_begin();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int hp = blockIdx.y * kKvStoreWarps + (threadIdx.x >> 5);
  if (hp >= p.kv.H * (D / 64)) return;
  const int head = hp / (D / 64), plane = hp % (D / 64);
  const int first = blockIdx.x * p.window;
  uint32_t starts = __ballot_sync(0xffffffffu, lane < p.window && first + lane < p.T && kv_group_start(p, first + lane));
  while (starts) {
    const KvGroup gr = kv_group(p, first + __ffs(starts) - 1, lane);
    starts &= starts - 1;
    uint32_t word[2][2][4], pair[2][2];   // [key, value][token g, g + 8]
    bool live[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int row = gr.t0 + g + 8 * s - gr.i0;
      live[s] = g + 8 * s >= gr.i0 && g + 8 * s < gr.i0 + gr.n;
      float xk[16], xv[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) xk[i] = xv[i] = 0.f;
      if (live[s]) {
        const __nv_bfloat16* kr = p.k + (long long)row * p.k_stride + head * D;
        kv_load_row(kr + 64 * plane, t, xk);
        kv_load_row(p.v + (long long)row * p.v_stride + head * D + 64 * plane, t, xv);
        if (p.rope != nullptr) {
          const int at = p.pos[row];
          live[s] = at >= 0 && at < p.rope_len;
          const float2* cs = p.rope + (size_t)(live[s] ? at : 0) * (D / 2);
          if (D == 64) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const float2 c = __ldg(cs + 16 * (i >> 2) + 8 * ((i >> 1) & 1) + 2 * t + (i & 1));
              const float a = xk[i], b = xk[i + 8];
              xk[i] = round_bf16(kv_rot_lo(a, b, c));
              xk[i + 8] = round_bf16(kv_rot_hi(a, b, c));
            }
          } else {
            float other[16];
            kv_load_row(kr + 64 * (1 - plane), t, other);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const float2 c = __ldg(cs + 16 * (i >> 2) + 8 * ((i >> 1) & 1) + 2 * t + (i & 1));
              xk[i] = round_bf16(plane == 0 ? kv_rot_lo(xk[i], other[i], c) : kv_rot_hi(other[i], xk[i], c));
            }
          }
        }
      }
      pair[0][s] = kv_quantise(xk, word[0][s]);
      pair[1][s] = kv_quantise(xv, word[1][s]);
    }
    uint32_t kw[4], vw[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      kw[j] = word[0][0][j] | word[0][1][j] << 8;
      vw[j] = movmatrix_trans(word[1][0][j] | word[1][1][j] << 8);
    }
    uint8_t* tile = p.kv.pages + p.kv.tile_at(gr.page, head, gr.tile) + plane * kKvTileBytes;
    const uint32_t rows = __ballot_sync(0xffffffffu, live[0]), rows8 = __ballot_sync(0xffffffffu, live[1]);   // bit 4 g: token g
    if ((rows & rows8) == 0xffffffffu) {
      reinterpret_cast<uint4*>(tile)[lane] = make_uint4(kw[0], kw[1], kw[2], kw[3]);
      reinterpret_cast<uint4*>(tile + 512)[lane] = make_uint4(vw[0], vw[1], vw[2], vw[3]);
      if (t == 0) reinterpret_cast<uint4*>(tile + kKvPairs)[g] = make_uint4(pair[0][0], pair[0][1], pair[1][0], pair[1][1]);
      continue;
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (live[s]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          tile[16 * lane + 4 * j + s] = (uint8_t)(kw[j] >> (8 * s));
          tile[16 * lane + 4 * j + 2 + s] = (uint8_t)(kw[j] >> (16 + 8 * s));
        }
        if (t == 0) {
          uint32_t* pr = reinterpret_cast<uint32_t*>(tile + kKvPairs) + 4 * g + s;
          pr[0] = pair[0][s];
          pr[2] = pair[1][s];
        }
      }
      const uint32_t r = s == 0 ? rows : rows8;
#pragma unroll
      for (int c = 0; c < 2; ++c)      // value bytes: this lane's tokens 2 t + c (+ 8)
        if (r >> (4 * (2 * t + c)) & 1u) {
#pragma unroll
          for (int j = 0; j < 4; ++j) tile[512 + 16 * lane + 4 * j + 2 * c + s] = (uint8_t)(vw[j] >> (16 * c + 8 * s));
        }
    }
  }
}

// The rows of a group back as bf16(zero + scale code); rows without a slot are zeros.
template <int D>
__global__ void __launch_bounds__(32 * kKvStoreWarps)
kv_read_kernel(const KvStoreParams p) {
  pdl_begin();
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int hp = blockIdx.y * kKvStoreWarps + (threadIdx.x >> 5);
  if (hp >= p.kv.H * (D / 64)) return;
  const int head = hp / (D / 64), plane = hp % (D / 64);
  const int first = blockIdx.x * p.window;
  const bool mine = lane < p.window && first + lane < p.T;
  uint32_t none = __ballot_sync(0xffffffffu, mine && !kv_slot_ok(p, p.slot[mine ? first + lane : 0]));
  for (; none; none &= none - 1) {
    const int row = first + __ffs(none) - 1;
    reinterpret_cast<uint32_t*>(p.k_out + (long long)row * p.k_stride + head * D + 64 * plane)[lane] = 0u;
    reinterpret_cast<uint32_t*>(p.v_out + (long long)row * p.v_stride + head * D + 64 * plane)[lane] = 0u;
  }
  uint32_t starts = __ballot_sync(0xffffffffu, mine && kv_group_start(p, mine ? first + lane : 0));
  while (starts) {
    const KvGroup gr = kv_group(p, first + __ffs(starts) - 1, lane);
    starts &= starts - 1;
    const uint8_t* tile = p.kv.pages + p.kv.tile_at(gr.page, head, gr.tile) + plane * kKvTileBytes;
    const uint4 k4 = reinterpret_cast<const uint4*>(tile)[lane], v4 = reinterpret_cast<const uint4*>(tile + 512)[lane];
    const uint4 pr = reinterpret_cast<const uint4*>(tile + kKvPairs)[g];
    const uint32_t kw[4] = {k4.x, k4.y, k4.z, k4.w};
    const uint32_t vw[4] = {movmatrix_trans(v4.x), movmatrix_trans(v4.y), movmatrix_trans(v4.z), movmatrix_trans(v4.w)};
    const uint32_t pk[2] = {pr.x, pr.y}, pv[2] = {pr.z, pr.w};
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (g + 8 * s < gr.i0 || g + 8 * s >= gr.i0 + gr.n) continue;
      const long long row = gr.t0 + g + 8 * s - gr.i0;
      uint32_t* ko = reinterpret_cast<uint32_t*>(p.k_out + row * p.k_stride + head * D + 64 * plane) + t;
      uint32_t* vo = reinterpret_cast<uint32_t*>(p.v_out + row * p.v_stride + head * D + 64 * plane) + t;
      const float ks = kv_scale(pk[s]), kz = kv_zero(pk[s]), vs = kv_scale(pv[s]), vz = kv_zero(pv[s]);
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int sh = 8 * s + 4 * h;
          ko[8 * j + 4 * h] = pack_bf16(fmaf((float)(kw[j] >> sh & 15u), ks, kz), fmaf((float)(kw[j] >> (sh + 16) & 15u), ks, kz));
          vo[8 * j + 4 * h] = pack_bf16(fmaf((float)(vw[j] >> sh & 15u), vs, vz), fmaf((float)(vw[j] >> (sh + 16) & 15u), vs, vz));
        }
    }
  }
}

// Rows a CTA looks for groups in: one while warps are few, so that every token has its own; sixteen beyond, where groups are whole
// tiles and most of the warps of single rows would find nothing.
static int kv_window(int T) { return T <= 2048 ? 1 : 16; }

template <class Fn>
static moin_status kv_store_launch(Fn* fn64, Fn* fn128, KvStoreParams& p, int head_dim, cudaStream_t s) {
  p.window = kv_window(p.T);
  const dim3 grid((unsigned)((p.T + p.window - 1) / p.window), (unsigned)((p.kv.H * p.kv.planes + kKvStoreWarps - 1) / kKvStoreWarps));
  ProfScope prof(MOIN_K_KV_STORE, 1, s);
  return record_cuda(launch_pdl(head_dim == 64 ? fn64 : fn128, grid, 32 * kKvStoreWarps, 0, s, p));
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
  return kv_store_launch(kv_append_kernel<64>, kv_append_kernel<128>, p, kv->head_dim, (cudaStream_t)stream);
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
  return kv_store_launch(kv_read_kernel<64>, kv_read_kernel<128>, p, kv->head_dim, (cudaStream_t)stream);
}
