// The 4-bit key/value cache: layout and the small device functions its kernels share.
//
// A page holds page_tokens tokens of every kv head: [kv head][page_tokens / 16 tiles][head_dim / 64 planes][1152 bytes].
// A tile's 64 channels of 16 tokens are 512 bytes of key codes, 512 of value codes and 128 of (scale, zero) pairs.  The
// codes lie in the order in which a warp needs them as the A operand of an m16n8k16 product, keys as [token x channel],
// values as [channel x token]: lane 4 g + t owns 16 bytes, one 32-bit word for each of the four steps of 16 channels, and
// a 16-byte load of the cache is four whole fragments, with neither shuffle nor shared memory in between.  In word j
//   keys    nibble 0, 1 of the low half: token g,     channels 16 j + 2 t, 8 more;  of the high half: one channel on
//           nibble 2, 3                  token g + 8, the same
//   values  nibble 0, 1 of the low half: channels 16 j + g, 8 more, of token 2 t;   of the high half: of token 2 t + 1
//           nibble 2, 3                  the same of tokens 8 on
// so a byte belongs to one token (tokens are stored by byte stores that do not touch their neighbours), and the words of
// the values are those of the keys' order with the 8 x 8 blocks of 16-bit units transposed (one movmatrix a word).
// Pairs: 16 bytes for each g: key of token g, of token g + 8, value of g, of g + 8; scale in a pair's low half.
#pragma once
#include "common.cuh"

namespace moin {

constexpr int kKvTile = 16;            // tokens
constexpr int kKvTileBytes = 1152;
constexpr int kKvPairs = 1024;         // offset of the pairs in a tile

__device__ __forceinline__ float kv_scale(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float kv_zero(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t v) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
  return d;
}

// Rotation of a pair (i, i + head_dim / 2): products and their difference rounded one by one, so that the stored codes are
// what the formula gives in any implementation of it (a fused multiply-add can move a rotated key by a bit).
__device__ __forceinline__ float kv_rot_lo(float a, float b, float2 cs) { return __fsub_rn(__fmul_rn(a, cs.x), __fmul_rn(b, cs.y)); }
__device__ __forceinline__ float kv_rot_hi(float a, float b, float2 cs) { return __fadd_rn(__fmul_rn(b, cs.x), __fmul_rn(a, cs.y)); }
__device__ __forceinline__ float round_bf16(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

struct KvView {          // a cache, by value
  uint8_t* pages;
  int n_pages, page_tokens, H, planes;
  __host__ __device__ size_t tile_at(int page, int head, int tile) const {
    return ((((size_t)page * H + head) * (page_tokens / kKvTile)) + tile) * (size_t)planes * kKvTileBytes;
  }
};

inline moin_status kv_view(const moin_kv* kv, KvView* out) {
  if (!kv || !kv->pages || kv->n_pages < 1 || kv->n_kv_heads < 1) return MOIN_ERR_INVALID_ARG;
  if (kv->head_dim != 64 && kv->head_dim != 128) return MOIN_ERR_BAD_SHAPE;
  if (kv->page_tokens != 16 && kv->page_tokens != 32 && kv->page_tokens != 64 && kv->page_tokens != 128) return MOIN_ERR_BAD_SHAPE;
  if (kv->n_kv_heads > 16384 || (long long)kv->n_pages * kv->page_tokens > 0x7FFFFFFFll) return MOIN_ERR_BAD_SHAPE;   // slots are 32-bit
  if (!aligned16(kv->pages)) return MOIN_ERR_MISALIGNED;
  *out = {reinterpret_cast<uint8_t*>(kv->pages), kv->n_pages, kv->page_tokens, kv->n_kv_heads, kv->head_dim / 64};
  return MOIN_OK;
}

// A row length between two tokens of a tensor [T, heads, head_dim] whose heads lie side by side.
inline bool kv_stride_ok(long long stride, int heads, int head_dim) {
  return stride >= (long long)heads * head_dim && (stride % 8) == 0;
}

// Attention of long chunks (kv_chunk.cu, head_dim 64, positive scale): workspace, launch.  What `workers` CTAs leave of the items that they
// share is for kv_join_kernel.
struct KvPieces { float* part; int4* desc; int workers; long long items; };
size_t kv_chunk_bytes(int R, int T, int max_kv, int n_heads, int H);
moin_status launch_kv_chunk(HostState* hs, const KvView& kv, const int* table, const int* rows, const int* cu_q, const int* kv_len, int n_rows,
                            int max_pages, int R, int T, int max_q, int max_kv, int n_heads, const __nv_bfloat16* q, long long q_stride,
                            __nv_bfloat16* out, long long out_stride, const float2* rope, float scale_log2, void* workspace, KvPieces* pieces, cudaStream_t s);

}  // namespace moin
