// Attention of long chunks over the 4-bit cache on tcgen05 (head_dim 64): the products of prompts, where kv_attention.cu's warp
// MMAs, made for a few rows, are bound by their instructions.
//
// kv_dense_kernel lays the requests' keys and values out as fp16 [request, position, kv head, 64] in the workspace, each tile of 64
// tokens times a power of two that brings its largest value to 2^13 .. 2^14 (a value is off by 2^-11 of itself, or by 2^-38 of the
// tile's largest) - or, in a tile whose tokens are unlike (their largest values differ by more than 2^12), each token times its own,
// so that no token's precision depends on another, which a row may not even see -, and the queries as fp16 rows (rotated; times a power of two per row: exact) in the order the tiles take
// them, [kv head, token, head of the group]: a tile of 128 rows is one box whatever the group is.  What is stored as NaN is laid
// out as 0 and noted in the tile's mask; a row that sees such a token becomes NaN, no other row meets it.
//
// kv_chunk_kernel: work items are (request, kv head, 128 rows); persistent CTAs, two per SM, take equal shares of their key tiles, each with
// two streams: even and odd tiles, each stream with its own scores, maximum, sum and accumulator, which meet at the item's end.
//   warps 0, 1  a stream's loads and MMAs, in turn: K and V tiles [64 keys x 64 dims] into two slots each by TMA (warp 0 the Q tiles
//               too, into two buffers), S = Q K^T in two halves of 32 keys, O += P V
//   warps 2-5   stream 0, warps 6-9 stream 1: a thread per row
// A stream's chain is weights - product - scores, since P lies where the lower 32 keys' scores were; those of the upper 32 are
// computed while the product is, and their weights while the lower ones are.
// With the tile's factors (K: 2^a, V: 2^b) a weight is w = 2^(s 2^a + b - m), at most 2^15 (m lags), P = fp16(w), and the row's sum takes
// w 2^-b in fp32.  Weights are taken against the maximum that stands, and the tile's own maximum found beside them; where that is
// 2^15 above, the maximum moves to leave 2^5 and the tile is taken again (with 2^10 left that is more often: 17 us of the case below).
// A weight below 2^-14 is off by 2^-25 at most: 2^-30 of the row's largest, so that 2^19 keys stay within 2^-11 of the sum.
// Tensor memory: S_h / P_h at columns 64 h, O_h at 128 + 64 h.  Every mbarrier wait is bounded; on expiry the CTA raises the status
// flag, drains and returns.
// 4 requests of 512 new tokens behind 830 to 5900, 32 heads on 4: about 109 us for 52 GFLOP, bound by the instructions and exponentials of the
// weights (a warp's tile 1.3 us, four warps on a scheduler: issue slots 48 % busy, exponentials 52 %, tensor cores 23 %) and by the chain.  One warp that issued both streams' MMAs took 900
// cycles a round, and with the maximum found first, whole items per CTA and all scores behind the product it was 125 us.
#include <cuda.h>
#include <float.h>

#include "kv.cuh"
#include "ptx.cuh"
#include "tc_gemm.cuh"

namespace moin {

constexpr int kChThreads = 320;
constexpr int kChKeys = 64, kChRows = 128;
constexpr int kChQ = kChRows * 64 * 2, kChKV = kChKeys * 64 * 2, kChRing = 4;
constexpr int kChMerge = 4096;               // (maximum, sum) of every row by stream, for two items
constexpr int kChSmem = 2 * kChQ + 2 * kChRing * kChKV + 1024 /*align*/ + 256 /*barriers*/ + kChMerge;
constexpr int kChMaxWorkers = 320;           // CTAs
constexpr int kChItemCost = 2;               // pairs of tiles that beginning and ending an item costs
constexpr int kChLeast = 4;                  // of a share, at least
constexpr int kChPitch = 64 + 4;             // floats of a row of a piece: sums, maximum, sum of weights
constexpr int kChTmemCols = 256;
constexpr float kChTop = 5.f, kChMost = 15.f;   // log2 of the largest weight after a move of the maximum, and at all
// The tensor core's accumulator truncates: over a chain of n keys a sum loses about n 2^-28 of itself, always the same way (measured:
// behind 2^19 keys, 2^18 a stream, 2^-9.9 of every value, where rounding to bf16 is 2^-9.3 in the mean square).  Behind kChFlush tiles
// of a stream the sum goes into memory, by fp32 additions, and a new one begins.
constexpr int kChFlush = 512;                   // a power of two
constexpr int kChKeep = 17;                     // float4 of a row there: sums, the maximum that they are taken against
constexpr float kChHuge = 0x1p20f;              // scores (powers of two) from which a step of fp32 is 2^-4 and more

constexpr uint32_t kChIdesc = (1u << 4) | ((uint32_t)(64 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);   // D fp32, A and B fp16, 128 x 64
constexpr uint32_t kChIdescHalf = (1u << 4) | ((uint32_t)(32 >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);   // D 128 x 32
constexpr uint64_t kChHalf = (32 * 128) >> 4;            // 32 keys further on
constexpr uint32_t kChIdescPV = kChIdesc | (1u << 16);   // B with its rows along the output dimension
constexpr uint64_t kChVStep = 2048 >> 4;                 // 16 keys further on

struct ChunkParams {
  KvView kv;
  const int *table, *rows, *cu_q, *kv_len;
  int n_rows, max_pages, R, T, max_q, max_kv, G, n_heads, n_blk, tiles;   // row blocks of the longest request, tiles of 64 of the longest
  uint32_t inv_g;
  const __nv_bfloat16* q;
  __nv_bfloat16* out;
  long long q_stride, out_stride;
  const float2* rope;
  float scale_log2;
  __half *kd, *vd, *qd;     // dense keys, values [R tiles 64, H 64]; queries [H, T G, 64]
  float* q_fac;             // [H, T G] 1 / (what the row was multiplied with)
  uint4* info;              // [R, H, tiles]: scale log2(e) 2^a, b (fp32; low bits: hidden groups, unlike tokens), mask of NaN tokens
  float2* tok;              // [R, H, tiles, 64], of tiles of unlike tokens: (scale log2(e) 2^a, b) of every token
  int dense_blocks, workers;
  int4* share;              // [worker]: (row block of a request, head, what of that item is passed) where its share begins, its size
  float* part;              // [worker][2][128][kChPitch]: pieces of items, in slot 1 of one that begins here without ending, else in slot 0
  float4* keep;             // [worker][stream][kChKeep][128]: sums of the tiles before (kChFlush)
  int4* desc;               // [worker][2]: the item that it begins without ending it, as kv_join_kernel takes it
  DeviceStatus* status;
};

__device__ __forceinline__ int ch_div_g(const ChunkParams& p, int row) { return p.G == 1 ? row : (int)__umulhi((uint32_t)row, p.inv_g); }
struct ChReq { int t0, q_len, kv_len, row; };
__device__ __forceinline__ ChReq ch_request(const ChunkParams& p, int req) {   // as kv_item of kv_attention.cu
  ChReq r;
  r.t0 = min(max(p.cu_q[req], 0), p.T);
  r.q_len = min(max(p.cu_q[req + 1], r.t0), p.T) - r.t0;
  r.kv_len = p.kv_len[req];
  r.row = p.rows ? p.rows[req] : req;
  if (r.kv_len < 0 || r.kv_len > p.max_kv || r.q_len > p.max_q || r.row < 0 || r.row >= p.n_rows) r.kv_len = 0;
  r.q_len = min(r.q_len, p.max_q);
  return r;
}

// Work is measured in pairs of key tiles, and kChItemCost of them to begin and end an item: items (row block of a request, kv head) one behind
// the other, cut into equal shares, one per CTA,
// so that a long request is no longer chain than any other and few items fill the GPU.  An item that begins or ends inside another share is left as
// a piece (its sums, maximum and sum of weights) that kv_join_kernel adds up.
struct ChItem { int req, head, row0, t0, n_rows, past, first_pos, last_pos, n_pairs, j0, n; bool whole; };   // n tiles from j0
__device__ __forceinline__ ChItem ch_item(const ChunkParams& p, int block, int head) {
  ChItem it;
  it.req = block / p.n_blk;
  it.head = head;
  it.row0 = (block - it.req * p.n_blk) * kChRows;
  const ChReq r = ch_request(p, it.req);
  it.t0 = r.t0;
  it.n_rows = r.q_len * p.G;
  it.past = r.kv_len - r.q_len;
  it.first_pos = it.past + ch_div_g(p, it.row0);
  it.last_pos = it.row0 < it.n_rows ? it.past + ch_div_g(p, min(it.row0 + kChRows, it.n_rows) - 1) : -1;
  it.n = it.last_pos < 0 || r.kv_len == 0 ? 0 : it.last_pos / kChKeys + 1;
  it.n_pairs = (it.n + 1) >> 1;
  it.j0 = 0;
  return it;
}
// What to look at behind a block that has nothing to do: the blocks behind a request's last rows are passed at once.
__device__ __forceinline__ int ch_behind(const ChunkParams& p, const ChItem& it, int block) {
  return it.n == 0 && it.row0 >= it.n_rows ? (it.req + 1) * p.n_blk : block + 1;
}
__device__ __forceinline__ int ch_cost(const ChItem& it) { return it.n == 0 ? 0 : it.n_pairs + kChItemCost; }
struct ChWalk {   // over the items of a CTA's share
  int block, head, at, left;   // what of the item is passed, what of the share is left
  __device__ __forceinline__ explicit ChWalk(const int4& share) : block(share.x), head(share.y), at(share.z), left(share.w) {}
  __device__ __forceinline__ bool next(const ChunkParams& p, ChItem& it) {
    while (left > 0 && block < p.R * p.n_blk) {
      it = ch_item(p, block, head);
      if (it.n == 0) {
        block = ch_behind(p, it, block);
        continue;
      }
      const int to = min(ch_cost(it), at + left), pair = max(at - kChItemCost, 0), end = to - kChItemCost;
      left -= to - at;
      at = 0;
      if (++head == p.kv.H) {
        head = 0;
        ++block;
      }
      if (end <= pair) continue;   // (the share ends in what it costs to begin: the item is the next CTA's)
      it.whole = pair == 0 && end == it.n_pairs;
      it.j0 = 2 * pair;
      it.n = min(it.n, 2 * end) - it.j0;
      return true;
    }
    return false;
  }
};
struct ChCursor {   // over the tiles of one stream
  ChWalk walk;
  ChItem it;
  int j = 0;             // in the item
  uint32_t item = ~0u;   // items so far, this one not counted
  bool have = true;
  __device__ __forceinline__ explicit ChCursor(const int4& share) : walk(share) { it.n = 0; }
  __device__ __forceinline__ void next(const ChunkParams& p, int stream) {   // to an item's first tile, if the stream has one there
    have = walk.next(p, it);
    ++item;
    j = stream;
  }
};
// Where the shares begin, by one block beside those that lay out: sums over runs of row blocks, then a search for each share.
__device__ __forceinline__ void ch_shares(const ChunkParams& p) {
  __shared__ long long s_before[129];   // cost of the runs before, of one head
  __shared__ long long s_warp[4];
  const int blocks = p.R * p.n_blk, run = (blocks + 127) / 128, tid = threadIdx.x, lane = tid & 31;
  const long long first = (long long)tid * run, last = first + run < blocks ? first + run : blocks;
  long long sum = 0;
  for (long long b = first; b < last;) {
    const ChItem it = ch_item(p, (int)b, 0);
    sum += ch_cost(it);
    b = ch_behind(p, it, (int)b);
  }
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, sum, o);
    if (lane >= o) sum += v;
  }
  if (lane == 31) s_warp[tid >> 5] = sum;
  __syncthreads();
  for (int w = 0; w < tid >> 5; ++w) sum += s_warp[w];
  s_before[tid + 1] = sum;
  if (tid == 0) s_before[0] = 0;
  __syncthreads();
  const long long H = p.kv.H, all = s_before[128] * H;
  long long share = (all + p.workers - 1) / p.workers;
  if (share < kChLeast) share = kChLeast;
  for (int k = tid; k <= p.workers; k += 128) {
    const long long at = k * share;
    int4 begin = make_int4(0, 0, 0, 0), open = make_int4(0, 0, 0, 0);
    int open_rows = 0;
    if (at < all) {
      int lo = 0, hi = 127;   // the last run that begins at or before it and is not empty
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (s_before[mid + 1] * H > at) hi = mid; else lo = mid + 1;
      }
      long long before = s_before[lo] * H, b = (long long)lo * run;
      ChItem it = ch_item(p, (int)b, 0);
      while (before + ch_cost(it) * H <= at) {   // (ends inside the run: its sum is above `at`)
        before += ch_cost(it) * H;
        b = ch_behind(p, it, (int)b);
        it = ch_item(p, (int)b, 0);
      }
      const uint32_t cost = (uint32_t)ch_cost(it), off = (uint32_t)(at - before), head = off / cost;
      const int in = (int)(off - head * cost);
      begin = make_int4((int)b, (int)head, in, (int)(all - at < share ? all - at : share));
      if (in > kChItemCost && in - share <= kChItemCost) {   // begun by the CTA before
        open = make_int4((int)head, it.row0, it.t0, (int)((cost - in + share - 1) / share));
        open_rows = it.n_rows;
      }
    }
    if (k < p.workers) p.share[k] = begin;
    if (k > 0) {
      p.desc[2 * (k - 1)] = open;
      p.desc[2 * (k - 1) + 1] = make_int4(open_rows, 0, 0, 0);
    }
  }
}

// Block 0: the shares.  The dense_blocks behind it: 64 tokens of a request and kv head, a warp per 16 of them.  The others: the queries of a
// token; for one that sees nothing, zeros are its result.
// Bound by the traffic of what they write; small beside the products.
constexpr uint32_t kChUnlike = 0x10u, kChNan = 0x20u, kChFlags = 0x3Fu;   // in the low bits of b, above those of hidden groups
constexpr int kChRange = 12;            // powers of two between the tokens of a tile that are alike
constexpr int kDensePitch = 36;   // words of a row in shared memory: neither side meets a bank twice
__global__ void __launch_bounds__(128)
kv_dense_kernel(const ChunkParams p) {
  __shared__ __align__(16) uint32_t s_rows[4][kKvTile * kDensePitch];
  __shared__ float s_max[4][2], s_min[4][2];
  __shared__ uint32_t s_bad[4];
  pdl_begin();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  if (blockIdx.x == 0) {
    ch_shares(p);
    return;
  }
  if ((int)blockIdx.x > p.dense_blocks) {
    const int tok = (int)blockIdx.x - 1 - p.dense_blocks;
    // the request of the token: the first one that ends behind it
    int lo = 0, hi = p.R;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (p.cu_q[mid + 1] > tok) hi = mid; else lo = mid + 1;
    }
    int pos = -1;
    bool blind = false;
    if (lo < p.R) {
      const ChReq r = ch_request(p, lo);
      if (tok >= r.t0 && tok < r.t0 + r.q_len) pos = r.kv_len - r.q_len + tok - r.t0;
      blind = tok >= r.t0 && tok < r.t0 + r.q_len && (pos < 0 || r.kv_len == 0);
    }
    if (blind) {
      for (int i = threadIdx.x; i < p.n_heads * 8; i += 128)
        *reinterpret_cast<uint4*>(p.out + (long long)tok * p.out_stride + 8 * i) = make_uint4(0u, 0u, 0u, 0u);
    }
    // two heads at a time, a lane the pairs (c, c + 32), (c + 1, c + 33) of one
    const int c = 2 * (lane & 15);
    float4 cs = make_float4(1.f, 0.f, 1.f, 0.f);
    if (p.rope != nullptr && pos >= 0) cs = __ldg(reinterpret_cast<const float4*>(p.rope + (size_t)pos * 32 + c));
#pragma unroll 2
    for (int h0 = 2 * warp; h0 < p.n_heads; h0 += 8) {
      const int h = h0 + (lane >> 4);
      const bool there = h < p.n_heads;
      uint32_t a = 0u, b = 0u;
      if (pos >= 0 && there) {
        const __nv_bfloat16* src = p.q + (long long)tok * p.q_stride + (long long)h * 64 + c;
        a = __ldg(reinterpret_cast<const uint32_t*>(src));
        b = __ldg(reinterpret_cast<const uint32_t*>(src + 32));
      }
      float x0 = bf16_lo(a), x1 = bf16_hi(a), y0 = bf16_lo(b), y1 = bf16_hi(b);
      if (p.rope != nullptr) {
        const float2 c0 = make_float2(cs.x, cs.y), c1 = make_float2(cs.z, cs.w);
        const float u0 = round_bf16(kv_rot_lo(x0, y0, c0)), u1 = round_bf16(kv_rot_lo(x1, y1, c1));
        y0 = round_bf16(kv_rot_hi(x0, y0, c0));
        y1 = round_bf16(kv_rot_hi(x1, y1, c1));
        x0 = u0;
        x1 = u1;
      }
      float top = fmaxf(fmaxf(fabsf(x0), fabsf(x1)), fmaxf(fabsf(y0), fabsf(y1)));
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      // 2^(9 - exponent of the largest element); a row of zeros, subnormals or infinities stays as it is
      const int e = (int)(__float_as_uint(top) >> 23) - 127;
      const float f = (e > -118 && e < 128) ? __uint_as_float((uint32_t)(9 - e + 127) << 23) : 1.f;
      if (!there) continue;
      const int kvh = h / p.G;
      const long long row = (long long)kvh * p.T * p.G + (long long)tok * p.G + (h - kvh * p.G);
      const __half2 lo2 = __floats2half2_rn(x0 * f, x1 * f), hi2 = __floats2half2_rn(y0 * f, y1 * f);
      *reinterpret_cast<__half2*>(p.qd + row * 64 + c) = lo2;
      *reinterpret_cast<__half2*>(p.qd + row * 64 + c + 32) = hi2;
      if ((lane & 15) == 0) p.q_fac[row] = 1.f / f;
    }
    return;
  }
  const int at_block = (int)blockIdx.x - 1, tile = at_block % p.tiles, rh = at_block / p.tiles, head = rh % p.kv.H, req = rh / p.kv.H;
  const ChReq r = ch_request(p, req);
  if (tile * kChKeys >= r.kv_len || r.q_len == 0) return;
  const int first = tile * kChKeys + warp * kKvTile;   // this warp's tokens
  uint4 k4 = make_uint4(0u, 0u, 0u, 0u), v4 = k4, pr = k4;
  uint32_t gone = 0xFFFFu;   // of its tokens: not there
  if (first < r.kv_len) {
    const int page = p.table[(size_t)r.row * p.max_pages + first / p.kv.page_tokens];
    if (page >= 0 && page < p.kv.n_pages) {
      const uint8_t* at = p.kv.pages + p.kv.tile_at(page, head, first % p.kv.page_tokens / kKvTile);
      k4 = *reinterpret_cast<const uint4*>(at + 16 * lane);
      v4 = *reinterpret_cast<const uint4*>(at + 512 + 16 * lane);
      pr = *reinterpret_cast<const uint4*>(at + kKvPairs + 16 * g);
      gone = r.kv_len - first >= kKvTile ? 0u : 0xFFFFu & ~((1u << (r.kv_len - first)) - 1u);
    }
  }
  const uint32_t kw[4] = {k4.x, k4.y, k4.z, k4.w};
  const uint32_t vw[4] = {movmatrix_trans(v4.x), movmatrix_trans(v4.y), movmatrix_trans(v4.z), movmatrix_trans(v4.w)};
  const uint32_t pk[2] = {pr.x, pr.y}, pv[2] = {pr.z, pr.w};
  // A row's largest value is at one of its ends: its pair tells, and whether it is NaN.
  float tok[2][2], top[2] = {0.f, 0.f}, low[2] = {INFINITY, INFINITY};   // largest values: of the tokens, of the tile, of its least token
  uint32_t bad = 0;
  bool drop[2];                                                          // token g, g + 8: laid out as zeros
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    const bool out = gone >> (g + 8 * s) & 1u;
    float end[2][2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const uint32_t pair = c == 0 ? pk[s] : pv[s];
      end[c][0] = fabsf(kv_zero(pair));
      end[c][1] = fabsf(fmaf(15.f, kv_scale(pair), kv_zero(pair)));
    }
    const bool nan = !(end[0][0] < INFINITY && end[0][1] < INFINITY && end[1][0] < INFINITY && end[1][1] < INFINITY);
    if (nan && !out) bad |= 1u << (g + 8 * s);
    drop[s] = nan || out;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      tok[c][s] = drop[s] ? 0.f : fmaxf(end[c][0], end[c][1]);
      top[c] = fmaxf(top[c], tok[c][s]);
      if (tok[c][s] > 0.f) low[c] = fminf(low[c], tok[c][s]);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
    top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], o));
    low[0] = fminf(low[0], __shfl_xor_sync(0xffffffffu, low[0], o));
    low[1] = fminf(low[1], __shfl_xor_sync(0xffffffffu, low[1], o));
    bad |= __shfl_xor_sync(0xffffffffu, bad, o);
  }
  // tokens of a page that is not there are hidden, not NaN: noted apart, in the upper half
  const bool hidden = first < r.kv_len && (gone & 1u);
  if (lane == 0) {
    s_max[warp][0] = top[0];
    s_max[warp][1] = top[1];
    s_min[warp][0] = low[0];
    s_min[warp][1] = low[1];
    s_bad[warp] = bad | (hidden ? 0x10000u : 0u);
  }
  __syncthreads();
  auto power = [](float m) { return max((int)(__float_as_uint(m) >> 23) - 127 - 13, -64); };   // 2^it times 2^13 .. 2^14 is the largest value
  auto two_to = [](int e) { return __uint_as_float((uint32_t)(127 + e) << 23); };
  float f[2][2];   // [key, value][token g, g + 8]
  int e[2], et[2][2];
  bool unlike = false;
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const float m = fmaxf(fmaxf(s_max[0][c], s_max[1][c]), fmaxf(s_max[2][c], s_max[3][c]));
    const float l = fminf(fminf(s_min[0][c], s_min[1][c]), fminf(s_min[2][c], s_min[3][c]));
    e[c] = power(m);
    unlike = unlike || (l < INFINITY && e[c] - power(l) > kChRange);
  }
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      et[c][s] = unlike ? power(tok[c][s]) : e[c];
      f[c][s] = two_to(-et[c][s]);
    }
  const size_t at_tile = ((size_t)req * p.kv.H + head) * p.tiles + tile;
  if (unlike && t == 0) {
#pragma unroll
    for (int s = 0; s < 2; ++s) p.tok[at_tile * kChKeys + warp * kKvTile + g + 8 * s] = make_float2(p.scale_log2 * two_to(et[0][s]), (float)et[1][s]);
  }
  if (threadIdx.x == 0) {
    uint32_t hide = 0;
    for (int w = 0; w < 4; ++w) hide |= (s_bad[w] >> 16) << w;
    const uint32_t lo = (s_bad[0] & 0xFFFFu) | s_bad[1] << 16, hi = (s_bad[2] & 0xFFFFu) | s_bad[3] << 16;
    // b is a whole number of at most 114: its low mantissa bits are free
    p.info[at_tile] = make_uint4(__float_as_uint(p.scale_log2 * two_to(e[0])), __float_as_uint((float)e[1]) | hide | (unlike ? kChUnlike : 0u) | ((lo | hi) != 0u ? kChNan : 0u), lo, hi);
  }
  uint32_t* stage = s_rows[warp];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      // scale and zero times a power of two keep their 8 bits in fp16 (a step is above 2^-12 of its row's zero, a row above 2^-12 of
      // its tile); a code becomes an fp16 by its bits (1024 + code, less 1024), a value by one fused multiply-add
      const uint32_t pair = c == 0 ? pk[s] : pv[s];
      const float by = drop[s] ? 0.f : f[c][s];
      const __half2 scale2 = __float2half2_rn(drop[s] ? 0.f : kv_scale(pair) * by), zero2 = __float2half2_rn(drop[s] ? 0.f : kv_zero(pair) * by);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t w = c == 0 ? kw[i >> 1] : vw[i >> 1], bits = (w >> (8 * s + 4 * (i & 1)) & 0x000F000Fu) | 0x64006400u;
        const __half2 code = __hsub2(*reinterpret_cast<const __half2*>(&bits), __float2half2_rn(1024.f)), v = __hfma2(code, scale2, zero2);
        stage[(g + 8 * s) * kDensePitch + 4 * i + t] = *reinterpret_cast<const uint32_t*>(&v);
      }
    }
    __syncwarp();
    __half* dst = (c == 0 ? p.kd : p.vd) + (((size_t)req * p.tiles * kChKeys + first) * p.kv.H + head) * 64;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int row = 4 * k + (lane >> 3);
      *reinterpret_cast<uint4*>(dst + (size_t)row * p.kv.H * 64 + 8 * (lane & 7)) = *reinterpret_cast<const uint4*>(stage + row * kDensePitch + 4 * (lane & 7));
    }
    __syncwarp();
  }
}

__device__ __forceinline__ float ch_exp2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float ch_rescale(float l, float d) {   // l 2^d, where 2^d alone may be too small (kv_attention.cu)
  const float f = ch_exp2(0.5f * d);
  return l * f * f;
}

__global__ void __launch_bounds__(kChThreads, 2)
kv_chunk_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const ChunkParams p) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - raw);
  const uint32_t sQ = base, sK = base + 2 * kChQ, sV = sK + kChRing * kChKV, bars = sV + kChRing * kChKV;
  uint8_t* bar_ptr = base_ptr + (bars - base);
  const uint32_t kfull = bars, vfull = bars + 32, sready = bars + 64, supper = bars + 80, pready = bars + 96, pvdone = bars + 112,
                 qfull = bars + 128, qfree = bars + 144, ofree = bars + 160;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_ptr + 168);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bar_ptr + 172);
  volatile int* sm_fail = reinterpret_cast<volatile int*>(bar_ptr + 176);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kChRing; ++i) {
      mbar_init(kfull + 8 * i, 1);
      mbar_init(vfull + 8 * i, 1);
    }
    for (int h = 0; h < 2; ++h) {
      mbar_init(sready + 8 * h, 1); mbar_init(supper + 8 * h, 1); mbar_init(pready + 8 * h, 128); mbar_init(pvdone + 8 * h, 1);
      mbar_init(qfull + 8 * h, 1); mbar_init(qfree + 8 * h, 2);
    }
    mbar_init(ofree, 256);
    *abort_flag = 0;
    sm_fail[0] = sm_fail[1] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    tmem_alloc(smem_u32(tmem_slot), kChTmemCols);
    tmem_relinquish();
  }
  pdl_begin();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const int4 share = p.share[blockIdx.x];

  if (warp < 2) {
    // ------------------------------------------------------------------ loads and MMAs of a stream, one after the other: the whole
    // warp waits, one lane issues.  Tile i of the stream lies in slot i & 1; it is replaced when its product is complete.
    const int h = __shfl_sync(0xffffffffu, warp, 0);   // (known to be the warp's: descriptors stay in uniform registers)
    const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
    const bool leader = elect_one();
    const uint32_t sk = sK + 2 * h * kChKV, sv = sV + 2 * h * kChKV, kf = kfull + 16 * h, vf = vfull + 16 * h;
    bool ok = true;
    auto wait = [&](uint32_t bar, uint32_t parity, int site) { ok = ok && mbar_wait_warp(bar, parity, abort_flag, p.status, site); };
    ChCursor ld(share), at(share);   // the next tile to load; the one whose scores were issued last
    uint32_t i = 0, n_ld = 0;
    auto load = [&] {
      if (!ld.have) return;
      if (h == 0 && ld.j == 0) {     // an item begins: its queries, for both streams
        const uint32_t b = ld.item & 1u;
        wait(qfree + 8 * b, ((ld.item >> 1) & 1u) ^ 1u, 61);
        if (ok && leader) {
          mbar_expect_tx(qfull + 8 * b, kChQ);
          tma_load_2d(sQ + b * kChQ, &tmQ, qfull + 8 * b, 0, ld.it.head * p.T * p.G + ld.it.t0 * p.G + ld.it.row0);
        }
      }
      const uint32_t s = n_ld & 1u;
      const int row = (ld.it.req * p.tiles + ld.it.j0 + ld.j) * kChKeys;
      if (ok && leader) {
        mbar_expect_tx(kf + 8 * s, kChKV);
        tma_load_2d(sk + s * kChKV, &tmK, kf + 8 * s, ld.it.head * 64, row);
        mbar_expect_tx(vf + 8 * s, kChKV);
        tma_load_2d(sv + s * kChKV, &tmV, vf + 8 * s, ld.it.head * 64, row);
      }
      ++n_ld;
      ld.j += 2;
      while (ld.have && ld.j >= ld.it.n) ld.next(p, h);
    };
    auto forward = [&] {   // `at` to the next tile
      while (at.have && at.j >= at.it.n) {
        at.next(p, h);
        if (!at.have) return;
        wait(qfull + 8 * (at.item & 1u), (at.item >> 1) & 1u, 64);
        if (!ok) return;
        // an item of one tile: this stream has no scores there
        if (at.j >= at.it.n && leader) mbar_arrive(qfree + 8 * (at.item & 1u));
      }
    };
    auto scores = [&](uint32_t s, int upper) {   // of 32 keys
      const uint64_t dq = sdesc_k128(sQ + (at.item & 1u) * kChQ), dk = sdesc_k128(sk + s * kChKV) + (upper ? kChHalf : 0u);
      tc_fence_after();
      if (leader) {
#pragma unroll
        for (int k = 0; k < 4; ++k) tc_mma_bf16(tm + h * 64 + 32 * upper, dq + (uint64_t)(2 * k), dk + (uint64_t)(2 * k), kChIdescHalf, k > 0 ? 1u : 0u);
        tc_commit((upper ? supper : sready) + 8 * h);
        if (!upper && at.j + 2 >= at.it.n) tc_commit(qfree + 8 * (at.item & 1u));
      }
    };
    while (ld.have && ld.j >= ld.it.n) ld.next(p, h);
    load();
    load();
    forward();
    if (ok && at.have) {
      wait(kf, 0u, 62);
      if (ok) {
        scores(0, 1);
        scores(0, 0);
      }
    }
    while (ok && at.have) {
      const uint32_t s = i & 1u, ph = (i >> 1) & 1u;
      const uint32_t first = at.j == h ? 0u : 1u, more = (at.j >> 1) & (kChFlush - 1) ? 1u : 0u, item = at.item;
      // The next tile's scores: the upper 32 keys' columns are free since P is there, the lower ones' hold P.  Those of another item
      // come behind the product, for which its queries may wait.
      const bool same = at.j + 2 < at.it.n;
      at.j += 2;
      wait(pready + 8 * h, i & 1u, 65);
      if (same) {
        wait(kf + 8 * (s ^ 1u), ((i + 1) >> 1) & 1u, 62);
        if (ok) scores(s ^ 1u, 1);
      }
      if (!first) wait(ofree, (item & 1u) ^ 1u, 69);   // the accumulators are free once the O of the item before has been read
      wait(vf + 8 * s, ph, 63);
      if (!ok) break;
      tc_fence_after();
      if (leader) {
        const uint64_t dv = sdesc_k128(sv + s * kChKV);
#pragma unroll
        for (int k = 0; k < 4; ++k) tc_mma_bf16_ta(tm + 128 + h * 64, tm + h * 64 + 8 * k, dv + kChVStep * k, kChIdescPV, k > 0 ? 1u : more);
        tc_commit(pvdone + 8 * h);
      }
      if (!same) {
        forward();
        if (ok && at.have) {
          wait(kf + 8 * (s ^ 1u), ((i + 1) >> 1) & 1u, 62);
          if (ok) scores(s ^ 1u, 1);
        }
      }
      wait(pvdone + 8 * h, i & 1u, 70);
      if (!ok) break;
      if (at.have) scores(s ^ 1u, 0);
      load();
      ++i;
    }
  } else {
    // ------------------------------------------------------------------ softmax and result: a thread per row and stream
    // The streams of an item meet at a named barrier that all 256 threads reach whatever happened before; the decision to give
    // up is taken from the item's flag, which is only written before it (two flags in turn).
    const int quarter = warp & 3, half = (warp - 2) >> 2, row = quarter * 32 + lane;
    const uint32_t lane_addr = (uint32_t)(quarter * 32) << 16, s_addr = tmem + lane_addr + half * 64;
    float2* xml = reinterpret_cast<float2*>(bar_ptr + 256);   // [item parity][stream][row]: (maximum, sum)
    uint32_t n_s = 0, n_other = 0, nit = 0;   // tiles of this stream, of the other one; items
    bool ok = true;
    ChWalk walk(share);
    ChItem it;
    while (walk.next(p, it)) {
      const int r = it.row0 + row, qi = ch_div_g(p, min(r, it.n_rows - 1));
      const bool live = r < it.n_rows;
      const int pos = it.past + qi;
      const float fac = live ? __ldg(p.q_fac + (long long)it.head * p.T * p.G + (long long)it.t0 * p.G + r) : 1.f;
      const uint4* info = p.info + ((size_t)it.req * p.kv.H + it.head) * p.tiles;
      float m = 0.f, l = 0.f;   // maximum (powers of two), sum of 2^(s - m)
      bool fresh = true;        // no key seen yet: m means nothing
      const int j_end = it.j0 + it.n;
      // The sums so far to memory, added to what is there already, all against the present maximum.
      auto flush = [&](bool begun) {
        float4* keep = p.keep + (size_t)(blockIdx.x * 2 + half) * kChKeep * kChRows + row;
        const float corr = begun ? ch_exp2(keep[16 * kChRows].x - m) : 0.f;
#pragma unroll 1
        for (int q = 0; q < 16; q += 4) {
          uint32_t o[16];
          tmem_ld16(s_addr + 128 + 4 * q, o);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float4 v = make_float4(__uint_as_float(o[4 * i]), __uint_as_float(o[4 * i + 1]), __uint_as_float(o[4 * i + 2]), __uint_as_float(o[4 * i + 3]));
            float4* at = keep + (q + i) * kChRows;
            if (begun) {
              const float4 b = *at;
              v = make_float4(fmaf(b.x, corr, v.x), fmaf(b.y, corr, v.y), fmaf(b.z, corr, v.z), fmaf(b.w, corr, v.w));
            }
            *at = v;
          }
        }
        keep[16 * kChRows].x = fresh ? -FLT_MAX : m;
      };
      uint2 at = half < it.n ? __ldg(reinterpret_cast<const uint2*>(info + it.j0 + half)) : make_uint2(0u, 0u);
      for (int j = it.j0 + half, stop = min(j_end, j + 2 * kChFlush);; stop = min(j_end, j + 2 * kChFlush)) {
        for (; j < stop && ok; j += 2, ++n_s) {
          const uint2 now = at;
          if (j + 2 < j_end) at = __ldg(reinterpret_cast<const uint2*>(info + j + 2));
          const float c = __uint_as_float(now.x) * fac, ev = __uint_as_float(now.y & ~kChFlags);
          const int seen = pos - j * kChKeys;   // the last key of the tile that the row sees
          if (!(ok = mbar_wait_warp(supper + 8 * half, n_s & 1u, abort_flag, p.status, 66))) break;
          tc_fence_after();
          auto lower = [&] {   // the scores of the lower 32 keys: complete (and with them the product before)
            ok = mbar_wait_warp(sready + 8 * half, n_s & 1u, abort_flag, p.status, 68);
            tc_fence_after();
          };
          bool done = false;
          float base = ev;   // what the scores times c are to be added to
          // the maximum to what leaves 2^kChTop, the sums with it
          auto move = [&](float tm, bool grow) {
            const float m_new = grow ? tm - kChTop : m, corr = grow && !fresh ? ch_exp2(m - m_new) : 1.f;
            if (grow && !fresh) l = ch_rescale(l, m - m_new);
            m = m_new;
            fresh = fresh && !grow;
            if (j != it.j0 + half) {   // (these scores exist only because the product before is complete)
#pragma unroll 1
              for (int q = 0; q < 64; q += 16) {
                uint32_t o[16];
                tmem_ld16(s_addr + 128 + q, o);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
                tmem_st16(s_addr + 128 + q, o);
              }
            }
          };
#pragma unroll 1
          for (bool again = (now.y & kChFlags) == 0u; again;) {
            uint32_t va[16], vb[16];
            // Weights against the maximum so far, the tile's own maximum beside them: groups of 16 keys, the next group's read in
            // flight, P in registers until the maximum is known to hold.  Else it moves, and the tile is taken again.
            const uint64_t off2 = pair_f32(base - m, base - m), c2 = pair_f32(c, c);
            uint64_t l2 = pair_f32(0.f, 0.f);
            float ma = -INFINITY, mc = -INFINITY;
            uint32_t w[2][16];
            auto group = [&](const uint32_t (&v)[16], int k, bool masked) {
              auto out = [&](int i) { return masked && 16 * k + i > seen; };
              auto x = [&](int i) { return out(i) ? -INFINITY : __uint_as_float(v[i]); };
#pragma unroll
              for (int i = 0; i < 16; i += 4) {
                ma = fmax3(ma, x(i), x(i + 1));
                mc = fmax3(mc, x(i + 2), x(i + 3));
              }
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                float x0, x1;
                unpair_f32(fma2(pair_f32(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), c2, off2), x0, x1);
                const float p0 = out(i) ? 0.f : ch_exp2(x0), p1 = out(i + 1) ? 0.f : ch_exp2(x1);   // (c may be 0: not by scores of -inf)
                l2 = add2(l2, pair_f32(p0, p1));
                const __half2 h2 = __floats2half2_rn(p0, p1);
                w[k >> 1][8 * (k & 1) + (i >> 1)] = *reinterpret_cast<const uint32_t*>(&h2);
              }
            };
            auto tile = [&](bool masked) {
              tmem_ld16(s_addr + 32, va);
              tmem_ld_wait();
              tmem_ld16(s_addr + 48, vb);
              group(va, 2, masked);
              tmem_ld_wait();
              group(vb, 3, masked);
              lower();
              tmem_ld16(s_addr, va);
              tmem_ld_wait();
              tmem_ld16(s_addr + 16, vb);
              group(va, 0, masked);
              tmem_ld_wait();
              group(vb, 1, masked);
            };
            if (j * kChKeys + kChKeys - 1 <= it.first_pos) tile(false);
            else tile(true);
            if (!ok) break;
            const float tm = fmaf(fmaxf(ma, mc), c, base);
            // too small for fp32 (the maximum comes from values 2^80 times this tile's), of keys whose 2^(s - m) still counts in the sum
            // (differences, which are exact: of large maxima a sum with 15 rounds to 16, and 2^16 is beyond fp16)
            const bool grow = fresh ? tm > -INFINITY : tm - m > kChMost, small = !fresh && tm < m - 80.f && tm - ev > m - 60.f;
            // so large that a product not rounded, less a maximum that is, may be anything: the row's scores are first taken less the largest
            const bool huge = base == ev && fabsf(tm) > kChHuge && fabsf(tm) < INFINITY;
            const uint32_t votes = (grow ? 1u : 0u) | (small ? 2u : 0u) | (huge ? 4u : 0u), vote = __reduce_or_sync(0xffffffffu, votes);
            if (vote != 0u && !(vote & 2u)) {
              if (vote & 4u) {
                const float less = huge ? fmaxf(ma, mc) : 0.f;
                if (huge) base = tm;
#pragma unroll 1
                for (int q = 0; q < 64; q += 16) {
                  tmem_ld16(s_addr + q, va);
                  tmem_ld_wait();
#pragma unroll
                  for (int i = 0; i < 16; ++i) va[i] = __float_as_uint(__uint_as_float(va[i]) - less);
                  tmem_st16(s_addr + q, va);
                }
                tmem_st_wait();
              }
              if (vote & 1u) move(tm, grow);
              continue;
            }
            again = false;
            if (vote == 0u) {
              tmem_st16(s_addr, w[0]);
              tmem_st16(s_addr + 16, w[1]);
              float la, lb;
              unpair_f32(l2, la, lb);
              l = fmaf(la + lb, ch_exp2(-ev), l);
              done = true;
            }
          }
          if (ok && !done) lower();
          if (!ok) break;
          if (!done) {   // one by one: unlike, hidden or NaN tokens, weights that are too small, scores that are huge
            const uint32_t hide = now.y & 0xFu;
            const float2* unlike = (now.y & kChUnlike) ? p.tok + (((size_t)it.req * p.kv.H + it.head) * p.tiles + j) * kChKeys : nullptr;
            uint32_t v[16];
            float tm = -INFINITY;
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {
              tmem_ld16(s_addr + 16 * k, v);
              tmem_ld_wait();
              if (hide >> k & 1u) continue;
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                const float2 tk = unlike != nullptr ? __ldg(unlike + 16 * k + i) : make_float2(__uint_as_float(now.x), ev);
                if (16 * k + i <= seen) tm = fmaxf(tm, __fmaf_rn(__uint_as_float(v[i]), tk.x * fac, tk.y));
              }
            }
            const bool grow = fresh ? tm > -INFINITY : tm - m > kChMost;
            if (__any_sync(0xffffffffu, grow)) move(tm, grow);
            // Beyond kChHuge a step of the score's fp32 is whole powers of two: a weight is taken from the score as it was rounded for the
            // maximum, so that the largest has its 2^kChTop whatever the rounding did.
            const bool huge = fabsf(tm) > kChHuge && fabsf(tm) < INFINITY;
#pragma unroll 1
            for (int k = 0; k < 4; ++k) {   // P of 16 keys into columns whose scores have been read
              uint32_t w[8];
              tmem_ld16(s_addr + 16 * k, v);
              tmem_ld_wait();
#pragma unroll
              for (int i = 0; i < 16; i += 2) {
                float pr[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                  const float2 tk = unlike != nullptr ? __ldg(unlike + 16 * k + i + b) : make_float2(__uint_as_float(now.x), ev);
                  const float f = tk.x * fac, x = huge ? __fmaf_rn(__uint_as_float(v[i + b]), f, tk.y) - m - tk.y : fmaf(__uint_as_float(v[i + b]), f, -m);
                  const float pk = 16 * k + i + b <= seen && !(hide >> k & 1u) ? ch_exp2(x) : 0.f;
                  l += pk;
                  pr[b] = pk * ch_exp2(tk.y);
                }
                const __half2 h2 = __floats2half2_rn(pr[0], pr[1]);
                w[i >> 1] = *reinterpret_cast<const uint32_t*>(&h2);
              }
              tmem_st8(s_addr + 8 * k, w);
            }
            if (now.y & kChNan) {   // tokens stored as NaN: for the rows that see one
              const uint2 bad = __ldg(reinterpret_cast<const uint2*>(info + j) + 1);
              const unsigned long long mask = (unsigned long long)bad.y << 32 | bad.x;
              if (seen >= 0 && (mask & (seen >= 63 ? ~0ull : (1ull << (seen + 1)) - 1ull))) l = NAN;
            }
          }
          tmem_st_wait();
          tc_fence_before();
          mbar_arrive(pready + 8 * half);
        }
        if (!ok || j >= j_end) break;
        // the next tile's product begins a new sum; its scores exist only because the product before is complete
        ok = mbar_wait_warp(sready + 8 * half, n_s & 1u, abort_flag, p.status, 68);
        tc_fence_after();
        if (!ok) break;
        flush(((j - it.j0) >> 1) > kChFlush);
      }
      const bool kept[2] = {(it.n + 1) >> 1 > kChFlush, it.n >> 1 > kChFlush};   // streams with sums in memory: there they are completed
      if (kept[half] && ok) {
        ok = mbar_wait_warp(pvdone + 8 * half, (n_s - 1) & 1u, abort_flag, p.status, 67);
        tc_fence_after();
        if (ok) flush(true);
      }
      float2* mine = xml + (nit & 1u) * 256;
      mine[half * 128 + row] = make_float2(fresh ? -FLT_MAX : m, l);
      if (!ok) sm_fail[nit & 1u] = 1;
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (sm_fail[nit & 1u]) break;              // the same for all 256 threads
      const float2 own = mine[half * 128 + row], other = mine[(half ^ 1) * 128 + row];
      const float top = fmaxf(own.x, other.x);
      const float a_me = ch_exp2(own.x - top), a_ot = ch_exp2(other.x - top);
      const float sum = ch_rescale(own.y, own.x - top) + ch_rescale(other.y, other.x - top);
      const float inv = !it.whole ? 1.f : sum == 0.f ? 0.f : 1.f / sum;   // nothing to see: zeros
      const float f0 = (half == 0 ? a_me : a_ot) * inv, f1 = (half == 0 ? a_ot : a_me) * inv;
      // ---- (O_0 f_0 + O_1 f_1) -> out, or its piece: this thread's 32 of the row's 64 dims
      __nv_bfloat16* dst = p.out + (long long)(it.t0 + qi) * p.out_stride + (it.head * p.G + min(r, it.n_rows - 1) - qi * p.G) * 64 + half * 32;
      float* piece = p.part + ((blockIdx.x * 2 + (it.j0 == 0 ? 1 : 0)) * kChRows + row) * kChPitch;
      if (!it.whole && half == 0) *reinterpret_cast<float2*>(piece + 64) = make_float2(top, sum);
      n_other += (uint32_t)(half == 0 ? it.n >> 1 : (it.n + 1) >> 1);
      if (it.n > half) ok = mbar_wait_warp(pvdone + 8 * half, (n_s - 1) & 1u, abort_flag, p.status, 67);
      if (ok && it.n > 1 - half) ok = mbar_wait_warp(pvdone + 8 * (half ^ 1), (n_other - 1) & 1u, abort_flag, p.status, 67);
      if (ok) {
        tc_fence_after();
        uint32_t v[16], u[16];
#pragma unroll
        for (int c = 0; c < 32; c += 16) {
          tmem_ld16(tmem + lane_addr + 128 + half * 32 + c, v);
          if (it.n > 1) {
            tmem_ld16(tmem + lane_addr + 192 + half * 32 + c, u);
          } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = 0u;   // (nothing was ever accumulated there)
          }
          tmem_ld_wait();
          auto from_memory = [&](int stream, uint32_t (&o)[16]) {
            const float4* keep = p.keep + (size_t)(blockIdx.x * 2 + stream) * kChKeep * kChRows + (half * 8 + c / 4) * kChRows + row;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float4 b = keep[i * kChRows];
              o[4 * i] = __float_as_uint(b.x); o[4 * i + 1] = __float_as_uint(b.y);
              o[4 * i + 2] = __float_as_uint(b.z); o[4 * i + 3] = __float_as_uint(b.w);
            }
          };
          if (kept[0]) from_memory(0, v);
          if (kept[1]) from_memory(1, u);
          if (c == 16) {                          // O is in registers: the accumulators may be written again
            tc_fence_before();
            mbar_arrive(ofree);
          }
          float x[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) x[i] = fmaf(__uint_as_float(u[i]), f1, __uint_as_float(v[i]) * f0);
          if (!it.whole) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<float4*>(piece + half * 32 + c + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
          } else if (live) {
            uint32_t o[8];
#pragma unroll
            for (int i = 0; i < 16; i += 2) o[i >> 1] = pack_bf16(x[i], x[i + 1]);
            *reinterpret_cast<uint4*>(dst + c) = make_uint4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<uint4*>(dst + c + 8) = make_uint4(o[4], o[5], o[6], o[7]);
          }
        }
      }
      ++nit;
    }
  }
  // ------------------------------------------------------------------ teardown
  if (*abort_flag) {
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 2000000ull) __nanosleep(1000);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, kChTmemCols);
  }
}

// ---- host
struct ChunkSpace { size_t kd, vd, qd, fac, info, tok, share, part, desc, keep, total; };
static ChunkSpace chunk_space(long long R, long long T, long long max_kv, long long n_heads, long long H) {
  ChunkSpace c;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off += align_up(bytes, 256); return o; };
  const size_t tiles = (size_t)((max_kv + kChKeys - 1) / kChKeys), rows = (size_t)R * tiles * kChKeys;
  c.kd = take(rows * H * 128);
  c.vd = take(rows * H * 128);
  c.qd = take((size_t)T * n_heads * 128);
  c.fac = take((size_t)T * n_heads * 4);
  c.info = take((size_t)R * H * tiles * 16);
  c.tok = take(rows * H * 8);
  c.share = take(kChMaxWorkers * sizeof(int4));
  c.desc = take(2 * kChMaxWorkers * sizeof(int4));
  c.part = take((size_t)kChMaxWorkers * 2 * kChRows * kChPitch * sizeof(float));
  c.keep = take(tiles > 2 * kChFlush ? (size_t)kChMaxWorkers * 2 * kChKeep * kChRows * sizeof(float4) : 0);
  c.total = off;
  return c;
}

size_t kv_chunk_bytes(int R, int T, int max_kv, int n_heads, int H) { return chunk_space(R, T, max_kv, n_heads, H).total; }

moin_status launch_kv_chunk(HostState* hs, const KvView& kv, const int* table, const int* rows, const int* cu_q, const int* kv_len, int n_rows,
                            int max_pages, int R, int T, int max_q, int max_kv, int n_heads, const __nv_bfloat16* q, long long q_stride,
                            __nv_bfloat16* out, long long out_stride, const float2* rope, float scale_log2, void* workspace, KvPieces* pieces, cudaStream_t s) {
  const ChunkSpace c = chunk_space(R, T, max_kv, n_heads, kv.H);
  char* w = (char*)workspace;
  ChunkParams p = {};
  p.kv = kv; p.table = table; p.rows = rows; p.cu_q = cu_q; p.kv_len = kv_len; p.n_rows = n_rows; p.max_pages = max_pages;
  p.R = R; p.T = T; p.max_q = max_q; p.max_kv = max_kv; p.n_heads = n_heads; p.G = n_heads / kv.H;
  p.inv_g = (uint32_t)((0x100000000ull + p.G - 1) / p.G);
  p.n_blk = (int)(((long long)max_q * p.G + kChRows - 1) / kChRows);
  p.tiles = (max_kv + kChKeys - 1) / kChKeys;
  p.q = q; p.q_stride = q_stride; p.out = out; p.out_stride = out_stride; p.rope = rope; p.scale_log2 = scale_log2;
  p.kd = (__half*)(w + c.kd); p.vd = (__half*)(w + c.vd); p.qd = (__half*)(w + c.qd); p.q_fac = (float*)(w + c.fac); p.info = (uint4*)(w + c.info); p.tok = (float2*)(w + c.tok);
  p.dense_blocks = R * kv.H * p.tiles;
  p.share = (int4*)(w + c.share); p.part = (float*)(w + c.part); p.keep = (float4*)(w + c.keep); p.desc = (int4*)(w + c.desc);
  const long long items = (long long)p.n_blk * R * kv.H, most = items * ((p.tiles + 1) / 2 + kChItemCost) / kChLeast + 1;   // shares that there can be
  long long workers = 2L * hs->n_sms < kChMaxWorkers ? 2L * hs->n_sms : kChMaxWorkers;
  if (workers > most) workers = most;
  p.workers = (int)workers;
  *pieces = {p.part, p.desc, p.workers, items};
  p.status = hs->status;
  CUtensorMap mq, mk, mv;
  const uint64_t dense_rows = (uint64_t)R * p.tiles * kChKeys;
  moin_status st = make_map(&mq, p.qd, (uint64_t)T * n_heads, 64, kChRows);
  if (!st) st = make_map(&mk, p.kd, dense_rows, (uint64_t)kv.H * 64, kChKeys);
  if (!st) st = make_map(&mv, p.vd, dense_rows, (uint64_t)kv.H * 64, kChKeys);
  if (st) return st;
  cudaError_t e = ensure_smem_optin(OPTIN_KV_CHUNK, kv_chunk_kernel, kChSmem);
  if (e != cudaSuccess) return record_cuda(e);
  e = launch_pdl(kv_dense_kernel, 1u + (unsigned)p.dense_blocks + (unsigned)T, 128, 0, s, p);
  if (e == cudaSuccess)
    e = launch_pdl(kv_chunk_kernel, (unsigned)workers, kChThreads, kChSmem, s, mq, mk, mv, p);
  return record_cuda(e);
}

}  // namespace moin
