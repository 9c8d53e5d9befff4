// Page tables of the key/value cache, kept on the GPU: wanted request lengths in, pages taken and given back, slot and
// position of every new token out.  No read-back: a generation loop can be captured whole.
#include "kv.cuh"

namespace moin {

constexpr int kKvMaxRows = 65536;       // rows of a table (two bits each in shared memory)
constexpr int kKvTokensHere = 8192;     // tokens whose slots the first kernel writes itself

struct KvTabParams {
  int *table, *stack, *lens, *n_free, *lens_out, *n_free_out;
  const int *rows, *want;
  int *cu_q, *kv_len, *slot, *pos, *refused;
  int n_rows, max_pages, n_pages, P, R, T, tokens_here;
};

// Inclusive sums over the CTA of N values; the totals in `sum`.  64 bits: lengths that no pool could hold may be asked for.
template <int THREADS, int N>
__device__ __forceinline__ void block_scan(long long (&v)[N], long long (*part)[32], long long (&sum)[N]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const long long a = __shfl_up_sync(0xffffffffu, v[i], o);
      if (lane >= o) v[i] += a;
    }
  __syncthreads();   // (the array's last readers are done)
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (lane == 31) part[i][warp] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {   // every warp scans the warps' sums
    long long x = lane < THREADS / 32 ? part[i][lane] : 0;
#pragma unroll
    for (int o = 1; o < THREADS / 32; o <<= 1) {
      const long long a = __shfl_up_sync(0xffffffffu, x, o);
      if (lane >= o) x += a;
    }
    sum[i] = __shfl_sync(0xffffffffu, x, THREADS / 32 - 1);
    const long long before = __shfl_sync(0xffffffffu, x, (warp + 31) & 31);
    if (warp > 0) v[i] += before;
  }
}
// First index whose inclusive sum exceeds x.
__device__ __forceinline__ int first_above(const int* inc, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (inc[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// One CTA.  Requests go through in chunks of its threads, twice: first the pages given back go on the stack, then pages are
// taken from its top.  Prefix sums say whose the k-th page or token is, and threads walk pages and tokens, not requests, so
// that a long request costs no more than many short ones.  Bound by latency: the chain row, length, prefix sums, page, slot.
// 256 threads where a chunk of them holds the batch and its tokens are few, else 1024.
template <int THREADS>
__global__ void __launch_bounds__(THREADS)
kv_update_kernel(const KvTabParams p) {
  __shared__ uint32_t seen[kKvMaxRows / 32], twice[kKvMaxRows / 32];
  __shared__ int s_inc[THREADS], s_new[THREADS], s_row[THREADS], s_at[THREADS], s_old[THREADS], s_have[THREADS], s_ok[THREADS];
  __shared__ long long s_part[3][32];
  __shared__ int s_got;
  pdl_begin();
  const int tid = threadIdx.x, P = p.P;
  // a request: its row, cached and wanted tokens; `named` unless there is no such row or the call has it twice, `good` if its lengths
  // are possible too
  struct Req { int row, old, want; bool named, good; };
  auto load = [&](int i) {
    Req q = {0, 0, 0, false, false};
    if (i >= p.R) return q;
    const int row = p.rows ? p.rows[i] : i;
    if (row < 0 || row >= p.n_rows) return q;
    const int old = p.lens[row], want = p.want[i], most = p.max_pages * P;
    q.row = row;
    q.named = true;
    q.old = old;
    q.good = old >= 0 && want >= 0 && old <= most && want <= most;
    q.want = q.good ? want : old;
    return q;
  };
  auto drop_twice = [&](Req& q) {
    if (p.rows && q.named && (twice[q.row >> 5] >> (q.row & 31) & 1u)) q = {0, 0, 0, false, false};
  };
  int top = min(max(*p.n_free, 0), p.n_pages);
  Req only = load(tid);    // the batch, where one chunk holds it
  const bool one = p.R <= THREADS;
  if (p.rows != nullptr) {
    for (int i = tid; i < (p.n_rows + 31) / 32; i += THREADS) seen[i] = twice[i] = 0;
    __syncthreads();
    for (int i = tid; i < p.R; i += THREADS) {
      const int r = p.rows[i];
      if (r < 0 || r >= p.n_rows) continue;
      const uint32_t bit = 1u << (r & 31);
      if (atomicOr(&seen[r >> 5], bit) & bit) atomicOr(&twice[r >> 5], bit);   // (which of the two comes second does not matter)
    }
    __syncthreads();
    drop_twice(only);
  }
  auto request = [&](int i) {
    if (one) return only;
    Req q = load(i);
    drop_twice(q);
    return q;
  };
  for (int c0 = 0; c0 < p.R; c0 += THREADS) {   // pages given back
    const Req q = request(c0 + tid);
    const int need = (q.want + P - 1) / P;
    const int back = q.good ? max(0, (q.old + P - 1) / P - need) : 0;
    if (!__syncthreads_or(back > 0)) continue;
    long long sum[1], v[1] = {back};
    block_scan<THREADS>(v, s_part, sum);
    const int inc = (int)v[0];   // (rows times pages of a row fit: the host has looked)
    s_inc[tid] = inc;
    s_row[tid] = q.row;
    s_at[tid] = need - (inc - back);   // k-th page given back by the chunk, of this request: its table entry s_at + k
    __syncthreads();
#pragma unroll 4
    for (int k = tid; k < (int)sum[0]; k += THREADS) {
      const int i = first_above(s_inc, THREADS, k);
      if (top + k < p.n_pages) p.stack[top + k] = p.table[(size_t)s_row[i] * p.max_pages + s_at[i] + k];
    }
    top = (int)min((long long)p.n_pages, top + sum[0]);
    __syncthreads();
  }
  long long tokens = 0, asked = 0;
  int taken = 0, refused = 0;
  if (tid == 0) p.cu_q[0] = 0;
  for (int c0 = 0; c0 < p.R; c0 += THREADS) {   // pages taken, tokens placed
    const int i = c0 + tid;
    const Req q = request(i);
    const int have = (q.old + P - 1) / P;
    const int n_new = q.good ? max(0, q.want - q.old) : 0;
    const int wants = q.good ? max(0, (q.want + P - 1) / P - have) : 0;
    // tokens come first: a request whose tokens do not all fit into the batch takes no pages
    long long sum[2], v[2] = {n_new, wants};
    block_scan<THREADS>(v, s_part, sum);
    const long long tok = tokens + v[0];
    const bool room = n_new == 0 || tok <= p.T;
    int ask = wants;
    if (__syncthreads_or(!room)) {
      ask = room ? wants : 0;
      long long again[1], u[1] = {ask};
      block_scan<THREADS>(u, s_part, again);
      v[1] = u[0];
      sum[1] = again[0];
    }
    const long long upto = asked + v[1];
    const bool ok = q.good && room && (ask == 0 || upto <= top);
    // those that get pages stand before all others that ask: the sum before one of them is what has been taken
    const int end = (int)min(tok, (long long)p.T);
    s_inc[tid] = (int)min(upto, (long long)top);
    s_new[tid] = end;
    s_row[tid] = q.row;
    s_old[tid] = q.old - ((int)min(tok - n_new, (long long)p.T));   // token t of the batch: position s_old + t
    s_at[tid] = have - (int)min(upto - ask, (long long)top);        // k-th page taken by the call, of this request: entry s_at + k
    s_have[tid] = have;
    s_ok[tid] = ok;
    if (i < p.R) {
      p.cu_q[i + 1] = end;
      p.kv_len[i] = ok ? q.want : 0;
      if (q.named) p.lens_out[q.row] = ok ? q.want : q.old;
    }
    if (tid == 0) s_got = taken;
    refused += __syncthreads_count(i < p.R && !ok);
    if (ok && ask > 0) atomicMax(&s_got, (int)upto);
    __syncthreads();
    const int got = s_got;
#pragma unroll 4
    for (int k = taken + tid; k < got; k += THREADS) {
      const int j = first_above(s_inc, THREADS, k);
      p.table[(size_t)s_row[j] * p.max_pages + s_at[j] + k] = p.stack[top - 1 - k];
    }
    if (p.tokens_here) {
      const int t0 = (int)min(tokens, (long long)p.T), t1 = s_new[THREADS - 1];
      for (int t = t0 + tid; t < t1; t += THREADS) {
        const int j = first_above(s_new, THREADS, t);
        const int at = s_old[j] + t, entry = at / P;
        int page = -1;   // an entry that this call has taken comes from the stack: the table's is on its way
        if (s_ok[j]) page = entry >= s_have[j] ? p.stack[top - 1 - (entry - s_at[j])] : p.table[(size_t)s_row[j] * p.max_pages + entry];
        p.slot[t] = s_ok[j] ? page * P + at % P : -1;
        p.pos[t] = s_ok[j] ? at : -1;
      }
    }
    tokens += sum[0];
    asked += sum[1];
    taken = got;
    __syncthreads();
  }
  if (p.tokens_here)
    for (int t = (int)min(tokens, (long long)p.T) + tid; t < p.T; t += THREADS) p.slot[t] = p.pos[t] = -1;
  if (tid == 0) {
    *p.n_free_out = top - taken;
    *p.refused = refused;
  }
}

// Slots of many tokens: a thread each, its request found in the offsets that the kernel above wrote.
__global__ void __launch_bounds__(256)
kv_slots_kernel(const KvTabParams p) {
  pdl_begin();
  const int t = blockIdx.x * 256 + threadIdx.x;
  if (t >= p.T) return;
  if (t >= p.cu_q[p.R]) {
    p.slot[t] = p.pos[t] = -1;
    return;
  }
  const int i = first_above(p.cu_q + 1, p.R, t);
  const int len = p.kv_len[i];
  const int at = len - (p.cu_q[i + 1] - t);   // the last of a request's tokens is its last cached one
  p.pos[t] = len > 0 ? at : -1;
  p.slot[t] = len > 0 ? p.table[(size_t)(p.rows ? p.rows[i] : i) * p.max_pages + at / p.P] * p.P + at % p.P : -1;
}

__global__ void __launch_bounds__(256)
kv_reset_kernel(int* lens, int n_rows, int* stack, int n_pages, int* n_free) {
  pdl_begin();
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < n_rows) lens[i] = 0;
  if (i < n_pages) stack[i] = n_pages - 1 - i;   // page 0 is taken first
  if (i == 0) *n_free = n_pages;
}

}  // namespace moin

using namespace moin;

static moin_status tables_ok(const moin_kv_tables* t) {
  if (!t || !t->block_table || !t->free_pages || !t->lens || !t->n_free) return MOIN_ERR_INVALID_ARG;
  if (t->n_rows < 1 || t->max_pages < 1 || t->n_pages < 1) return MOIN_ERR_INVALID_ARG;
  if (t->page_tokens != 16 && t->page_tokens != 32 && t->page_tokens != 64 && t->page_tokens != 128) return MOIN_ERR_BAD_SHAPE;
  if (t->n_rows > kKvMaxRows || (long long)t->n_pages * t->page_tokens > 0x7FFFFFFFll || (long long)t->max_pages * t->page_tokens > (1 << 30))
    return MOIN_ERR_BAD_SHAPE;
  return MOIN_OK;
}

extern "C" moin_status moin_kv_tables_reset(const moin_kv_tables* t, moin_stream stream) {
  moin_status st = tables_ok(t);
  if (st) return st;
  HostState* hs;
  if ((st = host_state(&hs))) return st;
  const int n = t->n_rows > t->n_pages ? t->n_rows : t->n_pages;
  ProfScope prof(MOIN_K_KV_TABLES, 1, (cudaStream_t)stream);
  return record_cuda(launch_pdl(kv_reset_kernel, (unsigned)((n + 255) / 256), 256, 0, (cudaStream_t)stream, t->lens, t->n_rows,
                                t->free_pages, t->n_pages, t->n_free));
}

extern "C" moin_status moin_kv_update(const moin_kv_tables* t, const int32_t* rows, const int32_t* want, const moin_kv_batch* b,
                                      int32_t* lens_out, int32_t* n_free_out, moin_stream stream) {
  moin_status st = tables_ok(t);
  if (st) return st;
  if (!b || b->R < 0 || b->T < 0 || !b->cu_q || !b->refused) return MOIN_ERR_INVALID_ARG;
  if (b->R > 0 && (!want || !b->kv_len)) return MOIN_ERR_INVALID_ARG;
  if (b->T > 0 && (!b->slot || !b->pos)) return MOIN_ERR_INVALID_ARG;
  // without a list of rows the requests are rows 0, 1, ..; with one no row may be named twice
  if (b->R > t->n_rows) return MOIN_ERR_BAD_SHAPE;
  if ((long long)b->R * t->max_pages > 0x7FFFFFFFll) return MOIN_ERR_BAD_SHAPE;   // pages are counted in 32 bits
  HostState* hs;
  if ((st = host_state(&hs))) return st;
  KvTabParams p = {};
  p.table = t->block_table; p.stack = t->free_pages; p.lens = t->lens; p.n_free = t->n_free;
  p.lens_out = lens_out ? lens_out : t->lens;
  p.n_free_out = n_free_out ? n_free_out : t->n_free;
  p.rows = rows; p.want = want;
  p.cu_q = b->cu_q; p.kv_len = b->kv_len; p.slot = b->slot; p.pos = b->pos; p.refused = b->refused;
  p.n_rows = t->n_rows; p.max_pages = t->max_pages; p.n_pages = t->n_pages; p.P = t->page_tokens; p.R = b->R; p.T = b->T;
  p.tokens_here = b->T <= kKvTokensHere;
  ProfScope prof(MOIN_K_KV_TABLES, p.tokens_here ? 1 : 2, (cudaStream_t)stream);
  st = record_cuda(b->R <= 256 && b->T <= 1024 ? launch_pdl(kv_update_kernel<256>, 1, 256, 0, (cudaStream_t)stream, p)
                                               : launch_pdl(kv_update_kernel<1024>, 1, 1024, 0, (cudaStream_t)stream, p));
  if (st || p.tokens_here) return st;
  return record_cuda(launch_pdl(kv_slots_kernel, (unsigned)((b->T + 255) / 256), 256, 0, (cudaStream_t)stream, p));
}
