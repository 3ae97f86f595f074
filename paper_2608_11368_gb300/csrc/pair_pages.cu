// Paged cache of the rollouts being generated: pair_pages_extend (block
// tables, chunk offsets and slots from request lengths) and
// pair_cache_append (keys and values into their slots).
#include "pair_common.cuh"

namespace pairk {
namespace {

constexpr int kExtendThreads = 1024;
// Slots per thread: four where that still gives every SM a block, as the scan of
// all requests is then shared by more of them.
constexpr int kExtendMany = 4;
constexpr int64_t kExtendSlots = 152 * kExtendThreads;

struct ExtendArgs {
  int32_t R, page, width;
  const int32_t *len, *held, *n_new, *free_pages;
  int32_t free_capacity;
  const int32_t *free_count;
  int64_t T;
  int32_t *table, *kv_len, *held_out, *cu;
  int64_t *slots;
  int32_t *taken, *dev_err;
};

// One request's needs. `bad`: its entries do not fit together or its table
// row is too short; it then needs no pages (its rows still count in cu).
struct Need {
  int32_t len, held, n, pages;
  bool bad;
};
__device__ __forceinline__ Need request_need(const ExtendArgs &a, int i) {
  Need r;
  r.len = a.len[i];
  r.held = a.held[i];
  const int32_t n = a.n_new[i];
  r.n = n > 0 ? n : 0;
  const int64_t kv = (int64_t)r.len + r.n;
  // (32 bits: a division of 64 costs some hundred instructions.)
  const uint32_t total = kv <= 0 ? 0 : (uint32_t)(kv - 1) / (uint32_t)a.page + 1;
  r.bad = r.len < 0 || r.held < 0 || n < 0 || r.held > a.width || kv > INT32_MAX ||
          (int64_t)r.held * a.page < r.len || total > (uint32_t)a.width;
  r.pages = r.bad || total <= (uint32_t)r.held ? 0 : (int32_t)(total - r.held);
  return r;
}

// Whether a request is served, given the sums of tokens and of pages before it. The
// sum of pages counts requests that are not served too, so behind one whose pages
// run out nobody is given any; who needs none is served all the same.
__device__ __forceinline__ bool served(const ExtendArgs &a, const Need &r, int64_t row,
                                       int64_t before, int32_t avail) {
  return !r.bad && (r.pages == 0 || before + r.pages <= avail) && row + r.n <= a.T;
}

// The prefix sums of tokens and of pages over all requests are formed by
// every block for itself (12 bytes per request, from L2 after the first), a run
// of consecutive requests per thread, so one launch does. A block writes the
// requests of its share and its 1024 or 4096 slots: a thread finds a token's
// request by bisection over the runs and a walk along the run. A slot's page is
// read from the old table entries or from the free list, never from entries this
// launch writes. Bound by latency: loads of the lengths, one block scan, the
// bisection, two dependent loads, stores. 64 requests of one token take 4 us with
// the launch, 4096 of one 9, 4096 of 128 on average 11.6 (a list of requests per
// block and a warp to each: 38; a bisection per token: 18).
template <int kPerLane>
__global__ void __launch_bounds__(kExtendThreads) pages_extend_kernel(ExtendArgs a) {
  constexpr int kTokens = kPerLane * kExtendThreads;
  __shared__ int64_t warp_n[32], warp_p[32];
  __shared__ int64_t run_n[kExtendThreads], run_p[kExtendThreads];  // sums before a run
  __shared__ int last_page;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.R + kExtendThreads - 1) / kExtendThreads;
  const int i0 = (int)min((int64_t)tid * per, (int64_t)a.R), i1 = min(i0 + per, a.R);
  int64_t sn = 0, sp = 0;
  for (int i = i0; i < i1; ++i) {
    const Need r = request_need(a, i);
    sn += r.n;
    sp += r.pages;
  }
  const int32_t avail = min(max(a.free_count[0], 0), a.free_capacity);
  int64_t xn = sn, xp = sp;
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t yn = __shfl_up_sync(0xffffffffu, xn, o);
    const int64_t yp = __shfl_up_sync(0xffffffffu, xp, o);
    if (lane >= o) {
      xn += yn;
      xp += yp;
    }
  }
  if (lane == 31) {
    warp_n[warp] = xn;
    warp_p[warp] = xp;
  }
  if (tid == 0) last_page = 0;
  __syncthreads();
  if (warp == 0) {
    const bool there = lane < kExtendThreads / 32;
    int64_t yn = there ? warp_n[lane] : 0, yp = there ? warp_p[lane] : 0;
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t zn = __shfl_up_sync(0xffffffffu, yn, o);
      const int64_t zp = __shfl_up_sync(0xffffffffu, yp, o);
      if (lane >= o) {
        yn += zn;
        yp += zp;
      }
    }
    warp_n[lane] = yn;
    warp_p[lane] = yp;
  }
  __syncthreads();
  const int64_t total_n = warp_n[31];
  xn += (warp ? warp_n[warp - 1] : 0) - sn;  // exclusive
  xp += (warp ? warp_p[warp - 1] : 0) - sp;
  run_n[tid] = xn;
  run_p[tid] = xp;
  __syncthreads();

  // A warp has consecutive tokens, a lane every 32nd of them: the next one is
  // mostly in the same run, a step or none further.
  const int64_t t0 = (int64_t)blockIdx.x * kTokens + warp * (32 * kPerLane) + lane;
  int run = -1, i = 0;
  int64_t run_end = 0, row = 0, before = 0;
  Need r{};
#pragma unroll
  for (int x = 0; x < kPerLane; ++x) {
    const int64_t t = t0 + 32 * x;
    if (t >= a.T) break;
    int64_t slot = -1;
    if (t < total_n) {
      if (t >= run_end) {
        int lo = run < 0 ? 0 : run, hi = kExtendThreads;  // run_n[lo] <= t < run_n[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (run_n[mid] <= t) lo = mid; else hi = mid;
        }
        run = lo;
        run_end = lo + 1 < kExtendThreads ? run_n[lo + 1] : total_n;
        i = lo * per;
        row = run_n[lo];
        before = run_p[lo];
        r = request_need(a, i);
      }
      while (row + r.n <= t) {
        row += r.n;
        before += r.pages;
        r = request_need(a, ++i);
      }
      if (served(a, r, row, before, avail)) {
        const uint32_t pos = r.len + (uint32_t)(t - row);
        const uint32_t at = pos / (uint32_t)a.page;
        const uint32_t off = pos - at * (uint32_t)a.page;
        int32_t *entry = a.table + (int64_t)i * a.width + at;
        const bool fresh = (int32_t)at >= r.held;
        const int32_t id = fresh ? a.free_pages[before + at - r.held] : *entry;
        // The held pages cover the cached tokens, so a new one begins with a
        // new token, whose thread enters it.
        if (fresh && off == 0) *entry = id;
        slot = (int64_t)id * a.page + off;
      }
    }
    a.slots[t] = slot;
  }

  const int share = (a.R + gridDim.x - 1) / gridDim.x;
  const int r0 = (int)min((int64_t)blockIdx.x * share, (int64_t)a.R), r1 = min(r0 + share, a.R);
  int top = 0;
  for (int i = i0; i < i1; ++i) {
    // Another block's requests count as far as this block's lie behind them in
    // the run (in block 0, which looks for the last page taken, all do).
    if (blockIdx.x != 0 && (i1 <= r0 || i >= r1)) break;
    const bool mine = i >= r0 && i < r1;
    const Need r = request_need(a, i);
    const bool ok = served(a, r, xn, xp, avail);
    if (ok && r.pages) top = (int32_t)(xp + r.pages);
    if (mine) {
      a.kv_len[i] = ok ? r.len + r.n : max(r.len, 0);
      a.held_out[i] = r.held + (ok ? r.pages : 0);
      a.cu[i + 1] = (int32_t)min(xn + r.n, a.T);
      if (i == 0) a.cu[0] = 0;
      if (!ok) flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
    }
    xn += r.n;
    xp += r.pages;
  }
  if (blockIdx.x != 0) return;
  top = __reduce_max_sync(0xffffffffu, top);
  if (lane == 0 && top) atomicMax(&last_page, top);
  __syncthreads();
  if (tid == 0) a.taken[0] = last_page;
}

struct AppendArgs {
  int64_t T;
  int32_t vecs_per_head, vecs;  // 16-byte pieces of a head, of a row
  const uint4 *k, *v;
  int64_t k_row, k_head, v_row, v_head;  // strides in 16-byte pieces, as below
  const int64_t *slots;
  int64_t n_slots;
  int32_t page;
  uint4 *kc, *vc;
  pair_cache_strides ks, vs;
  int32_t *dev_err;
};

constexpr int kAppendThreads = 128;
constexpr int kAppendAhead = 4;  // 16-byte pieces of keys and of values in flight per lane

// A warp moves a token's keys and values; its slot is taken apart once. Bound by
// HBM: every byte is read and written once (8192 tokens of 8 heads of 128 bf16:
// 12.7 us, 5.3 TB/s; a thread per 16-byte piece, dividing for itself, 14.1).
__global__ void __launch_bounds__(kAppendThreads) cache_append_kernel(AppendArgs a) {
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5);
  if (t >= a.T) return;
  const int64_t slot = a.slots[t];
  if (slot == -1) return;
  if (slot < 0 || slot >= a.n_slots) {
    if (lane == 0) flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
    return;
  }
  const int64_t pg = a.n_slots <= INT32_MAX ? (uint32_t)slot / (uint32_t)a.page : slot / a.page;
  const int64_t off = slot - pg * a.page;
  const uint4 *k = a.k + t * a.k_row, *v = a.v + t * a.v_row;
  uint4 *kc = a.kc + pg * a.ks.for_page + off * a.ks.for_token;
  uint4 *vc = a.vc + pg * a.vs.for_page + off * a.vs.for_token;
  for (int x0 = lane; x0 < a.vecs; x0 += 32 * kAppendAhead) {
    uint4 kx[kAppendAhead], vx[kAppendAhead];
#pragma unroll
    for (int y = 0; y < kAppendAhead; ++y) {
      const int x = x0 + 32 * y, h = x / a.vecs_per_head, c = x - h * a.vecs_per_head;
      if (x < a.vecs) {
        kx[y] = __ldg(k + h * a.k_head + c);
        vx[y] = __ldg(v + h * a.v_head + c);
      }
    }
#pragma unroll
    for (int y = 0; y < kAppendAhead; ++y) {
      const int x = x0 + 32 * y, h = x / a.vecs_per_head, c = x - h * a.vecs_per_head;
      if (x < a.vecs) {
        kc[h * a.ks.for_head + c] = kx[y];
        vc[h * a.vs.for_head + c] = vx[y];
      }
    }
  }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace pairk

using namespace pairk;

extern "C" {

pair_status pair_pages_extend(int32_t R, int32_t page_size, int32_t table_width,
                              const int32_t *len, const int32_t *held, const int32_t *n_new,
                              const int32_t *free_pages, int32_t free_capacity,
                              const int32_t *free_count, int64_t T, int32_t *block_table,
                              int32_t *kv_len, int32_t *held_out, int32_t *cu_new,
                              int64_t *slots, int32_t *taken, int32_t *dev_err,
                              pair_stream_t stream) {
  reset_launches();
  if (R < 1 || R > kMaxRequests || page_size < 1 || table_width < 1 || T < 1 || T > INT32_MAX ||
      free_capacity < 0 || !len || !held || !n_new || (!free_pages && free_capacity > 0) ||
      !free_count || !block_table || !kv_len || !held_out || !cu_new || !slots || !taken)
    return PAIR_ERR_INVALID_ARG;
  const pair_status dv = check_device();
  if (dv != PAIR_OK) return dv;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const ExtendArgs a{R,    page_size, table_width, len,    held, n_new, free_pages, free_capacity,
                     free_count, T,   block_table, kv_len, held_out, cu_new, slots, taken,
                     dev_err};
  PAIR_BEGIN("pages_extend", s);
  if (T > kExtendSlots)
    pages_extend_kernel<kExtendMany>
        <<<(unsigned)ceil_div(T, kExtendMany * kExtendThreads), kExtendThreads, 0, s>>>(a);
  else
    pages_extend_kernel<1><<<(unsigned)ceil_div(T, kExtendThreads), kExtendThreads, 0, s>>>(a);
  PAIR_LAUNCH_CHECK(s);
  return PAIR_OK;
}

pair_status pair_cache_append(int64_t T, int32_t Hkv, int32_t D, pair_dtype dt, const void *k,
                              int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                              int64_t v_head, const int64_t *slots, int32_t num_pages,
                              int32_t page_size, void *k_cache, pair_cache_strides ks,
                              void *v_cache, pair_cache_strides vs, int32_t *dev_err,
                              pair_stream_t stream) {
  reset_launches();
  if (T < 1 || T > INT32_MAX || Hkv < 1 || D < 1 || (dt != PAIR_F32 && dt != PAIR_BF16) || !k ||
      !v || !slots || num_pages < 1 || page_size < 1 || !k_cache || !v_cache)
    return PAIR_ERR_INVALID_ARG;
  const int per = dt == PAIR_BF16 ? 8 : 4;  // elements of 16 bytes
  // A stride over a single entry says nothing.
  const int64_t strides[][2] = {{k_row, T}, {v_row, T}, {k_head, Hkv}, {v_head, Hkv},
                                {ks.for_page, num_pages}, {vs.for_page, num_pages},
                                {ks.for_token, page_size}, {vs.for_token, page_size},
                                {ks.for_head, Hkv}, {vs.for_head, Hkv}};
  for (const auto &x : strides)
    if (x[1] > 1 && x[0] % per != 0) return PAIR_ERR_INVALID_ARG;
  if (D % per != 0 || (int64_t)Hkv * D > INT32_MAX || !aligned16(k) || !aligned16(v) ||
      !aligned16(k_cache) || !aligned16(v_cache))
    return PAIR_ERR_INVALID_ARG;
  const pair_status dv = check_device();
  if (dv != PAIR_OK) return dv;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const auto cut = [per](pair_cache_strides x) {
    return pair_cache_strides{x.for_page / per, x.for_token / per, x.for_head / per};
  };
  const AppendArgs a{T,
                     D / per,
                     Hkv * (D / per),
                     static_cast<const uint4 *>(k),
                     static_cast<const uint4 *>(v),
                     k_row / per,
                     k_head / per,
                     v_row / per,
                     v_head / per,
                     slots,
                     (int64_t)num_pages * page_size,
                     page_size,
                     static_cast<uint4 *>(k_cache),
                     static_cast<uint4 *>(v_cache),
                     cut(ks),
                     cut(vs),
                     dev_err};
  PAIR_BEGIN("cache_append", s);
  cache_append_kernel<<<(unsigned)ceil_div(T, kAppendThreads / 32), kAppendThreads, 0, s>>>(a);
  PAIR_LAUNCH_CHECK(s);
  return PAIR_OK;
}

}  // extern "C"
