// Attention over a paged cache: what its kernels share. Arguments, the rows a
// unit covers, the division of the work among the CTAs, and the hand-over of
// partial sums to the pass that joins them.
//
// Notation: a request's rows are its chunk's (token, query head of one key
// head) pairs, row r = token * g + head, g = Hq / Hkv: they all read the same
// keys. A unit is a tile of M consecutive rows of one (request, key head) over
// all the keys that any of them sees.
//
// Division of the work. The lengths are on the device and differ by orders of
// magnitude, so CTAs do not get units: the units are laid end to end in order
// (request, key head, row tile), each as long as its keys are many (plus a
// constant), and CTA c of n gets the c-th n-th of that line. A CTA works off
// the end of one unit, whole units, and the beginning of another; only the
// first and the last of its segments can be partial, so there are at most 2 n
// partial sums whatever the lengths, and they are all the workspace. Row tiles
// of one (request, key head) lie next to each other: the CTAs that read the
// same keys do so at the same time, out of L2.
#pragma once

#include <cuda_bf16.h>

#include "pair_common.cuh"
#include "tc_ptx.cuh"

namespace pairk {
namespace attend {

constexpr int kMaxCtas = 480;    // of a launch with units of up to kFewTile rows
constexpr int kMaxMany = 160;    // of a launch with units of kManyRows rows
constexpr int kMaxWorkers = 1920;  // warps with shares of their own, in a launch of them
constexpr int kManyRows = 256;   // rows of a unit of the kernel for many rows
constexpr int kFewTile = 64;     // rows of a unit of the kernel for few rows
// Chunks of up to so many rows go to the kernel for few rows, longer ones to the
// tensor cores: 64 chunks behind 2000 keys of 8 heads take 120 us at 32 rows in
// the former; at 48 161 there and 134 here.
constexpr int kFewRows = 32;
constexpr float kLn2 = 0.69314718055994531f;
// A unit's fixed cost, in keys: what a CTA spends between two units and on
// starting its tiles. Measured on 32/8 heads of 128: 64 chunks of 32 to 256 tokens
// behind 100 to 3000 keys (many rows): 474 us at 48 keys, 361 at 400, 322 at 800,
// 337 at 1600; 16 x 16 requests with drafts (few rows): 422 at 48, 404 at 128, 398 at
// 192. Heads of 64 and 256 go by the same values; the 48 of fp32's units of 16 rows
// was not swept.
constexpr int kManyCost = 800, kFewCost = 192, kSimtCost = 48;
// Keys of a request at most: tile numbers, and a unit's length with its fixed
// cost, stay within 32 bits.
constexpr int kMaxKeys = INT32_MAX - 4096;
constexpr int kMinKeys = 128;    // least share of the line worth a CTA of its own
// Or a warp, where those have shares (32 requests in fp32 of up to 640 keys: 16.6 us; 64
// keys 18.6, 128 keys 20.7).
constexpr int kMinWarp = 96;

struct Args {
  int64_t T;
  int32_t R, Hq, Hkv, g;
  int32_t rows_over, rows_upto;  // requests with rows in (rows_over, rows_upto] are this launch's
  const void *q;
  int64_t q_row, q_head;
  const void *kc, *vc;
  pair_cache_strides ks, vs;
  int32_t num_pages, page;
  const int32_t *table;
  int32_t width;
  const int32_t *kv_len, *cu;
  float scale;
  void *out;
  float *lse;
  struct Desc *desc;  // [CTAs][2] segments of each CTA
  float *part;        // partial sums, part_floats() each
  int32_t *dev_err;
  // Caches in 8 bits: exponent bytes (null: caches in the queries' type).
  const uint8_t *ke, *ve;
  pair_cache_strides kes, ves;
  bool narrow;        // strides of pages and tokens fit in 32 bits
  int32_t slice_pages, slice_rest;  // a slice further in the block table: pages, places
  int32_t heads;      // key heads on the line of units (a fourth where warps share a CTA's)
  int32_t unit_cost;  // fixed cost of a unit of this launch, in keys
};

// A segment of a CTA: key tiles [t0, t1) of the unit's `tiles`.
struct Desc {
  int32_t i, h, rt, t0, t1, tiles;
  int32_t row0, rows;  // first token of the request's chunk, rows of the unit
};

// Partial sums of M rows: max (log2 units), sum, output sums.
__host__ __device__ constexpr int64_t part_floats(int M, int D) { return (int64_t)M * (D + 2); }

struct Request {
  int32_t row0;   // first token of the chunk in the packed arrays
  int32_t n, kv;  // tokens of the chunk, keys in the cache (they include it)
};

// Request i with what does not fit together cut down to what does; without
// rows if they are another launch's.
__device__ __forceinline__ Request request(const Args &a, int i) {
  const int lo = a.cu[i], hi = a.cu[i + 1], len = a.kv_len[i];
  const bool sane = lo >= 0 && hi >= lo && hi <= a.T;
  const int64_t most = (int64_t)a.width * a.page;
  Request r{lo, sane ? hi - lo : 0, len < 0 ? 0 : (int32_t)(len > most ? most : len)};
  const int rows = r.n * a.g;
  if (rows <= a.rows_over || rows > a.rows_upto || r.kv > kMaxKeys) r.n = 0;
  return r;
}
// By a whole block: requests whose entries do not fit together.
__device__ __forceinline__ void report_requests(const Args &a) {
  bool bad = false;
  for (int i = threadIdx.x; i < a.R; i += blockDim.x) {
    const int lo = a.cu[i], hi = a.cu[i + 1], len = a.kv_len[i];
    bad |= lo < 0 || hi < lo || hi > a.T || len < 0 || len > kMaxKeys ||
           len > (int64_t)a.width * a.page;
  }
  if (bad || (threadIdx.x == 0 && a.cu[0] != 0)) flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
}

// The line of units of one request, in 1 / (2 g) keys (so that nothing is
// divided): unit k sees about (k + 1) M / g tokens of the chunk.
struct Line {
  int64_t base;   // of a unit, without its rows' own tokens
  int32_t units;  // row tiles per key head
  int32_t M;
  __device__ __forceinline__ Line(const Request &r, int M_, const Args &a) : M(M_) {
    base = (int64_t)2 * a.g * (a.unit_cost + max(0, r.kv - r.n));
    units = (int32_t)(((int64_t)r.n * a.g + M - 1) / M);
  }
  // Length of the first k units, and of unit k.
  __device__ __forceinline__ int64_t upto(int64_t k) const { return k * base + M * k * (k + 1); }
  __device__ __forceinline__ int64_t of(int64_t k) const { return base + 2 * M * (k + 1); }
};

__device__ __forceinline__ int64_t request_cost(const Args &a, int i, int M) {
  const Request r = request(a, i);
  const Line l(r, M, a);
  return (int64_t)a.heads * l.upto(l.units);
}

// Where on the line a CTA begins and ends.
struct Share {
  int64_t from, to;
  int64_t at;  // where request i begins
  int32_t i;
};

// By a whole block of NT threads; scratch: NT / 32 + 2 N int64 of shared memory. N
// shares of a block, from that of its first warp on: warp w's is the w-th of them, and
// `cta` that share's number (the block's, where N is 1).
template <int NT, int N = 1>
__device__ Share find_share(const Args &a, int M, int cta, int ctas, int64_t *scratch,
                            int least = kMinKeys) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  constexpr int W = NT / 32;
  const int per = (a.R + NT - 1) / NT;
  const int i0 = (int)min((int64_t)tid * per, (int64_t)a.R), i1 = min(i0 + per, a.R);
  int64_t sum = 0;
  for (int i = i0; i < i1; ++i) sum += request_cost(a, i, M);
  int64_t x = sum;
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) scratch[warp] = x;
  __syncthreads();
  int64_t total = 0, before = 0;
  for (int w = 0; w < W; ++w) {
    if (w == warp) before = total;
    total += scratch[w];
  }
  x += before - sum;  // exclusive
  int64_t n = max((int64_t)1, min((int64_t)ctas, total / (2 * a.g * least)));
  if (a.R == 1) {  // units of one length, nearly: no CTA across two of them
    const int64_t units = (int64_t)a.heads * Line(request(a, 0), M, a).units;
    if (n > units && units > 0) n -= n % units;
  }
  const int k0 = N > 1 ? warp : 0;  // the share that is returned
  // total * c / n, rounded down.
  const int64_t each = total / n;
  const uint32_t rest = (uint32_t)(total - each * n);
  const auto cut = [&](int c) { return each * c + rest * (uint32_t)c / (uint32_t)n; };
  Share s{0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int c = cta - k0 + k;
    if (c >= n) continue;
    const int64_t from = cut(c), to = cut(c + 1);
    if (k == k0) s.from = from, s.to = to;
    if (from < to && from >= x && from < x + sum) {
      int64_t at = x;
      int i = i0;
      for (; i < i1; ++i) {
        const int64_t c1 = request_cost(a, i, M);
        if (from < at + c1) break;
        at += c1;
      }
      scratch[W + 2 * k] = at;
      scratch[W + 2 * k + 1] = i;
    }
  }
  __syncthreads();
  if (s.from < s.to) {
    s.at = scratch[W + 2 * k0];
    s.i = (int32_t)scratch[W + 2 * k0 + 1];
  }
  return s;
}

// A segment as its CTA works on it.
struct Segment {
  int32_t i, h, rt;
  int32_t t0, t1, tiles;  // key tiles of the segment, of the unit
  int32_t row0;           // first packed token of the request's chunk
  int32_t r0, rows;       // first row of the tile in the chunk, rows in use
  int32_t first_seen;     // keys that row 0 of the chunk's first token sees (may be < 0)
  int32_t keys;           // keys that the tile's last row sees
  int32_t least;          // keys that every row of the tile sees
  int32_t kv;
  bool head;              // holds the unit's beginning
  __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == tiles; }
  // Keys seen by row r of the tile.
  __device__ __forceinline__ int seen(int r, int g) const {
    return max(0, first_seen + (r0 + r) / g);
  }
};

// Walks a CTA's share, one segment per call. All arguments are uniform. Units are cut
// between tiles of BN keys, between every S of them if the request table has more than one
// entry.
template <int M, int BN, int S = 1>
struct Walk {
  Share s;
  Request r;
  int32_t h, k, units;
  int64_t begin;  // where the unit begins
  bool started;

  __device__ __forceinline__ explicit Walk(const Share &share) : s(share), started(false) {}

  __device__ __forceinline__ bool next(const Args &a, Segment *g) {
    while (s.from < s.to) {
      if (!started) {  // the only search: the unit that the share begins in
        r = request(a, s.i);
        const Line l(r, M, a);
        const int64_t per_head = l.upto(l.units), off = s.from - s.at;
        h = (int)(off / per_head);
        const int64_t x = off - h * per_head;
        int lo = 0, hi = l.units;  // upto(lo) <= x < upto(hi)
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (l.upto(mid) <= x) lo = mid; else hi = mid;
        }
        k = lo;
        units = l.units;
        begin = s.at + h * per_head + l.upto(lo);
        started = true;
      } else {
        if (++k == units) {
          k = 0;
          if (++h == a.heads) {
            h = 0;
            do {
              if (++s.i >= a.R) return false;
              r = request(a, s.i);
            } while (r.n == 0);
            units = Line(r, M, a).units;
          }
        }
        begin = s.from;
      }
      const int64_t cost = Line(r, M, a).of(k);
      const int64_t x0 = s.from - begin, x1 = min(cost, x0 + (s.to - s.from));
      g->i = s.i;
      g->h = h;
      g->rt = k;
      g->row0 = r.row0;
      g->r0 = k * M;
      g->rows = min(M, r.n * a.g - k * M);
      g->first_seen = r.kv - r.n + 1;
      g->kv = r.kv;
      g->least = min(r.kv, g->seen(0, a.g));
      g->keys = min(r.kv, g->seen(g->rows - 1, a.g));
      g->tiles = (g->keys + BN - 1) / BN;
      const int every = a.R == 1 ? 1 : S;
      g->t0 = cut(x0, cost, g->tiles, every);
      g->t1 = cut(x1, cost, g->tiles, every);
      g->head = x0 == 0;
      s.from += x1 - x0;
      // A unit without keys is worked on (zeros are written) by whoever has
      // its beginning; an empty piece of another by nobody.
      if (g->t0 < g->t1 || (g->tiles == 0 && g->head)) return true;
    }
    return false;
  }

  // The key tile at which x of a unit's `cost` falls: the same for the CTA that
  // ends there and the one that begins there.
  static __device__ __forceinline__ int cut(int64_t x, int64_t cost, int tiles, int every) {
    if (x == 0) return 0;
    if (x == cost) return tiles;
    const int n = S == 1 ? tiles : (tiles + every - 1) / every;
    const int t = (int)__float2int_rn(__fdiv_rn((float)x, (float)cost) * (float)n);
    return S == 1 ? min(tiles, t) : t >= n ? tiles : t * every;
  }
};

// Rows that no request owns: out = 0, lse = -inf.
template <typename T, int D, int NT>
__device__ __forceinline__ void clear_spare_rows(const Args &a, int cta, int ctas) {
  const int64_t t0 = max(0, a.cu[a.R]);
  const int64_t vecs = (int64_t)a.Hq * D * sizeof(T) / 16;
  uint4 *out = static_cast<uint4 *>(a.out);
  for (int64_t x = t0 * vecs + (int64_t)cta * NT + threadIdx.x; x < a.T * vecs;
       x += (int64_t)ctas * NT)
    out[x] = make_uint4(0, 0, 0, 0);
  if (a.lse)
    for (int64_t x = t0 * a.Hq + (int64_t)cta * NT + threadIdx.x; x < a.T * a.Hq;
         x += (int64_t)ctas * NT)
      a.lse[x] = -INFINITY;
}

// Element offset of a key's or value's row in its cache. A page id outside the
// cache is reported and replaced by page 0.
__device__ __forceinline__ int64_t cache_row(const Args &a, const pair_cache_strides &st, int id,
                                             int off, int h) {
  return id * st.for_page + off * st.for_token + h * st.for_head;
}
__device__ __forceinline__ int page_of(const Args &a, int i, int key, int *off) {
  const int at = key / a.page;
  *off = key - at * a.page;
  const int id = a.table[(int64_t)i * a.width + at];
  if ((unsigned)id < (unsigned)a.num_pages) return id;
  flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
  return 0;
}

// Where row r of a segment's tile lies in the packed arrays: (token, head).
struct RowAt {
  int64_t token;
  int head;
};
__device__ __forceinline__ RowAt row_at(const Args &a, int row0, int r0, int h, int r) {
  const int tok = (r0 + r) / a.g;
  return {(int64_t)row0 + tok, h * a.g + (r0 + r) - tok * a.g};
}

// The k-th segment of CTA `cta`, if partial, is noted for the pass that joins
// the partial sums; its slot in the workspace.
__device__ __forceinline__ int64_t note_partial(const Args &a, const Segment &s, int cta, int k) {
  const int slot = cta * 2 + (k ? 1 : 0);
  if (threadIdx.x == 0) a.desc[slot] = {s.i, s.h, s.rt, s.t0, s.t1, s.tiles, s.row0, s.rows};
  return slot;
}
__device__ __forceinline__ void clear_notes(const Args &a, int cta) {
  if (threadIdx.x < 2) a.desc[cta * 2 + threadIdx.x] = {0, 0, 0, 0, 0, 0, 0, 0};
}

// Values that row r of a segment's tile sees and that are not finite, added
// to its sums of 8 columns. The kernels take such values out of tiles that
// not every row sees whole (key tiles of BN keys from the first row's limit
// on), where they would meet weights of 0.
template <int D>
__device__ __forceinline__ void add_not_finite(const Args &a, const Segment &s, int BN, int r,
                                               int col, float (&v)[8]) {
  const __nv_bfloat16 *vc = static_cast<const __nv_bfloat16 *>(a.vc);
  const int most = min(s.seen(r, a.g), s.kv);
#pragma unroll 1
  for (int key = max(s.t0 * BN, s.least / BN * BN); key < min(most, s.t1 * BN); ++key) {
    int off;
    const int id = page_of(a, s.i, key, &off);
    const __nv_bfloat16 *row = vc + cache_row(a, a.vs, id, off, s.h) + col;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const float x = __bfloat162float(row[c]);
      if (!(fabsf(x) <= 3.4e38f)) v[c] += x;
    }
  }
}

// Asynchronous 16-byte copy into shared memory, zeros where nothing is there.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there) {
  const int bytes = there ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() {
  asm volatile("cp.async.commit_group;" ::: "memory");
}
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// x s + r, x + y and x y, two lanes per instruction.
__device__ __forceinline__ float2 fma2(float2 x, float2 s, float2 r) {
  float2 o;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(reinterpret_cast<uint64_t &>(o))
      : "l"(reinterpret_cast<uint64_t &>(x)), "l"(reinterpret_cast<uint64_t &>(s)),
        "l"(reinterpret_cast<uint64_t &>(r)));
  return o;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 o;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t &>(o))
      : "l"(reinterpret_cast<uint64_t &>(x)), "l"(reinterpret_cast<uint64_t &>(y)));
  return o;
}
__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
  float2 o;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(reinterpret_cast<uint64_t &>(o))
      : "l"(reinterpret_cast<uint64_t &>(x)), "l"(reinterpret_cast<uint64_t &>(y)));
  return o;
}

// Programmatic dependent launch. The kernel for many rows starts beside the one
// for few, on whose results it does not depend (it waits for its end only before
// its own, so that what comes after it comes after both); the pass that joins the
// partial sums starts while the kernel before it drains, and waits for its end.
__device__ __forceinline__ void let_next_start() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}
__device__ __forceinline__ void wait_for_previous() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Host side: the kernels, and the pass that joins the partial sums of up to two
// launches.
struct Launch {
  Args a;
  int M, ctas;  // rows of its units; 0 CTAs: there is no such launch
};
pair_status launch_simt(Launch *l, int D, cudaStream_t s);
pair_status launch_few(Launch *l, int D, cudaStream_t s);
// Caches in 8 bits; most_rows: of a chunk, as far as the host knows.
// slots: partial sums of kFewTile rows that the workspace has room for.
using FewLauncher = pair_status(Launch *l, int D, int64_t most_rows, int slots, cudaStream_t s);
FewLauncher launch_few_i8, launch_few_e4m3, launch_few_i8_f32, launch_few_e4m3_f32;
bool many_applies(const Args &a, int D);
pair_status launch_many(Launch *l, int D, cudaStream_t s);
bool many_applies_q8(const Args &a, int D);
pair_status launch_many_q8(Launch *l, int D, int fmt, cudaStream_t s);
int sm_count();
int useful_ctas(const Args &a, int M, int fit, int least = kMinKeys);

}  // namespace attend
}  // namespace pairk
