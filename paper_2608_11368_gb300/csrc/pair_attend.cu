// pair_attend_paged: entry point, the fp32 kernel on the CUDA cores, and the
// pass that joins partial sums.
#include <math.h>

#include "pair_attend.cuh"

namespace pairk {
namespace attend {
namespace {

constexpr int kSimtThreads = 128;
constexpr int kSimtRows = 16;
constexpr int kSimtKeys = 64;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float *o, float x) { *o = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16 *o, float x) { *o = __float2bfloat16_rn(x); }

// One 16-byte piece as floats.
template <typename T>
__device__ __forceinline__ void widen(const uint4 &u, float *o) {
  const T *t = reinterpret_cast<const T *>(&u);
#pragma unroll
  for (int k = 0; k < 16 / (int)sizeof(T); ++k) o[k] = to_float(t[k]);
}

template <int D>
struct SimtSmem {
  float q[kSimtRows][D];
  float k[kSimtKeys][D + 4];
  float v[kSimtKeys][D];
  float p[kSimtRows][kSimtKeys];
  float m[kSimtRows], l[kSimtRows], fix[kSimtRows];
  int64_t krow[kSimtKeys], vrow[kSimtKeys];
  int seen[kSimtRows];
  int64_t scratch[kSimtThreads / 32 + 2];
};

// fp32 products on the CUDA cores: a tile of 64 keys and values in shared
// memory, 16 rows against it. A thread forms the scores of one key with 8
// rows, then the output sums of its columns for 16 rows (8 at D = 64).
template <typename T, int D>
__global__ void __launch_bounds__(kSimtThreads) attend_simt_kernel(Args a) {
  extern __shared__ __align__(16) uint8_t raw[];
  SimtSmem<D> &sm = *reinterpret_cast<SimtSmem<D> *>(raw);
  constexpr int M = kSimtRows, BN = kSimtKeys, VEC = 16 / sizeof(T);
  constexpr int CPT = D >= kSimtThreads ? D / kSimtThreads : 1;  // columns per thread
  constexpr int RG = D >= kSimtThreads ? 1 : kSimtThreads / D;   // row groups
  constexpr int RPT = M / RG;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cta = blockIdx.x, ctas = gridDim.x;
  clear_notes(a, cta);
  clear_spare_rows<T, D, kSimtThreads>(a, cta, ctas);
  if (cta == 0)
    report_requests(a);
  Walk<M, BN> walk{find_share<kSimtThreads>(a, M, cta, ctas, sm.scratch)};
  const T *q = static_cast<const T *>(a.q);
  const T *kc = static_cast<const T *>(a.kc), *vc = static_cast<const T *>(a.vc);
  const float scale = a.scale * kLog2e;
  const int col = (tid % (kSimtThreads / RG)), rg = tid / (kSimtThreads / RG);
  Segment s;
  for (int seg = 0; walk.next(a, &s); ++seg) {
    __syncthreads();
    for (int x = tid; x < M * (D / VEC); x += kSimtThreads) {
      const int r = x / (D / VEC), c = x % (D / VEC);
      uint4 u = make_uint4(0, 0, 0, 0);
      if (r < s.rows) {
        const RowAt at = row_at(a, s.row0, s.r0, s.h, r);
        u = *reinterpret_cast<const uint4 *>(q + at.token * a.q_row + at.head * a.q_head + c * VEC);
      }
      widen<T>(u, &sm.q[r][c * VEC]);
    }
    if (tid < M) {
      sm.m[tid] = -INFINITY;
      sm.l[tid] = 0.f;
      sm.seen[tid] = min(s.seen(tid, a.g), s.kv);
    }
    float o[RPT][CPT];
#pragma unroll
    for (int r = 0; r < RPT; ++r)
#pragma unroll
      for (int c = 0; c < CPT; ++c) o[r][c] = 0.f;
    for (int t = s.t0; t < s.t1; ++t) {
      const int key0 = t * BN, nk = min(BN, s.keys - key0);
      __syncthreads();
      if (tid < nk) {
        int off;
        const int id = page_of(a, s.i, key0 + tid, &off);
        sm.krow[tid] = cache_row(a, a.ks, id, off, s.h);
        sm.vrow[tid] = cache_row(a, a.vs, id, off, s.h);
      }
      __syncthreads();
      for (int x = tid; x < BN * (D / VEC); x += kSimtThreads) {
        const int k = x / (D / VEC), c = x % (D / VEC);
        uint4 ku = make_uint4(0, 0, 0, 0), vu = ku;
        if (k < nk) {
          ku = *reinterpret_cast<const uint4 *>(kc + sm.krow[k] + c * VEC);
          vu = *reinterpret_cast<const uint4 *>(vc + sm.vrow[k] + c * VEC);
        }
        widen<T>(ku, &sm.k[k][c * VEC]);
        widen<T>(vu, &sm.v[k][c * VEC]);
      }
      __syncthreads();
      {
        const int k = tid % BN, r0 = (tid / BN) * (M / 2);
        float acc[M / 2] = {};
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
          const float4 x = *reinterpret_cast<const float4 *>(&sm.k[k][d]);
#pragma unroll
          for (int r = 0; r < M / 2; ++r) {
            const float4 y = *reinterpret_cast<const float4 *>(&sm.q[r0 + r][d]);
            acc[r] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, acc[r]))));
          }
        }
#pragma unroll
        for (int r = 0; r < M / 2; ++r)
          sm.p[r0 + r][k] = key0 + k < sm.seen[r0 + r] ? acc[r] * scale : -INFINITY;
      }
      __syncthreads();
      // Running maximum and sum: a warp has four rows, two keys per lane.
      for (int r = warp; r < M; r += kSimtThreads / 32) {
        const float x = sm.p[r][lane], y = sm.p[r][lane + 32];
        float mx = fmaxf(x, y);
        for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float old = sm.m[r], m = fmaxf(old, mx), ref = m == -INFINITY ? 0.f : m;
        const float px = exp2f(x - ref), py = exp2f(y - ref);
        float sum = px + py;
        for (int w = 16; w > 0; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        sm.p[r][lane] = px;
        sm.p[r][lane + 32] = py;
        __syncwarp();
        if (lane == 0) {
          const float fix = exp2f(old - ref);
          sm.m[r] = m;
          sm.l[r] = fmaf(sm.l[r], fix, sum);
          sm.fix[r] = fix;
        }
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < RPT; ++r)
#pragma unroll
        for (int c = 0; c < CPT; ++c) o[r][c] *= sm.fix[rg * RPT + r];
      // A value that a row does not see must not reach its sums, not even
      // times zero: it may be NaN.
      const bool edge = key0 + nk > s.least;
      for (int k = 0; k < nk; ++k) {
        float v[CPT];
#pragma unroll
        for (int c = 0; c < CPT; ++c) v[c] = sm.v[k][col + c * kSimtThreads];
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
          if (edge && key0 + k >= sm.seen[rg * RPT + r]) continue;
          const float p = sm.p[rg * RPT + r][k];
#pragma unroll
          for (int c = 0; c < CPT; ++c) o[r][c] = fmaf(p, v[c], o[r][c]);
        }
      }
    }
    __syncthreads();
    if (s.whole()) {
#pragma unroll
      for (int r = 0; r < RPT; ++r) {
        const int rr = rg * RPT + r;
        if (rr >= s.rows) continue;
        const RowAt at = row_at(a, s.row0, s.r0, s.h, rr);
        const float l = sm.l[rr], inv = l == 0.f ? 0.f : 1.f / l;
        T *out = static_cast<T *>(a.out) + (at.token * a.Hq + at.head) * D;
#pragma unroll
        for (int c = 0; c < CPT; ++c) from_float(out + col + c * kSimtThreads, o[r][c] * inv);
        if (col == 0 && a.lse)
          a.lse[at.token * a.Hq + at.head] =
              l == 0.f ? -INFINITY : (sm.m[rr] + log2f(l)) * kLn2;
      }
    } else {
      float *part = a.part + note_partial(a, s, cta, seg) * part_floats(M, D);
      if (tid < M) {
        part[tid] = sm.m[tid];
        part[M + tid] = sm.l[tid];
      }
#pragma unroll
      for (int r = 0; r < RPT; ++r)
#pragma unroll
        for (int c = 0; c < CPT; ++c)
          part[2 * M + (rg * RPT + r) * D + col + c * kSimtThreads] = o[r][c];
    }
  }
}

constexpr int kJoinThreads = 256;

// Joins the partial sums of a unit: the block of the CTA that has the unit's
// beginning. Its other pieces are the first segments of the CTAs behind. A
// warp takes a row; sums go in the order of the keys.
template <typename T, int D>
__global__ void __launch_bounds__(kJoinThreads) attend_join_kernel(Args a, int M, int ctas) {
  __shared__ int slots[kMaxCtas];
  __shared__ int n_slots;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int which = 0; which < 2; ++which) {
    const int mine = blockIdx.x * 2 + which;
    const Desc d = a.desc[mine];
    if (d.tiles == 0 || d.t0 != 0) continue;
    __syncthreads();
    if (warp == 0) {
      int n = 1;
      if (lane == 0) slots[0] = mine;
      bool more = true;
      for (int c0 = blockIdx.x + 1; more && c0 < ctas; c0 += 32) {
        const int c = c0 + lane;
        Desc e{};
        if (c < ctas) e = a.desc[c * 2];
        const bool in = e.tiles > 0 && e.i == d.i && e.h == d.h && e.rt == d.rt;
        const unsigned ins = __ballot_sync(0xffffffffu, in);
        if (in) slots[n + __popc(ins & ((1u << lane) - 1))] = c * 2;
        n += __popc(ins);
        more = !__any_sync(0xffffffffu, in && e.t1 == e.tiles);
      }
      if (lane == 0) n_slots = n;
    }
    __syncthreads();
    const int n = n_slots;
    const Request req = request(a, d.i);
    const int rows = min(M, req.n * a.g - d.rt * M);
    for (int r = blockIdx.y * (kJoinThreads / 32) + warp; r < rows;
         r += gridDim.y * (kJoinThreads / 32)) {
      float mx = -INFINITY;
      for (int k = lane; k < n; k += 32)
        mx = fmaxf(mx, a.part[slots[k] * part_floats(M, D) + r]);
      for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
      const float ref = mx == -INFINITY ? 0.f : mx;
      float l = 0.f, o[D / 32] = {};
#pragma unroll 4
      for (int k = 0; k < n; ++k) {
        const float *p = a.part + slots[k] * part_floats(M, D);
        const float f = exp2f(p[r] - ref);
        l = fmaf(p[M + r], f, l);
        const float *src = p + 2 * M + r * D + lane * (D / 32);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) o[c] = fmaf(src[c], f, o[c]);
      }
      const RowAt at = row_at(a, req.row0, d.rt * M, d.h, r);
      const float inv = l == 0.f ? 0.f : 1.f / l;
      T *out = static_cast<T *>(a.out) + (at.token * a.Hq + at.head) * D + lane * (D / 32);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) from_float(out + c, o[c] * inv);
      if (lane == 0 && a.lse)
        a.lse[at.token * a.Hq + at.head] =
            l == 0.f ? -INFINITY : (mx + log2f(l)) * kLn2;
    }
  }
}

template <typename T, int D>
pair_status run_simt(const Args &a, cudaStream_t s) {
  const int smem = sizeof(SimtSmem<D>);
  PAIR_CUDA_TRY(cudaFuncSetAttribute(attend_simt_kernel<T, D>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const int per_sm = D <= 128 ? 2 : 1;
  const int ctas = min(kMaxCtas, per_sm * sm_count());
  PAIR_BEGIN("attend_simt", s);
  attend_simt_kernel<T, D><<<ctas, kSimtThreads, smem, s>>>(a);
  PAIR_LAUNCH_CHECK(s);
  return launch_join(a, D, kSimtRows, ctas, sizeof(T) == 2 ? PAIR_BF16 : PAIR_F32, s);
}

template <typename T, int D>
pair_status run_join(const Args &a, int M, int ctas, cudaStream_t s) {
  PAIR_BEGIN("attend_join", s);
  attend_join_kernel<T, D><<<dim3(ctas, M / 16), kJoinThreads, 0, s>>>(a, M, ctas);
  PAIR_LAUNCH_CHECK(s);
  return PAIR_OK;
}

template <typename F>
pair_status by_size(int D, F f) {
  if (D == 64) return f(std::integral_constant<int, 64>());
  if (D == 128) return f(std::integral_constant<int, 128>());
  return f(std::integral_constant<int, 256>());
}

size_t desc_bytes() { return kMaxCtas * 2 * sizeof(Desc); }

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return 1;
  }
  return n;
}

pair_status launch_simt(const Args &a, int D, pair_dtype dt, cudaStream_t s) {
  return by_size(D, [&](auto d) {
    return dt == PAIR_BF16 ? run_simt<__nv_bfloat16, decltype(d)::value>(a, s)
                           : run_simt<float, decltype(d)::value>(a, s);
  });
}

pair_status launch_join(const Args &a, int D, int M, int ctas, pair_dtype dt, cudaStream_t s) {
  return by_size(D, [&](auto d) {
    return dt == PAIR_BF16 ? run_join<__nv_bfloat16, decltype(d)::value>(a, M, ctas, s)
                           : run_join<float, decltype(d)::value>(a, M, ctas, s);
  });
}

}  // namespace attend
}  // namespace pairk

using namespace pairk;
using namespace pairk::attend;

extern "C" {

size_t pair_attend_workspace_size(int32_t R, int32_t Hq, int32_t Hkv, int32_t D, pair_dtype dt) {
  if (R < 1 || Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || (D != 64 && D != 128 && D != 256) ||
      (dt != PAIR_F32 && dt != PAIR_BF16))
    return 0;
  return desc_bytes() + kMaxCtas * 2 * part_floats(kMaxRows, D) * sizeof(float);
}

pair_status pair_attend_paged(int64_t T, int32_t R, int32_t Hq, int32_t Hkv, int32_t D,
                              pair_dtype dt, const void *q, int64_t q_row, int64_t q_head,
                              const void *k_cache, pair_cache_strides ks, const void *v_cache,
                              pair_cache_strides vs, int32_t num_pages, int32_t page_size,
                              const int32_t *block_table, int32_t table_width,
                              const int32_t *kv_len, const int32_t *cu_new, float scale,
                              int32_t max_new, void *out, float *lse, void *ws,
                              size_t ws_bytes, int32_t *dev_err, pair_stream_t stream) {
  reset_launches();
  if (T < 1 || T > INT32_MAX || R < 1 || Hkv < 1 || Hq < Hkv || Hq % Hkv != 0 || !q || !k_cache ||
      !v_cache || num_pages < 1 || page_size < 1 || !block_table || table_width < 1 || !kv_len ||
      !cu_new || !out || !(fabsf(scale) <= 3.0e38f) || max_new < 0 || (dt != PAIR_F32 && dt != PAIR_BF16) ||
      T * (Hq / Hkv) > INT32_MAX)
    return PAIR_ERR_INVALID_ARG;
  const int per = dt == PAIR_BF16 ? 8 : 4;  // elements of 16 bytes
  const int64_t strides[] = {q_row, q_head, ks.for_page, ks.for_token, ks.for_head, vs.for_page,
                             vs.for_token, vs.for_head};
  for (const int64_t x : strides)
    if (x % per != 0) return PAIR_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(out, 16))
    return PAIR_ERR_INVALID_ARG;
  const size_t need = pair_attend_workspace_size(R, Hq, Hkv, D, dt);
  if (need == 0) return PAIR_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < need || !aligned(ws, 256)) return PAIR_ERR_WORKSPACE;
  const pair_status dv = check_device();
  if (dv != PAIR_OK) return dv;
  const Args a{T,
               R,
               Hq,
               Hkv,
               Hq / Hkv,
               -1,
               INT32_MAX,
               q,
               q_row,
               q_head,
               k_cache,
               v_cache,
               ks,
               vs,
               num_pages,
               page_size,
               block_table,
               table_width,
               kv_len,
               cu_new,
               scale,
               out,
               lse,
               static_cast<Desc *>(ws),
               reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + desc_bytes()),
               dev_err};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (dt == PAIR_F32) return launch_simt(a, D, dt, s);
  // Which kernel a chunk goes to is decided by its rows, on the device; a
  // launch is left out where the host knows that no chunk can be its.
  const int64_t most_rows = (int64_t)(max_new > 0 && max_new < T ? max_new : T) * a.g;
  if (most_rows <= kFewRows || !many_applies(a, D)) return launch_few(a, D, s);
  if (R == 1) return launch_many(a, D, s);
  Args few = a, many = a;
  few.rows_upto = kFewRows;
  many.rows_over = kFewRows;
  const pair_status st = launch_few(few, D, s);
  return st != PAIR_OK ? st : launch_many(many, D, s);
}

}  // extern "C"
