// pair_verify_drafts: drafted tokens against the target's probabilities, and
// the token that follows the accepted ones (speculative sampling).
#include <cuda_bf16.h>

#include "pair_common.cuh"
#include "tc_ptx.cuh"

namespace pairk {
namespace {

using namespace tc;

constexpr int kVerifyThreads = 512;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyMaxCluster = 8;

template <typename T>
struct VerifyArgs {
  int64_t T_rows;
  int32_t R, V, C;  // C: CTAs per request
  const T *p, *q;
  int64_t p_row, q_row;
  const int32_t *ids, *cu;
  const float *u, *u_draw;
  int32_t *out_ids;
  float *logp;
  int32_t *n_emit, *dev_err;
};

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// Weights in units of 2^-40, w = floor(2^40 x) for x in [0, 1], summed over a
// vector: fp32 additions that round towards zero leave the upper and the lower
// 20 bits in the significand (8 + x in steps of 2^-20, then what is left of x
// plus 2^-17 in steps of 2^-40), where integer additions read them off. The
// sums of up to 2^22 weights fit 63 bits and, being integers, do not depend on
// their order. (Conversions to 64-bit integers go through the fp64 pipe: 80 %
// busy with them, 256 rows of p and q took 104 us.)
struct Weight {
  uint32_t hi, lo;  // bits of the two sums, without their constants
  __device__ __forceinline__ long long value() const {
    return ((long long)hi << 20) + lo;
  }
};
__device__ __forceinline__ Weight fixed_weight(float x) {
  const float t = __fadd_rz(x, 8.f);
  const float rest = x - (t - 8.f);
  return {__float_as_uint(t) - 0x41000000u, __float_as_uint(__fadd_rz(rest, 0x1p-17f)) - 0x37000000u};
}
// a - b held to [0, 1]; NaN gives 0.
__device__ __forceinline__ float sub_sat(float a, float b) {
  float o;
  asm("sub.sat.f32 %0, %1, %2;" : "=f"(o) : "f"(a), "f"(b));
  return o;
}

// VEC consecutive values from element e of a row of V (elements outside it
// are 0): one 16-byte load where the address allows it.
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T *row, int e, int V, float (&x)[VEC]) {
  const T *at = row + e;
  if (e >= 0 && e + VEC <= V && (reinterpret_cast<uintptr_t>(at) & 15u) == 0) {
    const uint4 r = __ldg(reinterpret_cast<const uint4 *>(at));
    const T *t = reinterpret_cast<const T *>(&r);
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[k] = as_float(t[k]);
  } else {
#pragma unroll
    for (int k = 0; k < VEC; ++k) x[k] = e + k >= 0 && e + k < V ? as_float(at[k]) : 0.f;
  }
}

// What a draw is made from: p alone, p - q, or p without the draft.
template <typename T>
struct Source {
  const T *p, *q;
  int V, skip;
  static constexpr int VEC = 16 / sizeof(T);
  __device__ __forceinline__ void load(int e, float (&x)[VEC]) const {
    load_vec<T, VEC>(p, e, V, x);
    if (q) {
      float y[VEC];
      load_vec<T, VEC>(q, e, V, y);
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[k] = sub_sat(x[k], y[k]);
    } else {
#pragma unroll
      for (int k = 0; k < VEC; ++k) x[k] = e + k == skip ? 0.f : __saturatef(x[k]);
    }
  }
  __device__ __forceinline__ long long sum(int e) const {
    float x[VEC];
    load(e, x);
    Weight s{0, 0};
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const Weight w = fixed_weight(x[k]);
      s.hi += w.hi;
      s.lo += w.lo;
    }
    return s.value();
  }
};

// One cluster of C CTAs per request. Every CTA decides the request's drafts
// for itself (a handful of gathers), then sums the weights of its share of
// the vocabulary; each warp has a contiguous segment. The shares' sums meet
// through distributed shared memory, and the one warp whose segment holds the
// threshold goes over that segment again. Bound by HBM: one row of p, and of q
// where a draft was refused, per request; C CTAs bring a single request's row
// in when there are few.
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_kernel(VerifyArgs<T> a) {
  constexpr int VEC = Source<T>::VEC;
  __shared__ int s_first, s_bad;
  __shared__ long long s_warp[kVerifyWarps];
  __shared__ long long s_cta[2][kVerifyMaxCluster];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = a.C, rank = blockIdx.x % C, i = blockIdx.x / C;
  const int lo = a.cu[i], hi = a.cu[i + 1];
  const bool sane = lo >= 0 && hi >= lo && hi <= a.T_rows;
  if (rank == 0 && i == a.R - 1 && sane) {
    for (int64_t t = hi + tid; t < a.T_rows; t += kVerifyThreads) {
      a.out_ids[t] = -1;
      if (a.logp) a.logp[t] = 0.f;
    }
  }
  if (!sane || hi == lo) {
    if (rank == 0 && tid == 0) {
      a.n_emit[i] = 0;
      if (!sane) flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
    }
    return;  // the whole cluster
  }
  // Drafts: the first one refused, or the last row.
  if (warp == 0) {
    const int K = hi - lo - 1;
    int first = K, bad = 0;
    for (int j0 = 0; j0 < K && first == K; j0 += 32) {
      const int j = j0 + lane;
      bool refuse = false, out = false;
      if (j < K) {
        const int y = a.ids[lo + j + 1];
        out = y < 0 || y >= a.V;
        if (out) {
          refuse = true;
        } else {
          const float py = as_float(a.p[(lo + j) * a.p_row + y]);
          const float qy = a.q ? as_float(a.q[(lo + j) * a.q_row + y]) : 1.f;
          refuse = !(a.u[lo + j] * qy < py);
        }
      }
      const unsigned any = __ballot_sync(0xffffffffu, refuse);
      if (any) {
        first = j0 + __ffs(any) - 1;
        bad = __shfl_sync(0xffffffffu, (int)out, __ffs(any) - 1);
      }
    }
    if (lane == 0) {
      s_first = first;
      s_bad = bad;
    }
  }
  __syncthreads();
  const int first = s_first, row = lo + first;
  const bool drafted = row + 1 < hi;
  const T *prow = a.p + row * a.p_row;
  Source<T> src{prow, drafted && a.q ? a.q + row * a.q_row : nullptr, a.V,
                drafted && !a.q && !s_bad ? a.ids[row + 1] : -1};
  if (rank == 0) {
    if (s_bad && tid == 0) flag_error(a.dev_err, PAIR_DEV_ERR_TARGET_RANGE);
    for (int t = lo + tid; t < hi; t += kVerifyThreads) {
      if (t == row) continue;
      const int y = t < row ? a.ids[t + 1] : -1;
      a.out_ids[t] = y;
      if (a.logp) a.logp[t] = t < row ? logf(as_float(a.p[t * a.p_row + y])) : 0.f;
    }
  }
  // Segments in whole vectors, counted from the 16-byte boundary at or before
  // the row of p.
  const int mis = (int)((reinterpret_cast<uintptr_t>(prow) & 15u) / sizeof(T));
  const int n_vec = (int)ceil_div((int64_t)a.V + mis, VEC);
  const int n_seg = C * kVerifyWarps;
  const int per = (n_vec + n_seg - 1) / n_seg;
  const int v0 = min((rank * kVerifyWarps + warp) * per, n_vec), v1 = min(v0 + per, n_vec);
  for (int pass = 0; pass < 2; ++pass) {
    long long sum = 0;
#pragma unroll 4
    for (int v = v0 + lane; v < v1; v += 32) sum += src.sum(v * VEC - mis);
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) s_warp[warp] = sum;
    __syncthreads();
    if (warp == 0) {
      long long x = lane < kVerifyWarps ? s_warp[lane] : 0;
      for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
      if (lane < C) {
        const uint32_t to = mapa(smem_u32(&s_cta[pass][rank]), lane);
        asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(to), "l"(x) : "memory");
      }
    }
    cluster_sync();
    long long total = 0, before = 0;
    for (int c = 0; c < C; ++c) {
      if (c == rank) before = total;
      total += s_cta[pass][c];
    }
    if (total == 0) {
      if (pass == 0) {  // nothing left of the difference: p alone
        src.q = nullptr;
        src.skip = -1;
        __syncthreads();
        continue;
      }
      if (rank == 0 && tid == 0) {
        a.out_ids[row] = -1;
        if (a.logp) a.logp[row] = 0.f;
        a.n_emit[i] = first;
        flag_error(a.dev_err, PAIR_DEV_ERR_PROBABILITY);
      }
      return;
    }
    long long at = (long long)((double)a.u_draw[i] * (double)total);
    at = max(min(at, total - 1), 0ll);
    for (int k = 0; k < warp; ++k) before += s_warp[k];
    if (at < before || at >= before + s_warp[warp]) return;
    // This warp's segment again, kAhead pieces of 32 vectors in flight.
    constexpr int kAhead = 8;
    for (int vb = v0; vb < v1; vb += 32 * kAhead) {
      long long mine[kAhead], all[kAhead];
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        const int v = vb + x * 32 + lane;
        mine[x] = v < v1 ? src.sum(v * VEC - mis) : 0;
        all[x] = mine[x];
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int x = 0; x < kAhead; ++x) all[x] += __shfl_xor_sync(0xffffffffu, all[x], o);
#pragma unroll
      for (int x = 0; x < kAhead; ++x) {
        if (at >= before + all[x]) {
          before += all[x];
          continue;
        }
        long long incl = mine[x];
        for (int o = 1; o < 32; o <<= 1) {
          const long long y = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += y;
        }
        long long c = before + incl - mine[x];
        if (at >= c && at < c + mine[x]) {
          const int e = (vb + x * 32 + lane) * VEC - mis;
          float f[VEC];
          src.load(e, f);
          int tok = e;
#pragma unroll
          for (int k = 0; k < VEC; ++k) {  // the first k whose sum passes `at`
            c += fixed_weight(f[k]).value();
            if (c <= at) tok = e + k + 1;
          }
          a.out_ids[row] = tok;
          if (a.logp) a.logp[row] = logf(as_float(prow[tok]));
          a.n_emit[i] = first + 1;
        }
        return;
      }
    }
    return;
  }
}

template <typename T>
pair_status launch_verify(VerifyArgs<T> a, cudaStream_t s) {
  // CTAs per request: a full cluster while the requests leave SMs idle.
  int C = kVerifyMaxCluster;
  while (C > 1 && (int64_t)a.R * C > 8 * 152) C /= 2;
  cudaLaunchConfig_t cfg = {};
  a.C = C;
  cfg.gridDim = dim3((unsigned)C * (unsigned)a.R, 1, 1);
  cfg.blockDim = dim3(kVerifyThreads, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = C;
  attr.val.clusterDim.y = 1;
  attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  PAIR_BEGIN("verify_drafts", s);
  if (cudaLaunchKernelEx(&cfg, verify_kernel<T>, a) != cudaSuccess) {
    cudaGetLastError();
    return PAIR_ERR_CUDA;
  }
  PAIR_LAUNCH_CHECK(s);
  return PAIR_OK;
}

}  // namespace
}  // namespace pairk

using namespace pairk;

extern "C" pair_status pair_verify_drafts(int64_t T, int32_t R, int32_t V, pair_dtype dt,
                                          const void *p, int64_t p_row, const void *q,
                                          int64_t q_row, const int32_t *ids,
                                          const int32_t *cu_new, const float *u,
                                          const float *u_draw, int32_t *out_ids, float *logp,
                                          int32_t *n_emit, int32_t *dev_err,
                                          pair_stream_t stream) {
  reset_launches();
  if (T < 1 || T > INT32_MAX || R < 1 || R > (1 << 27) || V < 1 || V > (1 << 22) ||
      (dt != PAIR_F32 && dt != PAIR_BF16) || !p || !ids || !cu_new || !u || !u_draw ||
      !out_ids || !n_emit || p_row < V || (q && q_row < V))
    return PAIR_ERR_INVALID_ARG;
  const pair_status dv = check_device();
  if (dv != PAIR_OK) return dv;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (dt == PAIR_BF16)
    return launch_verify<__nv_bfloat16>(
        {T, R, V, 1, static_cast<const __nv_bfloat16 *>(p), static_cast<const __nv_bfloat16 *>(q),
         p_row, q_row, ids, cu_new, u, u_draw, out_ids, logp, n_emit, dev_err}, s);
  return launch_verify<float>({T, R, V, 1, static_cast<const float *>(p),
                               static_cast<const float *>(q), p_row, q_row, ids, cu_new, u,
                               u_draw, out_ids, logp, n_emit, dev_err}, s);
}
