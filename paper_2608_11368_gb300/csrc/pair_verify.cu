// pair_verify_drafts: drafted tokens against the target's probabilities, and
// the token that follows the accepted ones (speculative sampling).
#include <cuda_bf16.h>

#include <atomic>

#include "pair_common.cuh"
#include "tc_ptx.cuh"

namespace pairk {
namespace {

using namespace tc;

constexpr int kVerifyWarps = 8;  // that read probabilities; one more controls
constexpr int kVerifyThreads = (kVerifyWarps + 1) * 32;
constexpr int kVerifyMaxCluster = 16;
constexpr int kVerifyLeast = 2048;  // values of a row worth a CTA of its own

template <typename T>
struct VerifyArgs {
  int64_t T_rows;
  int32_t R, V, C, clusters;  // C: CTAs of a cluster
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
  uint32_t hi = 0, lo = 0;  // bits of the two sums, constants included
  int n = 0;                // values added (at most 2^12, so that hi fits)
  __device__ __forceinline__ void add(float x, float y) {
    float2 t, s, r, u;
    const float2 v = {x, y}, c8 = {8.f, 8.f}, m8 = {-8.f, -8.f}, one = {-1.f, -1.f};
    const float2 c17 = {0x1p-17f, 0x1p-17f};
#define PAIR_U64(f) reinterpret_cast<const uint64_t &>(f)
    asm("add.rz.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<uint64_t &>(t))
        : "l"(PAIR_U64(v)), "l"(PAIR_U64(c8)));
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<uint64_t &>(s))
        : "l"(PAIR_U64(t)), "l"(PAIR_U64(m8)));
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<uint64_t &>(r))
        : "l"(PAIR_U64(s)), "l"(PAIR_U64(one)), "l"(PAIR_U64(v)));
    asm("add.rz.f32x2 %0, %1, %2;"
        : "=l"(reinterpret_cast<uint64_t &>(u))
        : "l"(PAIR_U64(r)), "l"(PAIR_U64(c17)));
#undef PAIR_U64
    hi += __float_as_uint(t.x) + __float_as_uint(t.y);
    lo += __float_as_uint(u.x) + __float_as_uint(u.y);
    n += 2;
  }
  __device__ __forceinline__ long long value() const {
    return ((long long)(hi - n * 0x41000000u) << 20) + (lo - n * 0x37000000u);
  }
};
__device__ __forceinline__ long long fixed_weight(float x) {
  Weight w;
  w.add(x, 0.f);
  return w.value();
}
// a - b held to [0, 1]; NaN gives 0.
__device__ __forceinline__ float sub_sat(float a, float b) {
  float o;
  asm("sub.sat.f32 %0, %1, %2;" : "=f"(o) : "f"(a), "f"(b));
  return o;
}

// What a draw is made from: p alone, p - q, or p without the draft. The row is
// cut into vectors of 16 bytes, counted from the boundary at or before its
// first element; those that lie in it whole are loaded whole (q's too, where it
// lies the same way), kPieces of them per lane in flight.
constexpr int kPieces = 4;
template <typename T>
struct Source {
  static constexpr int VEC = 16 / sizeof(T);
  const T *p, *q;
  int V, skip;
  int mis, n_vec, whole0, whole1;  // vectors [whole0, whole1) lie in the row
  int skip_vec;

  __device__ __forceinline__ Source(const T *p_, const T *q_, int V_, int skip_)
      : p(p_), q(q_), V(V_), skip(skip_) {
    mis = (int)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
    n_vec = (V + mis + VEC - 1) / VEC;
    whole0 = mis ? 1 : 0;
    whole1 = (V + mis) / VEC;
    if (q && ((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15u) != 0)
      whole1 = 0;
    skip_vec = skip < 0 ? -1 : (skip + mis) / VEC;
  }
  // One vector, element by element; elements outside the row are 0.
  __device__ __forceinline__ void load(int v, float (&x)[VEC]) const {
#pragma unroll
    for (int k = 0; k < VEC; ++k) {
      const int e = v * VEC - mis + k;
      x[k] = 0.f;
      if (e >= 0 && e < V && e != skip)
        x[k] = sub_sat(as_float(p[e]), q ? as_float(q[e]) : 0.f);
    }
  }
  __device__ __forceinline__ long long odd_sum(int v) const {
    float f[VEC];
    load(v, f);
    Weight s;
#pragma unroll
    for (int k = 0; k < VEC; k += 2) s.add(f[k], f[k + 1]);
    return s.value();
  }
  static __device__ __forceinline__ void add(const uint4 &a, const uint4 &b, Weight &s) {
    const T *t = reinterpret_cast<const T *>(&a), *u = reinterpret_cast<const T *>(&b);
#pragma unroll
    for (int k = 0; k < VEC; k += 2)
      s.add(sub_sat(as_float(t[k]), as_float(u[k])),
            sub_sat(as_float(t[k + 1]), as_float(u[k + 1])));
  }
  // The lane's vectors vb + 32 x + lane below v1, x < kPieces; bit x of the answer:
  // this one is to be read element by element.
  __device__ __forceinline__ unsigned fetch(int vb, int v1, uint4 (&a)[kPieces],
                                            uint4 (&b)[kPieces]) const {
    const int lane = threadIdx.x & 31;
    const uint4 *pv = reinterpret_cast<const uint4 *>(p - mis);
    const uint4 *qv = reinterpret_cast<const uint4 *>(q - mis);
    unsigned odd = 0;
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      const int v = vb + 32 * x + lane;
      const bool in = v >= whole0 && v < whole1 && v < v1 && v != skip_vec;
      a[x] = b[x] = make_uint4(0, 0, 0, 0);
      if (in) a[x] = __ldg(pv + v);
      if (in && q) b[x] = __ldg(qv + v);
      if (!in && v < v1) odd |= 1u << x;
    }
    return odd;
  }
  // Sums of these vectors, and the sum of all of the lane's in [v0, v1).
  __device__ __forceinline__ void pieces(int vb, int v1, long long (&s)[kPieces]) const {
    uint4 a[kPieces], b[kPieces];
    const unsigned odd = fetch(vb, v1, a, b);
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
      Weight w;
      add(a[x], b[x], w);
      s[x] = odd >> x & 1 ? odd_sum(vb + 32 * x + (threadIdx.x & 31)) : w.value();
    }
  }
  __device__ __forceinline__ long long segment(int v0, int v1) const {
    long long total = 0;
    for (int vb = v0; vb < v1; vb += 32 * kPieces) {
      uint4 a[kPieces], b[kPieces];
      unsigned odd = fetch(vb, v1, a, b);
      Weight w;
#pragma unroll
      for (int x = 0; x < kPieces; ++x) add(a[x], b[x], w);
      total += w.value();  // (the odd ones' places hold zeros)
      for (; odd; odd &= odd - 1) total += odd_sum(vb + 32 * (__ffs(odd) - 1) + (threadIdx.x & 31));
    }
    return total;
  }
};

// By a warp: the token in whose weight `at` falls, the vectors [v0, v1) of the
// row coming after weights of sum `before`; -1 in the lanes that do not have it.
template <typename T>
__device__ __forceinline__ int find(const Source<T> &src, int v0, int v1, long long before,
                                    long long at) {
  constexpr int VEC = Source<T>::VEC;
  const int lane = threadIdx.x & 31;
  for (int vb = v0; vb < v1; vb += 32 * kPieces) {
    long long mine[kPieces], all[kPieces];
    src.pieces(vb, v1, mine);
#pragma unroll
    for (int x = 0; x < kPieces; ++x) all[x] = mine[x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int x = 0; x < kPieces; ++x) all[x] += __shfl_xor_sync(0xffffffffu, all[x], o);
#pragma unroll
    for (int x = 0; x < kPieces; ++x) {
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
      if (at < c || at >= c + mine[x]) return -1;
      const int v = vb + x * 32 + lane;
      float f[VEC];
      src.load(v, f);
      int tok = v * VEC - src.mis;
#pragma unroll
      for (int k = 0; k < VEC; ++k) {  // the first element whose sum passes `at`
        c += fixed_weight(f[k]);
        tok += c <= at;
      }
      return tok;
    }
  }
  return -1;
}

// What a request's drafts came to.
struct Decision {
  int lo, hi;  // rows of the chunk (hi <= lo: none)
  int row;     // of the first draft refused, or the last one
  int bad;     // that draft is no token
  int skip;    // the token left out of the draw where the drafter has no probabilities
};

// By one warp, every lane gets it.
template <typename T>
__device__ Decision decide(const VerifyArgs<T> &a, int i) {
  const int lane = threadIdx.x & 31;
  const int lo = a.cu[i], hi = a.cu[i + 1];
  if (lo < 0 || hi < lo || hi > a.T_rows) return {0, -1, 0, 0, -1};
  Decision d{lo, hi, hi - 1, 0, -1};
  for (int t0 = lo; t0 < hi - 1; t0 += 32) {
    const int t = t0 + lane;
    bool refuse = false;
    int y = 0;
    if (t < hi - 1) {
      y = a.ids[t + 1];
      refuse = true;
      if (y >= 0 && y < a.V) {
        const float py = as_float(a.p[t * a.p_row + y]);
        const float qy = a.q ? as_float(a.q[t * a.q_row + y]) : 1.f;
        refuse = !(a.u[t] * qy < py);
      }
    }
    const unsigned any = __ballot_sync(0xffffffffu, refuse);
    if (any) {
      d.row = t0 + __ffs(any) - 1;
      y = __shfl_sync(0xffffffffu, y, __ffs(any) - 1);
      d.bad = y < 0 || y >= a.V;
      d.skip = a.q || d.bad ? -1 : y;
      break;
    }
  }
  return d;
}

// Clusters of C CTAs, each cluster one request after another. The reading
// warps of its CTAs sum the weights of a share of the vocabulary each, a
// contiguous segment per warp; the CTAs' sums meet through distributed shared
// memory. A ninth warp of each CTA decides the next request's drafts (three
// dependent loads) while the others read, writes the accepted tokens, and,
// where the draw falls into its CTA, goes over that warp's segment again while
// the others are at the next request. Bound by HBM: one row of p, and of q where
// a draft was refused, per request. 256 rows of 151,936 of both in fp32: 59 us,
// 4.6 TB/s (with every warp doing everything, a request per cluster, 84). Not
// faster: 2, 3 or 8 vectors per lane in flight, vectors through shared memory, a
// fourth CTA per SM, reading warps a request ahead of the exchange (60 to 120 us);
// the clusters' last round, which is not full, costs as much as a full one.
template <typename T>
__global__ void __launch_bounds__(kVerifyThreads) verify_kernel(VerifyArgs<T> a) {
  __shared__ Decision s_dec[2];
  __shared__ long long s_warp[2][kVerifyWarps];
  __shared__ long long s_cta[2][kVerifyMaxCluster];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int C = a.C, rank = blockIdx.x % C, cluster = blockIdx.x / C;
  const bool control = warp == kVerifyWarps;
  cluster_arrive();
  if (blockIdx.x == gridDim.x - 1) {  // rows that no request owns
    const auto clear = [&](int64_t t0, int64_t t1) {
      for (int64_t t = t0 + tid; t < t1; t += kVerifyThreads) {
        a.out_ids[t] = -1;
        if (a.logp) a.logp[t] = 0.f;
      }
    };
    clear(0, min((int64_t)a.cu[0], a.T_rows));
    clear(max(0, a.cu[a.R]), a.T_rows);
  }
  if (control) {
    const Decision d = decide(a, cluster);
    if (lane == 0) s_dec[0] = d;
  }
  __syncthreads();
  // Every CTA of the cluster runs before its shared memory is written to. (They
  // arrive at their start, so the first decision's loads cover the wait.)
  cluster_wait();
  int round = 0;  // of the exchange, alternating between two buffers
  for (int i = cluster, it = 0; i < a.R; i += a.clusters, ++it) {
    const Decision d = s_dec[it & 1];
    const bool empty = d.hi <= d.lo;
    if (control) {
      if (i + a.clusters < a.R) {
        const Decision next = decide(a, i + a.clusters);
        if (lane == 0) s_dec[(it + 1) & 1] = next;
      }
      if (rank == 0) {
        if (empty && lane == 0) {
          a.n_emit[i] = 0;
          if (d.hi < d.lo) flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
        }
        if (d.bad && lane == 0) flag_error(a.dev_err, PAIR_DEV_ERR_TARGET_RANGE);
        for (int t = d.lo + lane; t < d.hi; t += 32) {
          if (t == d.row) continue;
          const int y = t < d.row ? a.ids[t + 1] : -1;
          a.out_ids[t] = y;
          if (a.logp) a.logp[t] = t < d.row ? logf(as_float(a.p[t * a.p_row + y])) : 0.f;
        }
      }
    }
    if (empty) {
      __syncthreads();
      continue;
    }
    const T *prow = a.p + d.row * a.p_row;
    Source<T> src(prow, d.row + 1 < d.hi && a.q ? a.q + d.row * a.q_row : nullptr, a.V, d.skip);
    const int n_vec = src.n_vec;
    const int n_seg = C * kVerifyWarps;
    const int per = (n_vec + n_seg - 1) / n_seg;
    for (int pass = 0; pass < 2; ++pass) {
      const int buf = round++ & 1;
      if (!control) {
        const int v0 = min((rank * kVerifyWarps + warp) * per, n_vec), v1 = min(v0 + per, n_vec);
        long long sum = src.segment(v0, v1);
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) s_warp[buf][warp] = sum;
      }
      __syncthreads();
      if (control) {
        long long x = lane < kVerifyWarps ? s_warp[buf][lane] : 0;
        for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
        if (lane < C) {
          const uint32_t to = mapa(smem_u32(&s_cta[buf][rank]), lane);
          asm volatile("st.shared::cluster.b64 [%0], %1;" ::"r"(to), "l"(x) : "memory");
        }
        __syncwarp();  // the barrier wants whole warps
      }
      cluster_sync();
      long long total = 0, before = 0;
      for (int c = 0; c < C; ++c) {
        if (c == rank) before = total;
        total += s_cta[buf][c];
      }
      if (total == 0 && pass == 0) {  // nothing left of the difference: p alone
        src = Source<T>(prow, nullptr, a.V, -1);
        continue;
      }
      if (!control) break;
      if (total == 0) {
        if (rank == 0 && lane == 0) {
          a.out_ids[d.row] = -1;
          if (a.logp) a.logp[d.row] = 0.f;
          a.n_emit[i] = d.row - d.lo;
          flag_error(a.dev_err, PAIR_DEV_ERR_PROBABILITY);
        }
        break;
      }
      long long at = (long long)((double)a.u_draw[i] * (double)total);
      at = max(min(at, total - 1), 0ll);
      if (at < before || at >= before + s_cta[buf][rank]) break;
      int w = 0;
      while (at >= before + s_warp[buf][w]) before += s_warp[buf][w++];
      const int v0 = min((rank * kVerifyWarps + w) * per, n_vec), v1 = min(v0 + per, n_vec);
      const int tok = find(src, v0, v1, before, at);
      if (tok >= 0) {
        a.out_ids[d.row] = tok;
        if (a.logp) a.logp[d.row] = logf(as_float(prow[tok]));
        a.n_emit[i] = d.row - d.lo + 1;
      }
      break;
    }
  }
}

// Clusters of C CTAs that fit on device `dev`, the current one, at once (cached per
// type, device and C). The attribute that allows large ones is the device's too: it
// is set before an entry of that device is there.
template <typename T>
int resident_clusters(int dev, int C) {
  constexpr int kMaxDev = 128;
  static std::atomic<int> known[kMaxDev][kVerifyMaxCluster + 1];
  const bool cached = dev >= 0 && dev < kMaxDev;
  int n = cached ? known[dev][C].load(std::memory_order_acquire) : 0;
  if (n > 0) return n;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(C * 64, 1, 1);
  cfg.blockDim = dim3(kVerifyThreads, 1, 1);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = C;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaFuncSetAttribute(verify_kernel<T>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) !=
          cudaSuccess ||
      cudaOccupancyMaxActiveClusters(&n, verify_kernel<T>, &cfg) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return 0;
  }
  if (cached) known[dev][C].store(n, std::memory_order_release);
  return n;
}

template <typename T>
pair_status launch_verify(VerifyArgs<T> a, cudaStream_t s) {
  // CTAs of a cluster: the time goes with rounds x (1 / C + the exchange's share
  // of a row's reading), rounds = requests / clusters that fit. A large C leaves
  // the fewest SMs without work in the last round, and brings a single
  // request's row in from many SMs; short rows are not worth many CTAs.
  int best = 0, clusters = 0, dev = 0;
  double least = 0;
  PAIR_CUDA_TRY(cudaGetDevice(&dev));
  for (int C = 1; C <= kVerifyMaxCluster && (C == 1 || C * kVerifyLeast <= a.V); C *= 2) {
    const int n = resident_clusters<T>(dev, C);
    if (n < 1) continue;
    const double t = (double)ceil_div(a.R, n) * (1.0 / C + 3000.0 / a.V);
    if (best == 0 || t < least) {
      best = C;
      least = t;
      clusters = a.R < n ? a.R : n;
    }
  }
  if (best == 0) return PAIR_ERR_CUDA;
  a.C = best;
  a.clusters = clusters;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)best * (unsigned)clusters, 1, 1);
  cfg.blockDim = dim3(kVerifyThreads, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = best;
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
      !out_ids || !n_emit || (T > 1 && (p_row < V || (q && q_row < V))))
    return PAIR_ERR_INVALID_ARG;
  const pair_status dv = check_device();
  if (dv != PAIR_OK) return dv;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (dt == PAIR_BF16)
    return launch_verify<__nv_bfloat16>(
        {T, R, V, 1, 1, static_cast<const __nv_bfloat16 *>(p),
         static_cast<const __nv_bfloat16 *>(q),
         p_row, q_row, ids, cu_new, u, u_draw, out_ids, logp, n_emit, dev_err}, s);
  return launch_verify<float>({T, R, V, 1, 1, static_cast<const float *>(p),
                               static_cast<const float *>(q), p_row, q_row, ids, cu_new, u,
                               u_draw, out_ids, logp, n_emit, dev_err}, s);
}
