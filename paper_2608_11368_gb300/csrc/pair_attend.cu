// pair_attend_paged and pair_attend_paged_q8: entry points, the fp32 kernel on the
// CUDA cores, and the pass that joins partial sums.
#include <math.h>

#include "pair_attend.cuh"
#include "pair_cache_q8.cuh"

namespace pairk {
namespace attend {
namespace {

constexpr int kSimtThreads = 128;
constexpr int kSimtRows = 16;

__device__ __forceinline__ void from_float(float *o, float x) { *o = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16 *o, float x) {
  *o = __float2bfloat16_rn(x);
}

template <int D>
struct SimtSmem {
  static constexpr int kKeys = D == 64 ? 64 : 32;
  static constexpr int kStages = 3;
  float k[kStages][kKeys][D + 4];
  float v[kStages][kKeys][D];
  float q[kSimtRows][D];
  float p[kSimtRows][kKeys];
  float m[kSimtRows], l[kSimtRows], fix[kSimtRows];
  int64_t row[2][2][kKeys];  // offsets of a tile's keys and values
  int seen[kSimtRows];
  int64_t scratch[kSimtThreads / 32 + 2];
};

// fp32 products on the CUDA cores, 16 rows against tiles of keys and values
// that arrive two tiles ahead (asynchronous copies into shared memory). A
// thread forms the scores of one key with its group's rows (the queries are
// broadcast reads), then the output sums of its columns for 16 rows (8 at D =
// 64), four keys at a time; rows that are not in use are left out. Bound by
// latency at small sizes (three barriers and two exchanges per tile; 32 requests
// of up to 640 keys, heads of 64: 22 us with the joining pass), else by
// shared-memory reads.
template <int D>
__global__ void __launch_bounds__(kSimtThreads) attend_simt_kernel(Args a) {
  extern __shared__ __align__(16) uint8_t raw[];
  using S = SimtSmem<D>;
  S &sm = *reinterpret_cast<S *>(raw);
  constexpr int M = kSimtRows, BN = S::kKeys, NST = S::kStages, V4 = D / 4;
  constexpr int QR = M * BN / kSimtThreads;                      // rows of a thread's scores
  constexpr int QG = M / QR;                                     // groups of them
  constexpr int CPT = D >= kSimtThreads ? D / kSimtThreads : 1;  // columns per thread
  constexpr int RG = D >= kSimtThreads ? 1 : kSimtThreads / D;   // row groups
  constexpr int RPT = M / RG;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int cta = blockIdx.x, ctas = gridDim.x;
  clear_notes(a, cta);
  clear_spare_rows<float, D, kSimtThreads>(a, cta, ctas);
  if (cta == ctas - 1) report_requests(a);
  Walk<M, BN> walk{find_share<kSimtThreads>(a, M, cta, ctas, sm.scratch)};
  const float *q = static_cast<const float *>(a.q);
  const float *kc = static_cast<const float *>(a.kc), *vc = static_cast<const float *>(a.vc);
  const float scale = a.scale * kLog2e;
  const int col = tid % (kSimtThreads / RG), rg = tid / (kSimtThreads / RG);
  Segment s;
  for (int seg = 0; walk.next(a, &s); ++seg) {
    __syncthreads();
    // Offsets of a tile's rows, by the first BN threads, one tile before its
    // copies are started.
    auto put_offsets = [&](int t) {
      const int key = t * BN + tid;
      if (tid < BN && t < s.t1) {
        int off = 0;
        const int id = key < s.keys ? page_of(a, s.i, key, &off) : -1;
        sm.row[t & 1][0][tid] = id < 0 ? -1 : cache_row(a, a.ks, id, off, s.h);
        sm.row[t & 1][1][tid] = id < 0 ? -1 : cache_row(a, a.vs, id, off, s.h);
      }
    };
    auto fetch = [&](int t) {
      if (t < s.t1) {
        const int st = (t - s.t0) % NST;
#pragma unroll 4
        for (int x = tid; x < BN * V4; x += kSimtThreads) {
          const int k = x / V4, c = x % V4 * 4;
          const int64_t ko = sm.row[t & 1][0][k], vo = sm.row[t & 1][1][k];
          cp_async16(tc::smem_u32(&sm.k[st][k][c]), kc + (ko < 0 ? 0 : ko + c), ko >= 0);
          cp_async16(tc::smem_u32(&sm.v[st][k][c]), vc + (vo < 0 ? 0 : vo + c), vo >= 0);
        }
      }
      cp_async_commit();
    };
    put_offsets(s.t0);
    put_offsets(s.t0 + 1);
    for (int x = tid; x < M * V4; x += kSimtThreads) {
      const int r = x / V4, c = x % V4 * 4;
      float4 u = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < s.rows) {
        const RowAt at = row_at(a, s.row0, s.r0, s.h, r);
        u = *reinterpret_cast<const float4 *>(q + at.token * a.q_row + at.head * a.q_head + c);
      }
      *reinterpret_cast<float4 *>(&sm.q[r][c]) = u;
    }
    if (tid < M) {
      sm.m[tid] = -INFINITY;
      sm.l[tid] = 0.f;
      sm.seen[tid] = min(s.seen(tid, a.g), s.kv);
    }
    __syncthreads();
    fetch(s.t0);
    fetch(s.t0 + 1);
    float o[RPT][CPT];
    int seen[RPT];
#pragma unroll
    for (int r = 0; r < RPT; ++r) {
      seen[r] = sm.seen[r * RG + rg];
#pragma unroll
      for (int c = 0; c < CPT; ++c) o[r][c] = 0.f;
    }
    for (int t = s.t0; t < s.t1; ++t) {
      const int key0 = t * BN, st = (t - s.t0) % NST;
      cp_async_wait<1>();
      __syncthreads();  // tile t is there, tile t - 1's stage free
      put_offsets(t + 2);
      {
        const int k = tid % BN, g0 = tid / BN;  // rows g0, g0 + QG, ..
        float acc[QR] = {};
#pragma unroll 4
        for (int d = 0; d < D; d += 4) {
          const float4 x = *reinterpret_cast<const float4 *>(&sm.k[st][k][d]);
#pragma unroll
          for (int r = 0; r < QR; ++r) {
            if (r * QG >= s.rows) break;
            const float4 y = *reinterpret_cast<const float4 *>(&sm.q[r * QG + g0][d]);
            acc[r] = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, acc[r]))));
          }
        }
#pragma unroll
        for (int r = 0; r < QR; ++r)
          sm.p[r * QG + g0][k] = key0 + k < sm.seen[r * QG + g0] ? acc[r] * scale : -INFINITY;
      }
      __syncthreads();
      fetch(t + 2);
      // Running maximum and sum: a warp has four rows.
      float sc[M / 4][BN / 32], mx[M / 4], sum[M / 4];
#pragma unroll
      for (int r = 0; r < M / 4; ++r) {
        mx[r] = -INFINITY;
#pragma unroll
        for (int x = 0; x < BN / 32; ++x) {
          sc[r][x] = sm.p[warp * (M / 4) + r][lane + 32 * x];
          mx[r] = fmaxf(mx[r], sc[r][x]);
        }
      }
#pragma unroll
      for (int w = 16; w > 0; w >>= 1)
#pragma unroll
        for (int r = 0; r < M / 4; ++r)
          mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], w));
#pragma unroll
      for (int r = 0; r < M / 4; ++r) {
        mx[r] = fmaxf(mx[r], sm.m[warp * (M / 4) + r]);
        const float ref = mx[r] == -INFINITY ? 0.f : mx[r];
        sum[r] = 0.f;
#pragma unroll
        for (int x = 0; x < BN / 32; ++x) {
          sc[r][x] = exp2f(sc[r][x] - ref);
          sum[r] += sc[r][x];
          sm.p[warp * (M / 4) + r][lane + 32 * x] = sc[r][x];
        }
      }
#pragma unroll
      for (int w = 16; w > 0; w >>= 1)
#pragma unroll
        for (int r = 0; r < M / 4; ++r) sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], w);
      if (lane == 0) {
#pragma unroll
        for (int r = 0; r < M / 4; ++r) {
          const int rr = warp * (M / 4) + r;
          const float fix = exp2f(sm.m[rr] - (mx[r] == -INFINITY ? 0.f : mx[r]));
          sm.m[rr] = mx[r];
          sm.l[rr] = fmaf(sm.l[rr], fix, sum[r]);
          sm.fix[rr] = fix;
        }
      }
      __syncthreads();
#pragma unroll
      for (int r = 0; r < RPT; ++r)
#pragma unroll
        for (int c = 0; c < CPT; ++c) o[r][c] *= sm.fix[r * RG + rg];
      // A value that a row does not see must not reach its sums, not even
      // times zero: it may be NaN. Behind the last key the values are zeros.
      const bool edge = key0 + BN > s.least;
#pragma unroll 2
      for (int k = 0; k < BN; k += 4) {
        float v[4][CPT];
#pragma unroll
        for (int y = 0; y < 4; ++y)
#pragma unroll
          for (int c = 0; c < CPT; ++c) v[y][c] = sm.v[st][k + y][col + c * kSimtThreads];
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
          if (r * RG >= s.rows) break;
          const float4 p4 = *reinterpret_cast<const float4 *>(&sm.p[r * RG + rg][k]);
          const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int c = 0; c < CPT; ++c) {
              const float n = fmaf(p[y], v[y][c], o[r][c]);
              o[r][c] = edge && key0 + k + y >= seen[r] ? o[r][c] : n;
            }
        }
      }
    }
    cp_async_wait<0>();
    __syncthreads();
    if (s.whole()) {
#pragma unroll
      for (int r = 0; r < RPT; ++r) {
        const int rr = r * RG + rg;
        if (rr >= s.rows) continue;
        const RowAt at = row_at(a, s.row0, s.r0, s.h, rr);
        const float l = sm.l[rr], inv = l == 0.f ? 0.f : 1.f / l;
        float *out = static_cast<float *>(a.out) + (at.token * a.Hq + at.head) * D;
#pragma unroll
        for (int c = 0; c < CPT; ++c) out[col + c * kSimtThreads] = o[r][c] * inv;
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
          part[2 * M + (r * RG + rg) * D + col + c * kSimtThreads] = o[r][c];
    }
  }
  let_next_start();
}

// Blocks that share the rows of one of a launch's units: 4 rows a warp.
template <int NT>
__host__ __device__ int join_blocks(const Launch &l) {
  int64_t rows = l.a.T * l.a.g;
  if (rows > l.M) rows = l.M;
  if (rows > l.a.rows_upto) rows = l.a.rows_upto;
  return (int)((rows + NT / 8 - 1) / (NT / 8));
}

// Joins the partial sums of the units that more than one CTA worked on, of one
// launch or of two: blocks of the CTA that has a unit's beginning. The other
// pieces are the first segments of the CTAs behind. Sums go in the order of the
// keys. Bound by latency (notes, then sums, whose loads do not wait for the maxima) and,
// after a launch with many rows, by the 40 MB of its partial sums. NT threads, each with B
// floats of partial sums on their way.
template <typename T, int D, int NT, int B>
__global__ void __launch_bounds__(NT)
    attend_join_kernel(const __grid_constant__ Launch l0, const __grid_constant__ Launch l1) {
  const int first = l0.ctas * join_blocks<NT>(l0);  // blocks of the first launch's sums
  const bool second = (int)blockIdx.x >= first;
  const Args &a = second ? l1.a : l0.a;
  const int M = second ? l1.M : l0.M, ctas = second ? l1.ctas : l0.ctas;
  const int per = join_blocks<NT>(second ? l1 : l0);
  const int block = blockIdx.x - (second ? first : 0);
  const int cta = block / per, y = block - cta * per;
  __shared__ uint16_t slots[kMaxWorkers];
  __shared__ int n_slots;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  wait_for_previous();
  // A CTA has the beginning of one unit at most whose end it does not have.
  const Desc d0 = a.desc[cta * 2], d1 = a.desc[cta * 2 + 1];
  Desc e{};  // notes of the CTAs behind, 32 at a time
  if (warp == 0 && cta + 1 + lane < ctas) e = a.desc[(cta + 1 + lane) * 2];
  const bool is0 = d0.tiles != 0 && d0.t0 == 0;
  const Desc d = is0 ? d0 : d1;
  if (d.tiles == 0 || d.t0 != 0) return;
  const int mine = cta * 2 + (is0 ? 0 : 1);
  if (warp == 0) {
    int n = 1;
    if (lane == 0) slots[0] = mine;
    bool more = true;
    for (int c0 = cta + 1; more && c0 < ctas; c0 += 32) {
      const int c = c0 + lane;
      const bool in = e.tiles > 0 && e.i == d.i && e.h == d.h && e.rt == d.rt;
      const unsigned ins = __ballot_sync(0xffffffffu, in);
      if (in) slots[n + __popc(ins & ((1u << lane) - 1))] = c * 2;
      n += __popc(ins);
      more = !__any_sync(0xffffffffu, in && e.t1 == e.tiles);
      if (more) e = c + 32 < ctas ? a.desc[(c + 32) * 2] : Desc{};
    }
    if (lane == 0) n_slots = n;
  }
  __syncthreads();
  const int n = n_slots;
  constexpr int kWarps = NT / 32, C = D / 32;
  constexpr int P = B / C;  // partial sums on their way to a lane
  // With few partial sums a warp takes a row; with many (a long unit over many
  // CTAs) the warps share a row's, in runs, and the first adds up what they have.
  const bool share = n >= 2 * kWarps;
  const int k0 = share ? warp * n / kWarps : 0, k1 = share ? (warp + 1) * n / kWarps : n;
  const int step = share ? per : per * kWarps;
  for (int r = share ? y : y * kWarps + warp; r < d.rows; r += step) {
    float2 x[P][C / 2];
    float m[P], sum[P];
    const auto bring = [&](int k) {
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (k + i < k1) {
          const float *p = a.part + slots[k + i] * part_floats(M, D);
          m[i] = p[r], sum[i] = p[M + r];
          const float2 *src = reinterpret_cast<const float2 *>(p + 2 * M + r * D + lane * C);
#pragma unroll
          for (int c = 0; c < C / 2; ++c) x[i][c] = src[c];
        }
    };
    float mx = -INFINITY;
    for (int k = lane; k < n; k += 32) mx = fmaxf(mx, a.part[slots[k] * part_floats(M, D) + r]);
    bring(k0);  // beside the maxima
    for (int w = 16; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
    const float ref = mx == -INFINITY ? 0.f : mx;
    float l = 0.f, o[C] = {};
    for (int k = k0; k < k1; k += P) {
      if (k > k0) bring(k);
#pragma unroll
      for (int i = 0; i < P; ++i)
        if (k + i < k1) {
          const float f = exp2f(m[i] - ref);
          l = fmaf(sum[i], f, l);
#pragma unroll
          for (int c = 0; c < C / 2; ++c) {
            o[2 * c] = fmaf(x[i][c].x, f, o[2 * c]);
            o[2 * c + 1] = fmaf(x[i][c].y, f, o[2 * c + 1]);
          }
        }
    }
    if (share) {
      __shared__ float sums[kWarps][D + 1];
      __syncthreads();
#pragma unroll
      for (int c = 0; c < C; ++c) sums[warp][lane * C + c] = o[c];
      if (lane == 0) sums[warp][D] = l;
      __syncthreads();
      if (warp != 0) continue;
      for (int w = 1; w < kWarps; ++w) {
        l += sums[w][D];
#pragma unroll
        for (int c = 0; c < C; ++c) o[c] += sums[w][lane * C + c];
      }
    }
    const RowAt at = row_at(a, d.row0, d.rt * M, d.h, r);
    const float inv = l == 0.f ? 0.f : 1.f / l;
    T *out = static_cast<T *>(a.out) + (at.token * a.Hq + at.head) * D + lane * C;
#pragma unroll
    for (int c = 0; c < C; ++c) from_float(out + c, o[c] * inv);
    if (lane == 0 && a.lse)
      a.lse[at.token * a.Hq + at.head] = l == 0.f ? -INFINITY : (mx + log2f(l)) * kLn2;
  }
}

template <int D>
pair_status run_simt(Launch *l, cudaStream_t s) {
  Args &a = l->a;
  a.unit_cost = kSimtCost;
  constexpr int smem = sizeof(SimtSmem<D>);
  static_assert(smem <= 232448, "shared memory of a CTA");
  PAIR_CUDA_TRY(cudaFuncSetAttribute(attend_simt_kernel<D>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const int ctas = useful_ctas(a, kSimtRows, min(kMaxCtas, (D <= 128 ? 2 : 1) * sm_count()));
  PAIR_BEGIN("attend_simt", s);
  attend_simt_kernel<D><<<ctas, kSimtThreads, smem, s>>>(a);
  PAIR_LAUNCH_CHECK(s);
  l->M = kSimtRows;
  l->ctas = ctas;
  return PAIR_OK;
}

template <typename T, int D, int NT, int B>
pair_status run_join(const Launch &l0, const Launch &l1, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(l0.ctas * join_blocks<NT>(l0) + l1.ctas * join_blocks<NT>(l1), 1, 1);
  cfg.blockDim = dim3(NT, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  PAIR_BEGIN("attend_join", s);
  if (cudaLaunchKernelEx(&cfg, attend_join_kernel<T, D, NT, B>, l0, l1) != cudaSuccess) {
    cudaGetLastError();
    return PAIR_ERR_CUDA;
  }
  PAIR_LAUNCH_CHECK(s);
  return PAIR_OK;
}

// After a launch with many rows blocks are many and their rows have two or three partial
// sums: few registers (four chunks over bf16 388 us, with 32 floats 398). Else a row has all
// its sums on their way at once where they are many (a token over 20,000 of codes 38 us,
// four at a time and behind the maxima 47). Where warps have shares of their own and a
// unit falls to a few of them, blocks of four warps, all at once on the SMs (8 x 8 requests,
// a token each: 42.1 us, of eight warps 45.5).
template <typename T, int D>
pair_status run_join(const Launch &l0, const Launch &l1, cudaStream_t s) {
  if (l1.ctas) return run_join<T, D, 256, 8>(l0, l1, s);
  if (l0.a.ke && l0.ctas < 8 * (int64_t)l0.a.R * l0.a.Hkv)
    return run_join<T, D, 128, 16>(l0, l1, s);
  return run_join<T, D, 256, 32>(l0, l1, s);
}

template <typename F>
pair_status by_size(int D, F f) {
  if (D == 64) return f(std::integral_constant<int, 64>());
  if (D == 128) return f(std::integral_constant<int, 128>());
  return f(std::integral_constant<int, 256>());
}

// The workspace: notes and partial sums of a launch with few or, in fp32, any rows,
// then those of a launch with many.
constexpr size_t kNotes = kMaxCtas * 2 * sizeof(Desc), kManyNotes = kMaxMany * 2 * sizeof(Desc);
// Over caches in 8 bits warps have shares and notes of their own; the partial sums behind
// them take the rest.
constexpr size_t kHeldNotes = kMaxWorkers * 2 * sizeof(Desc);
size_t few_floats(int D) { return kMaxCtas * 2 * part_floats(kFewTile, D); }
size_t many_floats(int D) { return kMaxMany * 2 * part_floats(kManyRows, D); }

bool aligned(const void *p, uintptr_t to) {
  return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0;
}

}  // namespace

// CTAs (or pairs) of a launch: as many as fit at once, or as the work can be
// worth at most: the host knows the table's width, not the lengths.
int useful_ctas(const Args &a, int M, int fit, int least) {
  const double units = (double)ceil_div(a.T * a.g, M) + (double)(a.R < a.T ? a.R : a.T);
  const double keys = units * a.heads * (a.unit_cost + (double)a.width * a.page + (double)M / a.g);
  return keys < (double)fit * least ? 1 + (int)(keys / least) : fit;
}

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) {
    cudaGetLastError();
    return 1;
  }
  return n;
}

pair_status launch_simt(Launch *l, int D, cudaStream_t s) {
  return by_size(D, [&](auto d) { return run_simt<decltype(d)::value>(l, s); });
}

static pair_status launch_join(const Launch &l0, const Launch &l1, int D, pair_dtype dt,
                               cudaStream_t s) {
  return by_size(D, [&](auto d) {
    return dt == PAIR_BF16 ? run_join<__nv_bfloat16, decltype(d)::value>(l0, l1, s)
                           : run_join<float, decltype(d)::value>(l0, l1, s);
  });
}

// A call of either entry point. fmt q8::kPlain: caches in the type of q.
static pair_status attend_paged(int64_t T, int32_t R, int32_t Hq, int32_t Hkv, int32_t D,
                                pair_dtype dt, const void *q, int64_t q_row, int64_t q_head,
                                int fmt, const pair_cache_q8 &k, const pair_cache_q8 &v,
                                int32_t num_pages, int32_t page_size, const int32_t *block_table,
                                int32_t table_width, const int32_t *kv_len, const int32_t *cu_new,
                                float scale, int32_t max_new, void *out, float *lse, void *ws,
                                size_t ws_bytes, int32_t *dev_err, pair_stream_t stream) {
  reset_launches();
  const bool held = fmt != q8::kPlain;
  if (T < 1 || T > INT32_MAX || R < 1 || R > kMaxRequests || Hkv < 1 || Hq < Hkv ||
      Hq % Hkv != 0 || !q || !k.codes || !v.codes || (held && (!k.exps || !v.exps)) ||
      num_pages < 1 || page_size < 1 || !block_table || table_width < 1 || !kv_len || !cu_new ||
      !out || !(fabsf(scale) <= 3.0e38f) || max_new < 0 || (dt != PAIR_F32 && dt != PAIR_BF16) ||
      T * (Hq / Hkv) > INT32_MAX)
    return PAIR_ERR_INVALID_ARG;
  const int per = dt == PAIR_BF16 ? 8 : 4;  // elements of 16 bytes
  // A stride over a single entry says nothing; a tensor map wants one all the same.
  const auto over = [](int64_t stride, int64_t entries) { return entries > 1 ? stride : 256; };
  const auto all_over = [&](const pair_cache_strides &x) {
    return pair_cache_strides{over(x.for_page, num_pages), over(x.for_token, page_size),
                              over(x.for_head, Hkv)};
  };
  q_row = over(q_row, T), q_head = over(q_head, Hq);
  const pair_cache_strides ks = all_over(k.codes_at), vs = all_over(v.codes_at);
  if (q_row % per != 0 || q_head % per != 0) return PAIR_ERR_INVALID_ARG;
  for (const pair_cache_strides *x : {&ks, &vs})
    for (const int64_t y : {x->for_page, x->for_token, x->for_head})
      if (y % (held ? 16 : per) != 0) return PAIR_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(k.codes, 16) || !aligned(v.codes, 16) || !aligned(out, 16))
    return PAIR_ERR_INVALID_ARG;
  const size_t need = pair_attend_workspace_size(R, Hq, Hkv, D, dt);
  if (need == 0) return PAIR_ERR_UNSUPPORTED;
  if (!ws || ws_bytes < need || !aligned(ws, 256)) return PAIR_ERR_WORKSPACE;
  const pair_status dv = check_device();
  if (dv != PAIR_OK) return dv;
  const size_t notes = held ? kHeldNotes : kNotes;
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
               k.codes,
               v.codes,
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
               reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + notes + kManyNotes),
               dev_err,
               k.exps,
               v.exps,
               k.exps_at,
               v.exps_at,
               false,
               0,
               0,
               Hkv,
               0};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  Launch few{a, 0, 0}, many{a, 0, 0};
  many.a.desc = reinterpret_cast<Desc *>(static_cast<uint8_t *>(ws) + notes);
  many.a.part = reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + need) - many_floats(D);
  // Which kernel a chunk goes to is decided by its rows, on the device; a
  // launch is left out where the host knows that no chunk can be its.
  const int64_t most_rows = (int64_t)(max_new > 0 && max_new < T ? max_new : T) * a.g;
  const bool only_few = dt == PAIR_F32 || most_rows <= kFewRows ||
                        !(held ? many_applies_q8(a, D) : many_applies(a, D));
  if (!only_few && R > 1) {
    few.a.rows_upto = kFewRows;
    many.a.rows_over = kFewRows;
  }
  pair_status st = PAIR_OK;
  if (held && (only_few || R > 1)) {
    const float *end = reinterpret_cast<float *>(static_cast<uint8_t *>(ws) + need);
    const int64_t room = (only_few ? end : many.a.part) - few.a.part;
    FewLauncher *const launch = dt == PAIR_BF16
                                    ? (fmt == q8::kI8 ? launch_few_i8 : launch_few_e4m3)
                                    : (fmt == q8::kI8 ? launch_few_i8_f32 : launch_few_e4m3_f32);
    st = launch(&few, D, most_rows, (int)(room / part_floats(kFewTile, D)), s);
  } else if (dt == PAIR_F32) {
    st = launch_simt(&few, D, s);
  } else if (only_few || R > 1) {
    st = launch_few(&few, D, s);
  }
  if (st == PAIR_OK && !only_few)
    st = held ? launch_many_q8(&many, D, fmt, s) : launch_many(&many, D, s);
  return st == PAIR_OK ? launch_join(few, many, D, dt, s) : st;
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
  return kNotes + kManyNotes + (few_floats(D) + many_floats(D)) * sizeof(float);
}

pair_status pair_attend_paged(int64_t T, int32_t R, int32_t Hq, int32_t Hkv, int32_t D,
                              pair_dtype dt, const void *q, int64_t q_row, int64_t q_head,
                              const void *k_cache, pair_cache_strides ks, const void *v_cache,
                              pair_cache_strides vs, int32_t num_pages, int32_t page_size,
                              const int32_t *block_table, int32_t table_width,
                              const int32_t *kv_len, const int32_t *cu_new, float scale,
                              int32_t max_new, void *out, float *lse, void *ws,
                              size_t ws_bytes, int32_t *dev_err, pair_stream_t stream) {
  return attend_paged(T, R, Hq, Hkv, D, dt, q, q_row, q_head, q8::kPlain,
                      {const_cast<void *>(k_cache), ks, nullptr, {}},
                      {const_cast<void *>(v_cache), vs, nullptr, {}}, num_pages, page_size,
                      block_table, table_width, kv_len, cu_new, scale, max_new, out, lse, ws,
                      ws_bytes, dev_err, stream);
}

pair_status pair_attend_paged_q8(int64_t T, int32_t R, int32_t Hq, int32_t Hkv, int32_t D,
                                 pair_dtype dt, const void *q, int64_t q_row, int64_t q_head,
                                 pair_cache_format fmt, pair_cache_q8 k_cache,
                                 pair_cache_q8 v_cache, int32_t num_pages, int32_t page_size,
                                 const int32_t *block_table, int32_t table_width,
                                 const int32_t *kv_len, const int32_t *cu_new, float scale,
                                 int32_t max_new, void *out, float *lse, void *ws,
                                 size_t ws_bytes, int32_t *dev_err, pair_stream_t stream) {
  if ((int)fmt != q8::kI8 && (int)fmt != q8::kE4M3) {
    reset_launches();
    return PAIR_ERR_INVALID_ARG;
  }
  return attend_paged(T, R, Hq, Hkv, D, dt, q, q_row, q_head, fmt, k_cache, v_cache, num_pages,
                      page_size, block_table, table_width, kv_len, cu_new, scale, max_new, out, lse,
                      ws, ws_bytes, dev_err, stream);
}

}  // extern "C"
