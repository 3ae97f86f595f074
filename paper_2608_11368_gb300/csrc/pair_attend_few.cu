// pair_attend_paged for chunks with few rows (single tokens, drafts), bf16: one
// pass over the cached keys and values, bound by HBM. 16 x 16 requests of up to
// 4096 keys on 32/8 heads: a token each would read 2.4 GB; five rows each (20 per
// key head) take 390 us, 6.2 TB/s; 32 x 16 skewed ones with a token each run at
// the copy's rate (6.8 TB/s). mma.sync rather than tcgen05: a tile of 128 rows
// would be 16 to 32 rows full, and its chain of products and softmax takes as
// long as the bytes of a tile.
//
// The softmax weights enter the second product in bf16, as its operands are: each
// is off by up to 2^-8 of itself, independently, while their sum takes them
// unrounded in fp32. Against 64 bits a row of 700 keys is off by 1.7e-3 of its size,
// of which the output's one rounding to bf16 is 1.6e-3; weights of 16 more bits
// would take a second product per tile.
#include "pair_attend.cuh"

namespace pairk {
namespace attend {
namespace {

using namespace tc;

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int M = kFewTile;

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at)
               : "memory");
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                         uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t *>(&x);
}

template <int D>
struct Few {
  static constexpr int BN = D == 64 ? 128 : 64;     // keys of a tile
  static constexpr int kStages = 2;
  static constexpr int kTile = BN * D * 2;          // bytes of a tile of keys or values
  static constexpr int kChunks = D / 8;             // 16-byte pieces of a row
  static constexpr int kRowsPerPass = kThreads / kChunks;
  static constexpr int kOff = 0;                    // row offsets: [kStages][2][BN] int64
  static constexpr int kBad = kOff + kStages * 2 * BN * 8;  // a flag
  static constexpr int kKV = kBad + 128;            // stages: keys, values
  static constexpr int kEnd = kKV + kStages * 2 * kTile;
  // The queries are in registers before the last stage is first filled (two
  // CTAs per SM then fit); at D = 256 they stay.
  static constexpr int kQ = D <= 128 ? kKV + (kStages - 1) * 2 * kTile : kEnd;
  static constexpr int kMl = kKV + M * D * 4;       // the warps' statistics, at the end
  static constexpr int kBytes = D <= 128 ? kEnd : kEnd + M * D * 2;
  static_assert(M * D * 4 + kWarps * 16 * 8 * 4 <= kStages * 2 * kTile, "the warps' sums fit");
};

// Tiles go through two stages of shared memory, three CTAs per SM (two with three
// stages: 473 us instead of 440), by 16-byte asynchronous copies (one bulk copy
// per row of 256 bytes: 594 instead of 473).
//
// A segment whose tile has at most 16 WR rows in use: warp w has rows
// [16 (w % WR), +16) and the keys [w / WR * BN / WK, +BN / WK) of every tile,
// WK = 4 / WR. With one row group all four warps split the keys.
template <int D, int WR>
__device__ __forceinline__ void few_segment(const Args &a, const Segment &s, uint8_t *smem,
                                            int cta, int seg) {
  using F = Few<D>;
  constexpr int BN = F::BN, WK = kWarps / WR, KW = BN / WK, NT = KW / 8, NST = F::kStages;
  constexpr bool kQRegs = D <= 128;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int wr = warp % WR, wk = warp / WR;
  int64_t *offs = reinterpret_cast<int64_t *>(smem + F::kOff);
  int *any_bad = reinterpret_cast<int *>(smem + F::kBad);
  const uint32_t q_at = smem_u32(smem + F::kQ), kv_at = smem_u32(smem + F::kKV);
  const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(a.q);
  const __nv_bfloat16 *kc = static_cast<const __nv_bfloat16 *>(a.kc);
  const __nv_bfloat16 *vc = static_cast<const __nv_bfloat16 *>(a.vc);

  // The page of a tile's key tid (off < 0: no such key). What the cache's owner
  // wrote is looked at when it is used, so the reads overlap.
  auto find_page = [&](int t, int *off) {
    const int key = t * BN + tid;
    *off = -1;
    if (t >= s.t1 || tid >= BN || key >= s.keys) return 0;
    const int at = key / a.page;
    *off = key - at * a.page;
    return a.table[(int64_t)s.i * a.width + at];
  };
  // Offsets of a tile's rows: thread k < BN has key k's.
  auto put_offsets = [&](int buf, int id, int off) {
    if (tid < BN) {
      if (off >= 0 && (unsigned)id >= (unsigned)a.num_pages) {
        flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
        id = 0;
      }
      offs[(buf * 2) * BN + tid] = off < 0 ? -1 : cache_row(a, a.ks, id, off, s.h);
      offs[(buf * 2 + 1) * BN + tid] = off < 0 ? -1 : cache_row(a, a.vs, id, off, s.h);
    }
  };
  auto load_tile = [&](int t, int stage, int buf) {
    if (t < s.t1) {
      const int c = tid % F::kChunks;
      const uint32_t kd = kv_at + stage * 2 * F::kTile, vd = kd + F::kTile;
#pragma unroll
      for (int x = 0; x < BN / F::kRowsPerPass; ++x) {
        const int r = tid / F::kChunks + x * F::kRowsPerPass;
        const int64_t ko = offs[(buf * 2) * BN + r], vo = offs[(buf * 2 + 1) * BN + r];
        const uint32_t to = r * D * 2 + ((c ^ (r & 7)) << 4);
        cp_async16(kd + to, kc + (ko < 0 ? 0 : ko + c * 8), ko >= 0);
        cp_async16(vd + to, vc + (vo < 0 ? 0 : vo + c * 8), vo >= 0);
      }
    }
    cp_async_commit();
  };
  int id[NST], off[NST];
#pragma unroll
  for (int x = 0; x < NST; ++x) id[x] = find_page(s.t0 + x, &off[x]);
  constexpr int kQPieces = 16 * WR * F::kChunks / kThreads;
  uint4 qv[kQPieces];
#pragma unroll
  for (int y = 0; y < kQPieces; ++y) {
    const int x = tid + y * kThreads, r = x / F::kChunks, c = x % F::kChunks;
    qv[y] = make_uint4(0, 0, 0, 0);
    if (r < s.rows) {
      const RowAt at = row_at(a, s.row0, s.r0, s.h, r);
      qv[y] = *reinterpret_cast<const uint4 *>(q + at.token * a.q_row + at.head * a.q_head + c * 8);
    }
  }
  __syncthreads();  // the segment before is through
  if (tid == 0) *any_bad = 0;
#pragma unroll
  for (int x = 0; x < NST - 1; ++x) put_offsets(x, id[x], off[x]);
  int next_id = id[NST - 1], next_off = off[NST - 1];
#pragma unroll
  for (int y = 0; y < kQPieces; ++y) {
    const int x = tid + y * kThreads, r = x / F::kChunks, c = x % F::kChunks;
    *reinterpret_cast<uint4 *>(smem + F::kQ + r * D * 2 + ((c ^ (r & 7)) << 4)) = qv[y];
  }
  __syncthreads();
#pragma unroll
  for (int x = 0; x < NST - 1; ++x) load_tile(s.t0 + x, x, x);

  uint32_t qf[kQRegs ? D / 16 : 1][4];
  const uint32_t q_lane = q_at + (wr * 16 + (lane & 15)) * D * 2;
  auto load_q = [&](int kk, uint32_t (&f)[4]) {
    ldsm4(f, q_lane + (((kk * 2 + (lane >> 4)) ^ (lane & 7)) << 4));
  };
  if (kQRegs) {
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) load_q(kk, qf[kQRegs ? kk : 0]);
  }
  float o[D / 8][4];
#pragma unroll
  for (int j = 0; j < D / 8; ++j)
#pragma unroll
    for (int c = 0; c < 4; ++c) o[j][c] = 0.f;
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  const float scale = a.scale * kLog2e;
  const bool working = wr * 16 < s.rows;
  const int ra = wr * 16 + (lane >> 2);
  const int seen[2] = {min(s.seen(ra, a.g), s.kv), min(s.seen(ra + 8, a.g), s.kv)};
  const int least = s.least;

  for (int t = s.t0; t < s.t1; ++t) {
    const int it = t - s.t0, stage = it % NST;
    cp_async_wait<NST - 2>();
    const int nbuf = (it + NST - 1) % NST;
    put_offsets(nbuf, next_id, next_off);
    __syncthreads();
    load_tile(t + NST - 1, nbuf, nbuf);
    next_id = find_page(t + NST, &next_off);
    const uint32_t ks = kv_at + stage * 2 * F::kTile, vs = ks + F::kTile;
    const int key0 = t * BN;
    const bool edge = key0 + BN > least;
    if (edge && key0 < s.keys && least < s.keys) {
      // Values that some row does not see: a weight of 0 must not meet a NaN
      // or an infinity. They are taken out here and, being what they are,
      // added to the rows that do see them at the end.
      for (int x = tid; x < BN * F::kChunks; x += kThreads) {
        uint4 *at = reinterpret_cast<uint4 *>(smem + F::kKV + stage * 2 * F::kTile + F::kTile) + x;
        uint4 u = *at;
        uint32_t *w = reinterpret_cast<uint32_t *>(&u);
        bool bad = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if ((w[k] & 0x7f80u) == 0x7f80u) w[k] &= 0xffff0000u, bad = true;
          if ((w[k] & 0x7f800000u) == 0x7f800000u) w[k] &= 0xffffu, bad = true;
        }
        if (bad) {
          *at = u;
          *any_bad = 1;
        }
      }
      __syncthreads();
    }
    if (!working) continue;
    float sc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) sc[j][c] = 0.f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      if (!kQRegs) load_q(kk, qf[0]);
#pragma unroll
      for (int j = 0; j < NT; j += 2) {
        uint32_t b[4];
        const int key = wk * KW + j * 8 + ((lane >> 4) << 3) + (lane & 7);
        ldsm4(b, ks + key * D * 2 + (((kk * 2 + ((lane >> 3) & 1)) ^ (lane & 7)) << 4));
        mma16816(sc[j], qf[kQRegs ? kk : 0], b[0], b[1]);
        mma16816(sc[j + 1], qf[kQRegs ? kk : 0], b[2], b[3]);
      }
    }
    float mx[2] = {m[0], m[1]};
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        sc[j][c] *= scale;
        if (edge) {
          const int key = key0 + wk * KW + j * 8 + 2 * (lane & 3) + (c & 1);
          if (key >= seen[c >> 1]) sc[j][c] = -INFINITY;
        }
        mx[c >> 1] = fmaxf(mx[c >> 1], sc[j][c]);
      }
    }
    float ref[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
      mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
      ref[h] = mx[h] == -INFINITY ? 0.f : mx[h];
      const float fix = ex2_approx(m[h] - ref[h]);
      m[h] = mx[h];
      l[h] *= fix;
#pragma unroll
      for (int j = 0; j < D / 8; ++j) {
        o[j][2 * h] *= fix;
        o[j][2 * h + 1] *= fix;
      }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        sc[j][c] = ex2_approx(sc[j][c] - ref[c >> 1]);
        l[c >> 1] += sc[j][c];
      }
#pragma unroll
    for (int j = 0; j < NT; j += 2) {
      const uint32_t p[4] = {pack2(sc[j][0], sc[j][1]), pack2(sc[j][2], sc[j][3]),
                             pack2(sc[j + 1][0], sc[j + 1][1]), pack2(sc[j + 1][2], sc[j + 1][3])};
      const int key = wk * KW + j * 8 + (lane & 15);
#pragma unroll
      for (int dd = 0; dd < D / 16; ++dd) {
        uint32_t b[4];
        ldsm4_t(b, vs + key * D * 2 + (((dd * 2 + (lane >> 4)) ^ (lane & 7)) << 4));
        mma16816(o[2 * dd], p, b[0], b[1]);
        mma16816(o[2 * dd + 1], p, b[2], b[3]);
      }
    }
  }
  cp_async_wait<0>();
  __syncthreads();
  // The warps' sums meet in shared memory, in the stages' place.
  float *all = reinterpret_cast<float *>(smem + F::kKV);            // [WK][16 WR][D]
  float2 *ml = reinterpret_cast<float2 *>(smem + F::kMl);        // [WK][16 WR]
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int r = wk * 16 * WR + ra + 8 * h;
    if ((lane & 3) == 0) ml[r] = make_float2(m[h], l[h]);
#pragma unroll
    for (int j = 0; j < D / 8; ++j)
      *reinterpret_cast<float2 *>(all + r * D + j * 8 + 2 * (lane & 3)) =
          make_float2(o[j][2 * h], o[j][2 * h + 1]);
  }
  __syncthreads();
  const bool bad = *any_bad != 0;
  const bool whole = s.whole();
  float *part = whole ? nullptr : a.part + note_partial(a, s, cta, seg) * part_floats(M, D);
  for (int x = tid; x < s.rows * F::kChunks; x += kThreads) {
    const int r = x / F::kChunks, c = x % F::kChunks;
    float mx = -INFINITY, sum = 0.f, v[8] = {};
#pragma unroll
    for (int k = 0; k < WK; ++k) mx = fmaxf(mx, ml[k * 16 * WR + r].x);
    const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int k = 0; k < WK; ++k) {
      const float2 e = ml[k * 16 * WR + r];
      const float f = ex2_approx(e.x - ref);
      sum = fmaf(e.y, f, sum);
      const float4 *src = reinterpret_cast<const float4 *>(all + (k * 16 * WR + r) * D + c * 8);
      const float4 y = src[0], z = src[1];
      const float w[8] = {y.x, y.y, y.z, y.w, z.x, z.y, z.z, z.w};
#pragma unroll
      for (int e8 = 0; e8 < 8; ++e8) v[e8] = fmaf(w[e8], f, v[e8]);
    }
    if (bad) add_not_finite<D>(a, s, BN, r, c * 8, v);
    if (whole) {
      const RowAt at = row_at(a, s.row0, s.r0, s.h, r);
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      uint4 u;
      u.x = pack2(v[0] * inv, v[1] * inv);
      u.y = pack2(v[2] * inv, v[3] * inv);
      u.z = pack2(v[4] * inv, v[5] * inv);
      u.w = pack2(v[6] * inv, v[7] * inv);
      *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) +
                                 (at.token * a.Hq + at.head) * D + c * 8) = u;
      if (c == 0 && a.lse)
        a.lse[at.token * a.Hq + at.head] =
            sum == 0.f ? -INFINITY : (mx + log2f(sum)) * kLn2;
    } else {
      if (c == 0) {
        part[r] = mx;
        part[M + r] = sum;
      }
      float4 *dst = reinterpret_cast<float4 *>(part + 2 * M + r * D + c * 8);
      dst[0] = make_float4(v[0], v[1], v[2], v[3]);
      dst[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
}

template <int D>
__global__ void __launch_bounds__(kThreads, D <= 128 ? 3 : 1) attend_few_kernel(Args a) {
  extern __shared__ __align__(128) uint8_t smem[];
  const int cta = blockIdx.x, ctas = gridDim.x;
  if (a.rows_upto < INT32_MAX) let_next_start();  // the kernel for many rows
  clear_notes(a, cta);
  clear_spare_rows<__nv_bfloat16, D, kThreads>(a, cta, ctas);
  if (cta == ctas - 1)
    report_requests(a);
  Walk<M, Few<D>::BN> walk{
      find_share<kThreads>(a, M, cta, ctas, reinterpret_cast<int64_t *>(smem))};
  Segment s;
  for (int seg = 0; walk.next(a, &s); ++seg) {
    if (s.rows <= 16)
      few_segment<D, 1>(a, s, smem, cta, seg);
    else if (s.rows <= 32)
      few_segment<D, 2>(a, s, smem, cta, seg);
    else
      few_segment<D, 4>(a, s, smem, cta, seg);
  }
  let_next_start();
}

template <int D>
pair_status run_few(Launch *l, cudaStream_t s) {
  const Args &a = l->a;
  constexpr int smem = Few<D>::kBytes;
  PAIR_CUDA_TRY(cudaFuncSetAttribute(attend_few_kernel<D>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const int ctas = useful_ctas(a, M, min(kMaxCtas, (D <= 128 ? 3 : 1) * sm_count()));
  PAIR_BEGIN("attend_few", s);
  attend_few_kernel<D><<<ctas, kThreads, smem, s>>>(a);
  PAIR_LAUNCH_CHECK(s);
  l->M = M;
  l->ctas = ctas;
  return PAIR_OK;
}

}  // namespace

pair_status launch_few(Launch *l, int D, cudaStream_t s) {
  if (D == 64) return run_few<64>(l, s);
  if (D == 128) return run_few<128>(l, s);
  return run_few<256>(l, s);
}

}  // namespace attend
}  // namespace pairk
