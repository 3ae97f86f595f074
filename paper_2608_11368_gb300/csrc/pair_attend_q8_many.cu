// pair_attend_paged_q8 for chunks with many rows, bf16 queries: the kernel of
// pair_attend_tc.cuh over tiles that six warps form out of codes.
//
// A code times its row's power of two is a bf16 number, so a tile of stored values is
// exact and the products, the softmax and the epilogue are those over a bf16 cache. A
// former copies its rows' codes into shared memory (16 bytes per lane, asynchronously),
// one tile ahead; a lane then reads what it copied itself, so nobody waits for
// anybody's copy, forms 16 numbers of a piece (five instructions for four whole
// numbers, ten for four of e4m3) and stores them where the products read them.
#include <cuda_fp16.h>

#include "pair_attend_tc.cuh"

namespace pairk {
namespace attend {
namespace {

using q8::kE4M3;
using q8::kI8;

// CTA: warps 0-3 and 4-7 the softmax of a tile of 128 rows each, warp 9 the MMA issuer, warp
// 8 the scout, which finds the pages, warps 10 to 15 the formers. Registers: 200 x 256 + 56
// x 256 of the 128 x 512 that the block is launched with.
constexpr int kThreadsQ8 = 512;
constexpr int kFormers = 6;
constexpr int kOctets = BN / 8;  // of 8 keys, which lie in one page

// What a former has to know of a tile: where its keys and values lie.
struct Info {
  const uint8_t *src[kOctets][2];  // first row of each octet, keys and values
  uint8_t exps[2][BN];
  int32_t unseen, nk;  // keys that some row does not see, that do not exist: from here on
  int32_t more;        // there is a tile
};

template <int D>
struct SmemQ8 {
  static constexpr int kKeyStages = 2, kValueStages = 2;  // rings of tiles
  uint8_t q[2][Tc<D>::kTile];
  uint8_t k[kKeyStages][Tc<D>::kTile];
  uint8_t v[kValueStages][Tc<D>::kTile];
  uint4 codes[2][BN * D / 16];  // of the next tile of keys, of values
  Info info[2];
  uint64_t k_full[kKeyStages], k_empty[kKeyStages];
  uint64_t looked[kValueStages], v_empty[kValueStages];
  uint64_t info_full[2], info_empty[2];
  uint64_t done, q_full[2], s_full[2], p_ready[2][2], pv_done[2];
  int64_t scratch[kThreadsQ8 / 32 + 2];
  uint32_t tmem;
  int abort, any_bad;
};

__device__ __forceinline__ uint32_t bits(__nv_bfloat162 x) {
  return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ __nv_bfloat162 bf2_of(uint32_t x) {
  return *reinterpret_cast<const __nv_bfloat162 *>(&x);
}

// Tiles hold the stored values over kHeldUnit, so that a whole number takes one
// multiply-add for all scales that are met: its byte u = code + 128 is as a bf16 number u
// 2^-133 (below 128 a subnormal one, from there on one of the least exponent, in the same
// steps), and u 2^-133 2^(125 + e) - 2^(-1 + e) is code 2^(e - 8), e = b - 127 up to 2: rows
// up to 508. An e4m3 number's exponent and significand at bf16's places are the code times
// 2^-120, and its factor 2^(112 + e), e up to 15. Rows beyond take a second factor.
template <int F>
constexpr int kMost = F == kI8 ? 129 : 142;  // exponent bytes that one factor does for

// (Both factors of a row are pairs of bf16 numbers in a word: the multiplier or second
// factor, and what is subtracted or nothing.)
template <int F>
__device__ __forceinline__ uint32_t factor_of(uint32_t b) {
  // bf16 numbers by their exponent fields (2^-127 and 2^-128 have none).
  if (b == 255) return 0x7fc00000u | 0x7fc0u;
  const uint32_t c = min(b, (uint32_t)kMost<F>);
  if constexpr (F == kI8)  // 2^(125 + e), -2^(e - 1)
    return ((c + 125) << 7) | ((c > 1 ? (c - 1) << 7 : 0x20u << c) << 16) | 0x80000000u;
  else
    return (c + 112) << 7;
}
template <int F>
__device__ __forceinline__ uint32_t rest_of(uint32_t b) {
  return b == 255 || b <= (uint32_t)kMost<F> ? 0x3f803f80u
                                              : (127u + b - kMost<F>) * 0x00800080u;
}

// Four codes times a row's factor f; g: what is subtracted (whole numbers).
template <int F>
__device__ __forceinline__ uint2 form4(uint32_t w, uint32_t f, uint32_t g) {
  uint2 x;
  if constexpr (F == kI8) {
    w ^= 0x80808080u;
    x.x = bits(__hfma2(bf2_of(__byte_perm(w, 0, 0x4140)), bf2_of(f), bf2_of(g)));
    x.y = bits(__hfma2(bf2_of(__byte_perm(w, 0, 0x4342)), bf2_of(f), bf2_of(g)));
  } else {
    const uint32_t y = __byte_perm(w, 0, 0x1404), z = __byte_perm(w, 0, 0x3424);
    x.x = bits(__hmul2(bf2_of(((y >> 4) & 0x07f007f0u) | (y & 0x80008000u)), bf2_of(f)));
    x.y = bits(__hmul2(bf2_of(((z >> 4) & 0x07f007f0u) | (z & 0x80008000u)), bf2_of(f)));
  }
  return x;
}

// Warp 8: the pages of every tile, two tiles ahead of the formers at most. Lanes 0 to 15
// look up an octet each, all of them the exponents of four keys and values.
template <int D>
__device__ void scout(const Args &a, SmemQ8<D> &sm, Walk<M, BN> walk) {
  const int lane = threadIdx.x & 31;
  volatile int *abort = &sm.abort;
  Ring<2> ring;
  Segment s;
  const int by = BN / a.page, by_off = BN - by * a.page;
  bool ok = true;
  while (ok && walk.next(a, &s)) {
    const int32_t *table = a.table + (int64_t)s.i * a.width;
    int key = s.t0 * BN + (lane & 15) * 8, at = key / a.page, off = key - at * a.page;
    int id = key < s.keys ? table[at] : 0;
    for (int t = s.t0; t < s.t1; ++t) {
      const bool there = key < s.keys;
      int pg = id;
      const int o = off;
      if (there && (unsigned)pg >= (unsigned)a.num_pages) {
        flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
        pg = 0;
      }
      // The next tile's pages are on their way meanwhile.
      key += BN;
      at += by;
      off += by_off;
      if (off >= a.page) {
        off -= a.page;
        ++at;
      }
      if (t + 1 < s.t1) id = key < s.keys ? table[at] : 0;
      const int nk = min(BN, s.keys - t * BN);
      uint32_t e[2] = {0, 0};
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // keys lane + 32 x
        const int from = (lane >> 3) + 4 * x;
        const int p = __shfl_sync(0xffffffffu, pg, from), q = __shfl_sync(0xffffffffu, o, from);
        uint32_t k = 127, v = 127;
        if (lane + 32 * x < nk) {
          k = __ldg(a.ke + cache_row(a, a.kes, p, q + (lane & 7), s.h));
          v = __ldg(a.ve + cache_row(a, a.ves, p, q + (lane & 7), s.h));
        }
        e[0] |= k << 8 * x;
        e[1] |= v << 8 * x;
      }
      if (!(ok = warp_wait(&sm.info_empty[ring.stage], ring.phase ^ 1, abort, a.dev_err))) break;
      Info &info = sm.info[ring.stage];
      if (lane < kOctets) {
        info.src[lane][0] = static_cast<const uint8_t *>(a.kc) +
                            (there ? cache_row(a, a.ks, pg, o, s.h) : 0);
        info.src[lane][1] = static_cast<const uint8_t *>(a.vc) +
                            (there ? cache_row(a, a.vs, pg, o, s.h) : 0);
      }
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int x = 0; x < 4; ++x) info.exps[kv][lane + 32 * x] = (uint8_t)(e[kv] >> 8 * x);
      if (lane == 0) {
        info.unseen = edge_tile(s, t) ? max(0, s.least - t * BN) : BN;
        info.nk = nk;
        info.more = 1;
      }
      warp_arrive(&sm.info_full[ring.stage]);
      ring.step();
    }
  }
  if (ok && warp_wait(&sm.info_empty[ring.stage], ring.phase ^ 1, abort, a.dev_err)) {
    if (lane == 0) sm.info[ring.stage].more = 0;
    warp_arrive(&sm.info_full[ring.stage]);
  }
}

// Warps 10 to 15 (w = 0 to 5): the octets w, w + 6, .. of every tile. A lane has row lane %
// 8 of each and, of its 16-byte pieces, lane / 8 (and 4 behind that).
template <int D, int F>
struct Former {
  using C = Tc<D>;
  static constexpr int kOwn = (kOctets + kFormers - 1) / kFormers, PP = D / 64;
  const Args &a;
  SmemQ8<D> &sm;
  const int w, lane;

  // The codes of a tile, zeros where there is no key.
  __device__ __forceinline__ void copy(int kv, const Info &info) {
    const int64_t step = (lane & 7) * (kv ? a.vs : a.ks).for_token + (lane >> 3) * 16;
    const uint32_t dst = smem_u32(&sm.codes[kv][w * PP * 32 + lane]);
#pragma unroll
    for (int o = 0; o < kOwn; ++o) {
      const int octet = o * kFormers + w;
      if (octet >= kOctets) continue;
      const bool there = octet * 8 + (lane & 7) < info.nk;
      const uint8_t *src = info.src[octet][kv] + (there ? step : 0);
#pragma unroll
      for (int y = 0; y < PP; ++y)
        cp_async16(dst + (o * kFormers * PP + y) * 512, src + (there ? y * 64 : 0), there);
    }
    cp_async_commit();
  }
  // Forms a tile out of its codes. (The same code for keys and values: it has to fit in
  // the instruction caches beside the softmax's.)
  __device__ __forceinline__ void put(int kv, uint8_t *to, const Info &info) {
    const int c = (lane >> 3) * 2, r7 = lane & 7;
    uint8_t *row = to + (w * 8 + r7) * 128;
    const uint32_t c0 = (c ^ r7) << 4, c1 = ((c + 1) ^ r7) << 4;
    const uint4 *codes = &sm.codes[kv][w * PP * 32 + lane];
    const uint8_t *exps = &info.exps[kv][w * 8 + r7];
#pragma unroll 1
    for (int o = w; o < kOctets; o += kFormers, codes += kFormers * PP * 32,
             row += kFormers * 8 * 128, exps += kFormers * 8) {
      uint4 u[PP];
#pragma unroll
      for (int y = 0; y < PP; ++y) u[y] = codes[y * 32];
      const uint32_t b = *exps;
      uint32_t fg = factor_of<F>(b);
      if (kv && b == 255 && o * 8 + r7 >= info.unseen) {  // zero times NaN is NaN
        fg = 0;
        *reinterpret_cast<volatile int *>(&sm.any_bad) = 1;
      }
      const uint32_t f = __byte_perm(fg, 0, 0x1010), g = __byte_perm(fg, 0, 0x3232);
      const bool beyond = __any_sync(0xffffffffu, b > kMost<F>);
#pragma unroll
      for (int y = 0; y < PP; ++y) {
        // Piece lane / 8 + 4 y of 16 columns: chunks 2 (lane / 8) and the next of atom y.
        uint2 x[4] = {form4<F>(u[y].x, f, g), form4<F>(u[y].y, f, g), form4<F>(u[y].z, f, g),
                      form4<F>(u[y].w, f, g)};
        if (beyond) {
          const uint32_t rest = rest_of<F>(b);
#pragma unroll
          for (int k = 0; k < 4; ++k)
            x[k] = make_uint2(bits(__hmul2(bf2_of(x[k].x), bf2_of(rest))),
                              bits(__hmul2(bf2_of(x[k].y), bf2_of(rest))));
        }
        *reinterpret_cast<uint4 *>(row + y * C::kAtom + c0) =
            make_uint4(x[0].x, x[0].y, x[1].x, x[1].y);
        *reinterpret_cast<uint4 *>(row + y * C::kAtom + c1) =
            make_uint4(x[2].x, x[2].y, x[3].x, x[3].y);
      }
    }
    fence_async_smem();
  }

  __device__ void run() {
    volatile int *abort = &sm.abort;
    Ring<2> at, next;  // the tile's place in the rings (all of two stages), the next one's
    bool ok = warp_wait(&sm.info_full[0], 0, abort, a.dev_err);
    bool more = ok && sm.info[0].more;
    if (more) {
      copy(0, sm.info[0]);
      copy(1, sm.info[0]);
    }
    while (more) {
      const Info &info = sm.info[at.stage];
      if (!warp_wait(&sm.k_empty[at.stage], at.phase ^ 1, abort, a.dev_err)) break;
      cp_async_wait<1>();
      put(0, sm.k[at.stage], info);
      warp_arrive(&sm.k_full[at.stage]);
      next = at;
      next.step();
      if (!warp_wait(&sm.info_full[next.stage], next.phase, abort, a.dev_err)) break;
      more = sm.info[next.stage].more;
      if (more)
        copy(0, sm.info[next.stage]);
      else
        cp_async_commit();
      if (!warp_wait(&sm.v_empty[at.stage], at.phase ^ 1, abort, a.dev_err)) break;
      cp_async_wait<1>();
      put(1, sm.v[at.stage], info);
      warp_arrive(&sm.looked[at.stage]);
      warp_arrive(&sm.info_empty[at.stage]);
      if (more)
        copy(1, sm.info[next.stage]);
      else
        cp_async_commit();
      at = next;
    }
    cp_async_wait<0>();  // nothing is on its way into shared memory when the CTA ends
  }
};

template <int D, int F>
__global__ void __launch_bounds__(kThreadsQ8, 1) attend_q8_many_kernel(Args a) {
  extern __shared__ uint8_t raw[];
  SmemQ8<D> &sm = *reinterpret_cast<SmemQ8<D> *>(tck::align1k(raw));
  const int tid = threadIdx.x, warp = tid >> 5;
  const int cta = blockIdx.x, ctas = gridDim.x;
  clear_notes(a, cta);
  if (a.rows_over < 0) {
    clear_spare_rows<__nv_bfloat16, D, kThreadsQ8>(a, cta, ctas);
    if (cta == ctas - 1) report_requests(a);
  }
  if (tid == 0) {
    for (int x = 0; x < SmemQ8<D>::kKeyStages; ++x) {
      mbar_init(&sm.k_full[x], kFormers);
      mbar_init(&sm.k_empty[x], 1);
    }
    for (int x = 0; x < SmemQ8<D>::kValueStages; ++x) {
      mbar_init(&sm.looked[x], kFormers);
      mbar_init(&sm.v_empty[x], 1);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(&sm.info_full[x], 1);
      mbar_init(&sm.info_empty[x], kFormers);
    }
    mbar_init(&sm.done, 1);
    for (int w = 0; w < 2; ++w) {
      mbar_init(&sm.q_full[w], 4);
      mbar_init(&sm.s_full[w], 1);
      mbar_init(&sm.p_ready[w][0], 4);
      mbar_init(&sm.p_ready[w][1], 4);
      mbar_init(&sm.pv_done[w], 1);
    }
    sm.abort = 0;
    sm.any_bad = 0;
    fence_mbar_init();
  }
  __syncwarp();
  if (warp == 9) tmem_alloc(&sm.tmem, 512);
  const Walk<M, BN> walk{find_share<kThreadsQ8>(a, M, cta, ctas, sm.scratch)};
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 9)
      issue<D>(a, sm, walk);
    else if (warp == 8)
      scout<D>(a, sm, walk);
    else
      Former<D, F>{a, sm, warp - 10, tid & 31}.run();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
    softmax<D, F>(a, sm, walk, cta);
  }
  __syncwarp();
  let_next_start();
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_relinquish();
    tmem_dealloc(sm.tmem, 512);
  }
  if (a.rows_over >= 0) wait_for_previous();
}

template <int D, int F>
pair_status run_many(Launch *l, cudaStream_t s) {
  Args &a = l->a;
  a.unit_cost = kManyCost;
  constexpr int smem = sizeof(SmemQ8<D>) + 1024;
  static_assert(smem <= 232448, "shared memory of a CTA");
  const auto kernel = attend_q8_many_kernel<D, F>;
  PAIR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const int ctas = useful_ctas(a, M, min(kMaxMany, sm_count()));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas, 1, 1);
  cfg.blockDim = dim3(kThreadsQ8, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = a.rows_over >= 0 ? 1 : 0;  // behind the launch for few rows
  PAIR_BEGIN("attend_q8_many", s);
  if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) {
    cudaGetLastError();
    return PAIR_ERR_CUDA;
  }
  PAIR_LAUNCH_CHECK(s);
  l->M = M;
  l->ctas = ctas;
  return PAIR_OK;
}

}  // namespace

bool many_applies_q8(const Args &a, int D) { return D <= 128 && a.page % 8 == 0; }

pair_status launch_many_q8(Launch *l, int D, int fmt, cudaStream_t s) {
  if (fmt == kI8) return D == 64 ? run_many<64, kI8>(l, s) : run_many<128, kI8>(l, s);
  return D == 64 ? run_many<64, kE4M3>(l, s) : run_many<128, kE4M3>(l, s);
}

}  // namespace attend
}  // namespace pairk
