// pair_attend_paged_q8 for chunks with many rows, bf16 queries: the kernel of
// pair_attend_tc.cuh over tiles that six warps form out of codes.
//
// A code times its row's power of two is a bf16 number, so a tile of stored values is
// exact and the products, the softmax and the epilogue are those over a bf16 cache. A
// former reads 16 codes per lane out of shared memory, where TMA brings a tile of them,
// forms the numbers (five instructions for four whole ones, ten for four of e4m3) and
// stores them where the products read them.
//
// Four chunks of 1025 to 2048 tokens behind 1000 to 6144 (32/8 heads of 128, 0.44 TFLOP as
// the mean of their lengths): 510 us, 0.86 PFLOP/s, over whole numbers and 530 over e4m3,
// where a bf16 cache of the same lengths takes 390. The difference is the formers' stores,
// 64 KB a tile into the shared memory that the products read: without them 453 us, with
// or without their arithmetic. Measured and not kept: codes into registers instead of
// shared memory (755 us: the registers that the softmax leaves, 64, hold too few on their
// way), by 16-byte copies of the formers' own (585), three formers of 104 registers beside
// a softmax of 200 (941), four formers (546, e4m3 607).
#include <cuda_fp16.h>

#include "pair_attend_tc.cuh"

namespace pairk {
namespace attend {
namespace {

using q8::kE4M3;
using q8::kI8;

// CTA: warps 0-3 and 4-7 the softmax of a tile of 128 rows each, warp 9 the MMA issuer, warp
// 8 the scout, which finds the pages, warps 10 to 15 the formers. Registers: 192 x 256 + 64
// x 256 of the 128 x 512 that the block is launched with.
constexpr int kThreadsQ8 = 512;
constexpr int kFormers = 6;
constexpr int kOctets = BN / 8;  // of 8 keys, which lie in one page

// A warp's way along the CTA's share, in shared memory, stepped by its lane 0: registers
// are short.
struct Way {
  Walk<M, BN> walk;
  Segment s;
  bool more;
};
struct SharedWalk {
  Way &way;
  __device__ __forceinline__ bool next(const Args &a, Segment *s) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) way.more = way.walk.next(a, &way.s);
    __syncwarp();
    *s = way.s;
    return way.more;
  }
};

// What a former has to know of a tile beside its codes.
struct Info {
  uint8_t exps[2][BN];  // of keys, of values
  int32_t unseen, nk;   // keys that some row does not see, that do not exist: from here on
  int32_t more;         // there is a tile
};

template <int D>
struct SmemQ8 {
  static constexpr bool kLean = true;  // waits of the issuer
  static constexpr int kKeyStages = 2, kValueStages = 2;  // rings of tiles
  uint8_t q[2][Tc<D>::kTile];
  uint8_t k[kKeyStages][Tc<D>::kTile];
  uint8_t v[kValueStages][Tc<D>::kTile];
  uint8_t codes[2][BN * D];  // of the next tile of keys, of values
  Info info[2];
  uint64_t k_full[kKeyStages], k_empty[kKeyStages];
  uint64_t looked[kValueStages], v_empty[kValueStages];
  uint64_t info_full[2], info_empty[2], codes_full[2], codes_empty[2];
  uint64_t done, q_full[2], s_full[2], p_ready[2][2], pv_done[2];
  int64_t scratch[kThreadsQ8 / 32 + 2];
  Way way[2];  // the scout's and the issuer's
  uint32_t tmem;
  int abort, any_bad;
};

__device__ __forceinline__ uint32_t bits(__nv_bfloat162 x) {
  return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ __nv_bfloat162 bf2_of(uint32_t x) {
  return *reinterpret_cast<const __nv_bfloat162 *>(&x);
}

__device__ __forceinline__ uint32_t ld_shared32(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ uint32_t ld_shared8(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ uint4 ld_shared128(uint32_t at) {
  uint4 u;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
               : "r"(at)
               : "memory");
  return u;
}
__device__ __forceinline__ void st_shared128(uint32_t at, uint32_t x, uint32_t y, uint32_t z,
                                             uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
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

// Warp 8: brings the codes of every tile into shared memory by TMA, a box of tokens of one
// page per lane, and the exponents of its keys and values.
template <int D>
__device__ void scout(const Args &a, const Maps &maps, SmemQ8<D> &sm, SharedWalk walk) {
  const int lane = threadIdx.x & 31;
  const auto wait = [&](uint64_t *bar, uint32_t phase) {
    const bool ok = wait_lean(smem_u32(bar), phase, smem_u32(&sm.abort), a.dev_err);
    return __all_sync(0xffffffffu, ok);
  };
  Ring<2> ring;
  Ring<1> codes;
  Segment s;
  const int box = maps.box, by = BN / a.page, by_off = BN - by * a.page;
  const int box_bits = __ffs(box) - 1;
  const bool mine = lane * box < BN;
  bool ok = true;
  while (ok && walk.next(a, &s)) {
    // Of a unit that comes next, the queries too are fetched from afar beforehand.
    for (int r = lane; r < s.rows; r += 32) {
      const RowAt w = row_at(a, s.row0, s.r0, s.h, r);
      const uint8_t *p = static_cast<const uint8_t *>(a.q) +
                         (w.token * a.q_row + w.head * a.q_head) * sizeof(__nv_bfloat16);
      for (int x = 0; x < D * 2; x += 128)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(p + x));
    }
    const int32_t *table = a.table + (int64_t)s.i * a.width;
    int key = s.t0 * BN + lane * box, at = key / a.page, off = key - at * a.page;
    int id = mine && key < s.keys ? table[at] : 0;
    // Pages, places and exponents of the tile at hand; those of the next one are on
    // their way while it is brought in.
    int pg, o, nk;
    bool load;
    uint32_t exps[2][4];
    auto look = [&](int t) {
      load = mine && key < s.keys;
      pg = id;
      o = off;
      if (load && (unsigned)pg >= (unsigned)a.num_pages) {
        flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
        pg = 0;
      }
      key += BN;
      at += by;
      off += by_off;
      if (off >= a.page) {
        off -= a.page;
        ++at;
      }
      if (t + 1 < s.t1) id = mine && key < s.keys ? table[at] : 0;
      nk = min(BN, s.keys - t * BN);
#pragma unroll
      for (int x = 0; x < 4; ++x) {  // keys lane + 32 x
        const int k = lane + 32 * x, from = k >> box_bits, in = k & (box - 1);
        const int p = __shfl_sync(0xffffffffu, pg, from), q = __shfl_sync(0xffffffffu, o, from);
        exps[0][x] = exps[1][x] = 127;
        if (k < nk) {
          exps[0][x] = __ldg(a.ke + cache_row(a, a.kes, p, q + in, s.h));
          exps[1][x] = __ldg(a.ve + cache_row(a, a.ves, p, q + in, s.h));
        }
      }
    };
    look(s.t0);
    for (int t = s.t0; t < s.t1; ++t) {
      const int boxes = __popc(__ballot_sync(0xffffffffu, load));
      auto bring = [&](int kv) {
        if (!wait(&sm.codes_empty[kv], codes.phase ^ 1)) return false;
        if (lane == 0) mbar_expect_tx(&sm.codes_full[kv], boxes * box * D);
        __syncwarp();
        if (load) {
          const int8_t *where = kv ? maps.v_at : maps.k_at;
          const int c1 = where[0] == 1 ? pg : where[1] == 1 ? o : s.h;
          const int c2 = where[0] == 2 ? pg : where[1] == 2 ? o : s.h;
          const int c3 = where[0] == 3 ? pg : where[1] == 3 ? o : s.h;
          tma_load_4d(sm.codes[kv] + lane * box * D, kv ? &maps.v : &maps.k, &sm.codes_full[kv],
                      0, c1, c2, c3);
        }
        return true;
      };
      if (!(ok = bring(0))) break;
      if (!(ok = wait(&sm.info_empty[ring.stage], ring.phase ^ 1))) break;
      Info &info = sm.info[ring.stage];
#pragma unroll
      for (int kv = 0; kv < 2; ++kv)
#pragma unroll
        for (int x = 0; x < 4; ++x) info.exps[kv][lane + 32 * x] = (uint8_t)exps[kv][x];
      if (lane == 0) {
        info.unseen = edge_tile(s, t) ? max(0, s.least - t * BN) : BN;
        info.nk = nk;
        info.more = 1;
      }
      warp_arrive(&sm.info_full[ring.stage]);
      ring.step();
      if (!(ok = bring(1))) break;
      codes.step();
      if (t + 1 < s.t1) look(t + 1);
    }
  }
  if (ok && wait(&sm.info_empty[ring.stage], ring.phase ^ 1)) {
    if (lane == 0) sm.info[ring.stage].more = 0;
    warp_arrive(&sm.info_full[ring.stage]);
  }
  // Nothing may still be on its way into shared memory when the CTA ends. On the regular
  // path all codes have been consumed; after an abort the last ones are waited for, each
  // barrier's latest use that was begun.
  if (!ok) {
    volatile int never = 0;
    for (int kv = 0; kv < 2; ++kv) {
      wait_limit(&sm.codes_full[kv], codes.phase ^ 1, &never, a.dev_err, 10000000);
      wait_limit(&sm.codes_full[kv], codes.phase, &never, a.dev_err, 10000000);
    }
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

  __device__ __forceinline__ bool wait(uint64_t *bar, uint32_t phase) {
    const bool ok = wait_lean(smem_u32(bar), phase, smem_u32(&sm.abort), a.dev_err);
    return __all_sync(0xffffffffu, ok);
  }
  // Stores a piece's 16 numbers: chunks c and c + 1, c = 2 (lane / 8), of an atom's row at
  // `at` (turned by the row).
  template <bool rest>
  __device__ __forceinline__ void form(uint32_t at, const uint4 &u, uint32_t fg, uint32_t more) {
    const uint32_t f = __byte_perm(fg, 0, 0x1010), g = __byte_perm(fg, 0, 0x3232);
    uint2 x[4] = {form4<F>(u.x, f, g), form4<F>(u.y, f, g), form4<F>(u.z, f, g),
                  form4<F>(u.w, f, g)};
    if (rest) {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        x[k] = make_uint2(bits(__hmul2(bf2_of(x[k].x), bf2_of(more))),
                          bits(__hmul2(bf2_of(x[k].y), bf2_of(more))));
    }
    st_shared128(at, x[0].x, x[0].y, x[1].x, x[1].y);
    st_shared128(at ^ 16, x[2].x, x[2].y, x[3].x, x[3].y);
  }

  __device__ void run() {
    Ring<2> at;  // the tile's place in the rings of two stages
    Ring<1> codes;
    const uint32_t infos = smem_u32(&sm.info[0]);
    const int r7 = lane & 7, p = lane >> 3;
    const bool last = w + (kOwn - 1) * kFormers < kOctets;  // has as many octets as others
#pragma unroll 1
    while (true) {
      const uint32_t info = infos + at.stage * sizeof(Info);
      if (!wait(&sm.info_full[at.stage], at.phase)) return;
      if (ld_shared32(info + offsetof(Info, more)) == 0) return;
      // (The same code for keys and values: it has to fit in the instruction caches
      // beside the softmax's.)
#pragma unroll 1
      for (int kv = 0; kv < 2; ++kv) {
        uint32_t fg[kOwn], b[kOwn];
        bool beyond = false;
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
          const int key = min(o * kFormers + w, kOctets - 1) * 8 + r7;
          b[o] = ld_shared8(info + offsetof(Info, exps) + kv * BN + key);
        }
        // Codes as TMA's swizzle has placed them: of 128 bytes a row's pieces are turned by
        // the row, of 64 by half of it.
        if (!wait(&sm.codes_full[kv], codes.phase)) return;
        uint4 u[kOwn][PP];
        const uint32_t from = smem_u32(sm.codes[kv]) + (w * 8 + r7) * D;
#pragma unroll
        for (int o = 0; o < kOwn; ++o)
#pragma unroll
          for (int y = 0; y < PP; ++y)
            if (o < kOwn - 1 || last)
              u[o][y] = ld_shared128(from + o * kFormers * 8 * D +
                                     ((p + 4 * y) ^ (D == 64 ? r7 >> 1 : r7)) * 16);
#pragma unroll
        for (int o = 0; o < kOwn; ++o) {
          fg[o] = factor_of<F>(b[o]);
          beyond |= b[o] > kMost<F>;
        }
        if (kv) {
          // No row's value must meet a weight of 0 as NaN, nor be what was there before.
          const int unseen = ld_shared32(info + offsetof(Info, unseen));
          if (unseen < BN) {
            const int nk = ld_shared32(info + offsetof(Info, nk));
#pragma unroll
            for (int o = 0; o < kOwn; ++o) {
              const int key = (o * kFormers + w) * 8 + r7;
              const bool bad = b[o] == 255 && key >= unseen;
              if (bad) *reinterpret_cast<volatile int *>(&sm.any_bad) = 1;
              if (bad || key >= nk) fg[o] = 0;
            }
          }
        }
        if (!wait(kv ? &sm.v_empty[at.stage] : &sm.k_empty[at.stage], at.phase ^ 1)) return;
        warp_arrive(&sm.codes_empty[kv]);
        const uint32_t to = smem_u32(kv ? sm.v[0] : sm.k[0]) + at.stage * C::kTile +
                            (w * 8 + r7) * 128 + ((2 * p ^ r7) << 4);
        if (!__any_sync(0xffffffffu, beyond)) {
#pragma unroll
          for (int o = 0; o < kOwn; ++o)
#pragma unroll
            for (int y = 0; y < PP; ++y)
              if (o < kOwn - 1 || last)
                form<false>(to + y * C::kAtom + o * (kFormers * 8 * 128), u[o][y], fg[o], 0);
        } else {
#pragma unroll
          for (int o = 0; o < kOwn; ++o)
#pragma unroll
            for (int y = 0; y < PP; ++y)
              if (o < kOwn - 1 || last)
                form<true>(to + y * C::kAtom + o * (kFormers * 8 * 128), u[o][y], fg[o],
                           rest_of<F>(b[o]));
        }
        fence_async_smem();
        warp_arrive(kv ? &sm.looked[at.stage] : &sm.k_full[at.stage]);
      }
      warp_arrive(&sm.info_empty[at.stage]);
      at.step();
      codes.step();
    }
  }
};

template <int D, int F>
__global__ void __launch_bounds__(kThreadsQ8, 1)
    attend_q8_many_kernel(Args a, const __grid_constant__ Maps maps) {
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
      mbar_init(&sm.codes_full[x], 1);
      mbar_init(&sm.codes_empty[x], kFormers);
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
    prefetch_tmap(&maps.k);
    prefetch_tmap(&maps.v);
  }
  __syncwarp();
  if (warp == 9) tmem_alloc(&sm.tmem, 512);
  const Walk<M, BN> walk{find_share<kThreadsQ8>(a, M, cta, ctas, sm.scratch)};
  if (tid == 0) sm.way[0].walk = sm.way[1].walk = walk;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (warp == 9)
      issue<D>(a, sm, SharedWalk{sm.way[1]});
    else if (warp == 8)
      scout<D>(a, maps, sm, SharedWalk{sm.way[0]});
    else
      Former<D, F>{a, sm, warp - 10, tid & 31}.run();
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
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
pair_status run_many(Launch *l, const Maps &maps, cudaStream_t s) {
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
  if (cudaLaunchKernelEx(&cfg, kernel, a, maps) != cudaSuccess) {
    cudaGetLastError();
    return PAIR_ERR_CUDA;
  }
  PAIR_LAUNCH_CHECK(s);
  l->M = M;
  l->ctas = ctas;
  return PAIR_OK;
}

}  // namespace

bool many_applies_q8(const Args &a, int D) {
  Maps maps;
  return many_maps(a, D, 1, &maps);
}

pair_status launch_many_q8(Launch *l, int D, int fmt, cudaStream_t s) {
  Maps maps;
  if (!many_maps(l->a, D, 1, &maps)) return PAIR_ERR_CUDA;
  if (fmt == kI8) return D == 64 ? run_many<64, kI8>(l, maps, s) : run_many<128, kI8>(l, maps, s);
  return D == 64 ? run_many<64, kE4M3>(l, maps, s) : run_many<128, kE4M3>(l, maps, s);
}

}  // namespace attend
}  // namespace pairk
