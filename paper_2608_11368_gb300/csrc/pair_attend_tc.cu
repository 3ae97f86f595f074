// pair_attend_paged for chunks with many rows, bf16: keys and values by TMA into the layout
// that the products read. Warps 8 and 10 are the producers of keys and of values, warp 11
// looks values over.
#include "pair_attend_tc.cuh"

namespace pairk {
namespace attend {
namespace {

template <int D>
struct Smem {
  static constexpr bool kLean = false;
  static constexpr int kKeyStages = D == 64 ? 4 : 2;    // ring of key tiles
  static constexpr int kValueStages = D == 64 ? 4 : 3;  // ring of value tiles
  uint8_t q[2][Tc<D>::kTile];
  uint8_t k[kKeyStages][Tc<D>::kTile];
  uint8_t v[kValueStages][Tc<D>::kTile];
  uint64_t k_full[kKeyStages], k_empty[kKeyStages];
  uint64_t v_full[kValueStages], v_empty[kValueStages];
  uint64_t looked[kValueStages];  // values are there and, in an edge tile, looked over
  uint64_t done, q_full[2], s_full[2], p_ready[2][2], pv_done[2];
  int64_t scratch[kThreads / 32 + 2];
  uint32_t tmem;
  int abort, any_bad;
};

// Keys (kv = 0) or values (1) of every tile, a box per lane. A warp each: the
// 16 boxes of a tile of pages of 16 take some 1300 cycles to issue, and one warp
// for both kept the products waiting. The page of the tile after the next one is
// on its way meanwhile.
template <int D, int kv>
__device__ void produce(const Args &a, const Maps &maps, Smem<D> &sm, Walk<M, BN> walk) {
  using C = Tc<D>;
  const int lane = threadIdx.x & 31;
  volatile int *abort = &sm.abort;
  constexpr int ST = kv ? Smem<D>::kValueStages : Smem<D>::kKeyStages;
  Ring<ST> ring;
  uint64_t *full = kv ? sm.v_full : sm.k_full, *empty = kv ? sm.v_empty : sm.k_empty;
  int issued = 0;
  const int box = maps.box;
  const bool mine = lane * box < BN;
  const int8_t *where = kv ? maps.v_at : maps.k_at;
  const CUtensorMap *map = kv ? &maps.v : &maps.k;
  const int by = BN / a.page, by_off = BN % a.page;  // a tile's way in the table
  bool ok = true;
  Segment s;
  while (ok && walk.next(a, &s)) {
    int key = s.t0 * BN + lane * box, at = key / a.page, off = key - at * a.page;
    const int32_t *row = a.table + (int64_t)s.i * a.width;
    const int end = min(s.keys, s.t1 * BN);
    int id = mine && key < end ? row[at] : 0;
    for (int t = s.t0; t < s.t1; ++t) {
      const bool load = mine && key < end;
      const int cur_off = off;
      int cur = id;
      key += BN;
      at += by;
      off += by_off;
      if (off >= a.page) {
        off -= a.page;
        ++at;
      }
      if (mine && key < end) id = row[at];
      if (!(ok = warp_wait(&empty[ring.stage], ring.phase ^ 1, abort, a.dev_err))) break;
      uint64_t *bar = &full[ring.stage];
      const int n = __popc(__ballot_sync(0xffffffffu, load));
      if (lane == 0) mbar_expect_tx(bar, n * box * D * 2);
      __syncwarp();
      if (load) {
        if ((unsigned)cur >= (unsigned)a.num_pages) {
          flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
          cur = 0;
        }
        const int c1 = where[0] == 1 ? cur : where[1] == 1 ? cur_off : s.h;
        const int c2 = where[0] == 2 ? cur : where[1] == 2 ? cur_off : s.h;
        const int c3 = where[0] == 3 ? cur : where[1] == 3 ? cur_off : s.h;
        uint8_t *dst = (kv ? sm.v[ring.stage] : sm.k[ring.stage]) + lane * box * 128;
#pragma unroll
        for (int x = 0; x < C::kAtoms; ++x)
          tma_load_4d(dst + x * C::kAtom, map, bar, x * 64, c1, c2, c3);
      }
      ++issued;
      ring.step();
    }
  }
  // Nothing may still be on its way into shared memory when the CTA ends: on
  // the regular path every tile has been consumed; after an abort the last
  // ones are waited for here (the barrier of a stage completes once per use).
  if (!ok) {
    volatile int never = 0;
    Ring<ST> r;
    for (int x = 0; x < issued; ++x, r.step())
      if (x >= issued - ST) wait_limit(&full[r.stage], r.phase, &never, a.dev_err, 10000000);
  }
}

// Of every tile: waits for the values, and in an edge tile makes those of keys
// from `nk` on 0, and among those that some row does not see (from `from` on) what
// is not finite too (add_not_finite brings it back for the rows that see it).
template <int D>
__device__ void look_over(const Args &a, Smem<D> &sm, Walk<M, BN> walk) {
  using C = Tc<D>;
  const int lane = threadIdx.x & 31;
  volatile int *abort = &sm.abort;
  Ring<Smem<D>::kValueStages> ring;
  Segment s;
  while (walk.next(a, &s)) {
    for (int t = s.t0; t < s.t1; ++t) {
      const bool ok = wait(&sm.v_full[ring.stage], ring.phase, abort, a.dev_err);
      if (ok && edge_tile(s, t)) {
        const int from = max(0, s.least - t * BN), nk = min(BN, s.keys - t * BN);
        for (int atom = 0; atom < C::kAtoms; ++atom) {
          uint4 *base = reinterpret_cast<uint4 *>(sm.v[ring.stage] + atom * C::kAtom);
#pragma unroll 4
          for (int x = from * 8 + lane; x < BN * 8; x += 32) {
            if ((x >> 3) >= nk) {
              base[x] = make_uint4(0, 0, 0, 0);
              continue;
            }
            uint4 u = base[x];
            // Zero times what is not finite is NaN.
            const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
            const __nv_bfloat162 *v = reinterpret_cast<const __nv_bfloat162 *>(&u);
            const __nv_bfloat162 y = __hfma2(
                v[0], zero, __hfma2(v[1], zero, __hfma2(v[2], zero, __hmul2(v[3], zero))));
            if (__hisnan(y.x) || __hisnan(y.y)) {
              uint32_t *w = reinterpret_cast<uint32_t *>(&u);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                if ((w[k] & 0x7f80u) == 0x7f80u) w[k] &= 0xffff0000u;
                if ((w[k] & 0x7f800000u) == 0x7f800000u) w[k] &= 0xffffu;
              }
              base[x] = u;
              *reinterpret_cast<volatile int *>(&sm.any_bad) = 1;
            }
          }
        }
        fence_async_smem();
      }
      warp_arrive(&sm.looked[ring.stage]);
      if (!__all_sync(0xffffffffu, ok)) return;  // off the products' path
      ring.step();
    }
  }
}

// Two tiles of 128 rows share every key and value tile. While the softmax of
// one tile runs, the tensor cores have the other's products: S_w = Q_w K^T into
// TMEM, the weights back into TMEM in the place of the scores (bf16, the A
// operand of the second product), O_w += P_w V in TMEM throughout. Keys and
// values come by TMA, one box per page piece, into the layout the products
// read. The weights' rounding to bf16 (each off by up to 2^-8 of itself; their sums
// stay in fp32, unrounded) adds to the output's: 2.3e-3 of its size against 64 bits,
// 1.7e-3 if only the output were rounded; weights of 16 more bits would take the
// second product twice, in the pipe that binds. Four chunks of 1025 to 2048 tokens
// behind 1000 to 6144 (32/8 heads of 128, 0.52 TFLOP as the mean of two sets of
// lengths): 391 us, 1.34 PFLOP/s, the tensor pipe 60 % active. Bound by shared
// memory's reads (a product Q K^T of 64 cycles reads 8 KB at 128 bytes a cycle,
// beside TMA's writes) and by the step's chain: products, scores out of TMEM,
// maximum, exponentials, weights into TMEM.
template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    attend_many_kernel(Args a, const __grid_constant__ Maps maps) {
  extern __shared__ uint8_t raw[];
  Smem<D> &sm = *reinterpret_cast<Smem<D> *>(tck::align1k(raw));
  const int tid = threadIdx.x, warp = tid >> 5;
  const int cta = blockIdx.x, ctas = gridDim.x;
  clear_notes(a, cta);
  if (a.rows_over < 0) {
    clear_spare_rows<__nv_bfloat16, D, kThreads>(a, cta, ctas);
    if (cta == ctas - 1) report_requests(a);
  }
  if (tid == 0) {
    for (int x = 0; x < Smem<D>::kKeyStages; ++x) {
      mbar_init(&sm.k_full[x], 1);
      mbar_init(&sm.k_empty[x], 1);
    }
    for (int x = 0; x < Smem<D>::kValueStages; ++x) {
      mbar_init(&sm.v_full[x], 1);
      mbar_init(&sm.v_empty[x], 1);
      mbar_init(&sm.looked[x], 1);
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
  const Walk<M, BN> walk{find_share<kThreads>(a, M, cta, ctas, sm.scratch)};
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 8)
      produce<D, 0>(a, maps, sm, walk);
    else if (warp == 10)
      produce<D, 1>(a, maps, sm, walk);
    else if (warp == 9)
      issue<D>(a, sm, walk);
    else
      look_over<D>(a, sm, walk);
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    softmax<D, q8::kPlain>(a, sm, walk, cta);
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

template <int D>
pair_status run_many(Launch *l, const Maps &maps, cudaStream_t s) {
  Args &a = l->a;
  a.unit_cost = kManyCost;
  constexpr int smem = sizeof(Smem<D>) + 1024;
  static_assert(smem <= 232448, "shared memory of a CTA");
  PAIR_CUDA_TRY(cudaFuncSetAttribute(attend_many_kernel<D>,
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  const int ctas = useful_ctas(a, M, min(kMaxMany, sm_count()));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = a.rows_over >= 0 ? 1 : 0;  // behind the launch for few rows
  PAIR_BEGIN("attend_many", s);
  if (cudaLaunchKernelEx(&cfg, attend_many_kernel<D>, a, maps) != cudaSuccess) {
    cudaGetLastError();
    return PAIR_ERR_CUDA;
  }
  PAIR_LAUNCH_CHECK(s);
  l->M = M;
  l->ctas = ctas;
  return PAIR_OK;
}

}  // namespace

bool many_applies(const Args &a, int D) {
  Maps maps;
  return many_maps(a, D, 2, &maps);
}

pair_status launch_many(Launch *l, int D, cudaStream_t s) {
  Maps maps;
  if (!many_maps(l->a, D, 2, &maps)) return PAIR_ERR_CUDA;
  return D == 64 ? run_many<64>(l, maps, s) : run_many<128>(l, maps, s);
}

}  // namespace attend
}  // namespace pairk
