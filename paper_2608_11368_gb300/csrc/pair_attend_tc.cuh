// Attention over a paged cache for chunks with many rows, bf16: scores and output sums on
// the 5th-generation tensor cores. What its kernels share, whatever the cache holds: the
// issue of the products, the softmax, the epilogue.
#pragma once

#include "pair_attend.cuh"
#include "pair_cache_q8.cuh"
#include "tc_kernels.cuh"

namespace pairk {
namespace attend {
namespace {

using namespace tc;

// CTA: warps 0-3 and 4-7 the softmax of one tile of 128 rows each (a row per thread), warp
// 9 the MMA issuer, warps 8, 10 and 11 bring keys and values in. A row's 128 scores stay
// in registers: the third warpgroup gives up registers to the other two (208 x 256 + 80 x
// 128 of the 168 x 384 that the block is launched with).
constexpr int kThreads = 384;
constexpr int M = kManyRows;  // two tiles of 128
constexpr int BN = 128;       // keys of a tile

template <int D>
struct Tc {
  static constexpr int kAtoms = D / 64;            // 128 rows x 64 columns, 128-byte swizzle
  static constexpr uint32_t kAtom = 128 * 128;
  static constexpr uint32_t kTile = kAtoms * kAtom;
  static constexpr uint32_t kIdescS = idesc_bf16(128, 128, 0, 0);
  static constexpr uint32_t kIdescO = idesc_bf16(128, D, 0, 1);
};

struct Maps {
  CUtensorMap k, v;
  int8_t k_at[3], v_at[3];  // dimension (1 to 3) of page, token, head
  int box;                  // tokens of a box
};

__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *map, uint64_t *bar, int x,
                                            int y, int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}

// wait() by all lanes of a warp, which leave it together: a lane's poll can succeed
// before another's, and the TMEM instructions (.aligned) want whole warps.
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t phase, volatile int *abort,
                                          int32_t *dev_err) {
  const bool ok = wait(bar, phase, abort, dev_err);
  return __all_sync(0xffffffffu, ok);
}

// wait() with fewer registers: by the low word of the clock, on a barrier's and the abort
// flag's addresses in shared memory.
__device__ __forceinline__ bool wait_lean(uint32_t bar, uint32_t phase, uint32_t abort,
                                          int32_t *dev_err) {
  static_assert(kWaitCycles < (1ll << 32), "the limit in a word");
  uint32_t t0 = 0, first = 1;
  while (true) {
    uint32_t ok, gone;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(phase)
        : "memory");
    if (ok) return true;
    const uint32_t now = (uint32_t)clock();
    if (first) t0 = now, first = 0;
    asm volatile("ld.volatile.shared.b32 %0, [%1];" : "=r"(gone) : "r"(abort) : "memory");
    if (gone) return false;
    if (now - t0 > (uint32_t)kWaitCycles) {
      asm volatile("st.volatile.shared.b32 [%0], %1;" ::"r"(abort), "r"(1) : "memory");
      flag_error(dev_err, PAIR_DEV_ERR_TIMEOUT);
      return false;
    }
  }
}

// A warp's arrival, for what its lanes have done (and fenced) before.
__device__ __forceinline__ void warp_arrive(uint64_t *bar) {
  __syncwarp();
  if (elect_one()) mbar_arrive(bar);
}

__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc,
                                            uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
// tmem_ld32 without its wait, and the wait, which names the registers.
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, "
      "%30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]),
                 "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]),
                 "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]),
                 "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                 "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]),
                 "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_st_wait() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// 32 bytes, aligned so: a row's owner writes whole sectors.
__device__ __forceinline__ void store32(void *to, const uint32_t (&u)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(u[0]),
               "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
               : "memory");
}

// Place in a ring of tiles. A barrier's phase tells a waiter one round from the
// next only while it is in step: every waiter of a ring is its producer, its
// consumer or one that the consumer waits for in each tile.
template <int ST>
struct Ring {
  int stage = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step() {
    if (++stage == ST) {
      stage = 0;
      phase ^= 1;
    }
  }
};

// Tiles with keys that some row does not see: their scores are masked and their
// values looked over.
__device__ __forceinline__ bool edge_tile(const Segment &s, int t) {
  return (t + 1) * BN > s.least;
}

// Waits, each lane of the first `n` for a barrier and phase of its own: one poll
// of several costs a warp as much as one. `ok`: what the lane's waits since the
// last vote came to.
template <typename W>
__device__ __forceinline__ bool wait_lanes(W wait, int n, bool ok, uint64_t *bar, uint32_t phase) {
  if ((int)(threadIdx.x & 31) < n) ok &= wait(bar, phase);
  return __all_sync(0xffffffffu, ok);
}

// The warp votes on its waits once per step, in the first (a vote behind each of
// them: 20 us of 374 for the four chunks); until then all lanes go the same way, and
// products issued after a wait that gave up are of a call that has failed.
template <int D, typename S, typename W>
__device__ void issue(const Args &a, S &sm, W walk) {
  using C = Tc<D>;
  const auto wait = [&](uint64_t *bar, uint32_t phase) {
    if constexpr (S::kLean)
      return wait_lean(smem_u32(bar), phase, smem_u32(&sm.abort), a.dev_err);
    else
      return tc::wait(bar, phase, &sm.abort, a.dev_err);
  };
  const uint64_t dq = sdesc_sw128(smem_u32(sm.q[0]), 16, 1024);
  const uint64_t dk = sdesc_sw128(smem_u32(sm.k[0]), 16, 1024);
  const uint64_t dv = sdesc_sw128(smem_u32(sm.v[0]), C::kAtom, 1024);
  const uint32_t tmem = sm.tmem;
  Ring<S::kKeyStages> kr;
  Ring<S::kValueStages> vr;
  uint32_t q_ph = 0, p_ph = 0;  // a bit per tile
  bool ok = true;
  auto scores = [&](int w, int stage, bool last) {  // S_w = Q_w K^T
    if (elect_one()) {
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        const uint32_t in = (kk & 3) * 2;
        mma_bf16(tmem + w * 128, dq + (w * C::kTile + (kk >> 2) * C::kAtom) / 16 + in,
                 dk + (stage * C::kTile + (kk >> 2) * C::kAtom) / 16 + in, C::kIdescS, kk != 0);
      }
      mma_commit(&sm.s_full[w]);
      if (last) mma_commit(&sm.k_empty[stage]);
    }
    __syncwarp();
  };
  // O_w += P_w V, by halves of the tile's keys.
  auto sums = [&](int w, int stage, int half, bool first, bool last) {
    if (elect_one()) {
#pragma unroll
      for (int kk = 0; kk < BN / 32; ++kk) {
        const int at = half * (BN / 32) + kk;
        mma_bf16_ts(tmem + 256 + w * D, tmem + w * 128 + at * 8,
                    dv + stage * C::kTile / 16 + at * 128, C::kIdescO, !first || at != 0);
      }
      if (half) {
        mma_commit(&sm.pv_done[w]);
        if (last) mma_commit(&sm.v_empty[stage]);
      }
    }
    __syncwarp();
  };
  Segment s;
  while (ok && walk.next(a, &s)) {
    if (s.t0 == s.t1) continue;
    const int top = s.rows > 128;  // the last active tile
    ok &= wait(&sm.k_full[kr.stage], kr.phase);
    for (int w = 0; w <= top; ++w) {
      ok &= wait(&sm.q_full[w], q_ph >> w & 1);
      q_ph ^= 1 << w;
      tc_fence_after();
      scores(w, kr.stage, w == top);
    }
    kr.step();
    for (int t = s.t0; t < s.t1; ++t) {
      const bool more = t + 1 < s.t1;
      // Before the first products of a tile: weights, values, the next keys.
      const int lane = threadIdx.x & 31;
      uint64_t *bar = lane == 0   ? &sm.p_ready[0][0]
                      : lane == 1 ? &sm.looked[vr.stage]
                                  : &sm.k_full[kr.stage];
      const uint32_t phase = lane == 0 ? p_ph & 1 : lane == 1 ? vr.phase : kr.phase;
      if (!(ok = wait_lanes(wait, more ? 3 : 2, ok, bar, phase))) break;
#pragma unroll(S::kLean ? 1 : 2)
      for (int w = 0; w < 2; ++w) {
        if (w > top) break;
        if (w) ok &= wait(&sm.p_ready[w][0], p_ph >> w & 1);
        tc_fence_after();
        sums(w, vr.stage, 0, t == s.t0, false);
        ok &= wait(&sm.p_ready[w][1], p_ph >> w & 1);
        p_ph ^= 1 << w;
        tc_fence_after();
        sums(w, vr.stage, 1, false, w == top);
        // In the tensor pipe's order behind the sums, which read the weights in
        // the place of these scores.
        if (more) scores(w, kr.stage, w == top);
      }
      vr.step();
      if (more) kr.step();
    }
    ok = __all_sync(0xffffffffu, ok);
  }
  if (elect_one()) mma_commit(&sm.done);
  __syncwarp();
  volatile int never = 0;
  tc::wait(&sm.done, 0, &never, a.dev_err);
  __syncwarp();
}

// Tiles formed out of 8 bits hold the stored numbers over this.
constexpr float kHeldUnit = 256.f;

// add_not_finite for values in 8 bits: a row of them is NaN throughout, or finite.
__device__ __forceinline__ void add_not_finite_held(const Args &a, const Segment &s, int tile,
                                                    int r, float (&v)[8]) {
  const int most = min(s.seen(r, a.g), s.kv);
#pragma unroll 1
  for (int key = max(s.t0 * tile, s.least / tile * tile); key < min(most, s.t1 * tile); ++key) {
    int off;
    const int id = page_of(a, s.i, key, &off);
    if (a.ve[cache_row(a, a.ves, id, off, s.h)] == 255)
#pragma unroll
      for (int c = 0; c < 8; ++c) v[c] = NAN;
  }
}

// The lanes of a warp go through a segment together: TMEM is read and written by
// whole warps. A wait that gave up is therefore noticed at the segment's end; until
// then the warp goes on over scores of a call that has failed, its further waits
// returning at once. (A vote behind each tile's wait: 346 us instead of 342 for four
// chunks of 1025 to 2048 tokens.)
template <int D, int F, typename S>
__device__ void softmax(const Args &a, S &sm, Walk<M, BN> walk, int cta) {
  using C = Tc<D>;
  const int tid = threadIdx.x, w = tid >> 7, row = tid & 127, warp = tid >> 5;
  volatile int *abort = &sm.abort;
  const uint32_t lane_at = (uint32_t)((warp & 3) * 32) << 16;
  const uint32_t tS = sm.tmem + w * 128 + lane_at, tO = sm.tmem + 256 + w * D + lane_at;
  const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(a.q);
  // A negative scale goes into the queries' sign, a zero one makes them zero.
  const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
  constexpr float unit = F == q8::kPlain ? 1.f : kHeldUnit;
  const float scale = a.scale == 0.f ? 1.f : fabsf(a.scale) * kLog2e * unit;
  uint32_t s_ph = 0, pv_ph = 0;
  bool ok = true;
  const int r = w * 128 + row;
  // The warp's queries, in the K-major swizzled layout of the A operand: whole rows at a
  // time, D / 8 lanes to each.
  auto put_query = [&](const Segment &g) {
    if (g.t0 == g.t1 || (w == 1 && g.rows <= 128)) return;
    const bool there = r < g.rows && a.scale != 0.f;
    const RowAt at = row_at(a, g.row0, g.r0, g.h, r < g.rows ? r : 0);
    const uint64_t mine =
        there ? reinterpret_cast<uint64_t>(q + at.token * a.q_row + at.head * a.q_head) : 0;
    constexpr int per = D / 8, RP = 32 / per;  // lanes of a row, rows at once
    const int lane = tid & 31, c = lane % per;
    uint4 u[per];
#pragma unroll
    for (int x = 0; x < per; ++x) {
      const uint64_t src = __shfl_sync(0xffffffffu, mine, x * RP + lane / per);
      u[x] = src ? *(reinterpret_cast<const uint4 *>(src) + c) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int x = 0; x < per; ++x) {
      const int to = (row & ~31) + x * RP + lane / per;
      u[x].x ^= flip, u[x].y ^= flip, u[x].z ^= flip, u[x].w ^= flip;
      *reinterpret_cast<uint4 *>(sm.q[w] + (c >> 3) * C::kAtom + to * 128 +
                                 (((c & 7) ^ (to & 7)) << 4)) = u[x];
    }
    fence_async_smem();
    warp_arrive(&sm.q_full[w]);
  };
  Segment s, ahead;
  bool more = walk.next(a, &ahead);
  if (more) put_query(ahead);
  for (int seg = 0; ok && more; ++seg) {
    s = ahead;
    const bool active = w == 0 || s.rows > 128, mine = r < s.rows;
    float m = -INFINITY, l = 0.f;
    if (active && s.t0 < s.t1) {
      const int seen = min(s.seen(mine ? r : 0, a.g), s.kv);
      for (int t = s.t0; t < s.t1; ++t) {
        const bool edge = edge_tile(s, t);
        const int key0 = t * BN;
        wait(&sm.s_full[w], s_ph, abort, a.dev_err);
        __syncwarp();
        s_ph ^= 1;
        tc_fence_after();
        uint32_t x[4][32];
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld32_async(tS + c * 32, x[c]);
#pragma unroll
        for (int c = 0; c < 4; ++c) tmem_ld_wait(x[c]);
        if (edge) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const int upto = seen - key0 - c * 32;  // by selects: rows end at different keys
            if (__all_sync(0xffffffffu, upto >= 32)) continue;
#pragma unroll
            for (int k = 0; k < 32; ++k) x[c][k] = k >= upto ? 0xff800000u : x[c][k];  // -inf
          }
        }
        float mx4[4] = {m, m, m, m};
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int k = 0; k < 32; k += 2)
            mx4[(k >> 1) & 3] = fmaxf(mx4[(k >> 1) & 3], fmaxf(__uint_as_float(x[c][k]),
                                                               __uint_as_float(x[c][k + 1])));
        const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
        // The reference of the exponentials stays while no row's maximum has
        // grown by more than 2^8 over it: weights up to 256 are as good as
        // weights up to 1, and the sums need not be rescaled.
        if (t == s.t0) {
          m = mx;
        } else if (__any_sync(0xffffffffu, (mx - m) * scale > 8.f)) {
          const float fix = ex2_approx(mx == -INFINITY ? 0.f : (m - mx) * scale);
          m = mx;
          l *= fix;
          wait(&sm.pv_done[w], pv_ph ^ 1, abort, a.dev_err);
          __syncwarp();
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            float o[32];
            uint32_t u[32];
            tmem_ld32(tO + c * 32, o);
#pragma unroll
            for (int k = 0; k < 32; ++k) u[k] = __float_as_uint(o[k] * fix);
            tmem_st32(tO + c * 32, u);
          }
        }
        pv_ph ^= 1;
        const float ref = m == -INFINITY ? 0.f : -m * scale;
        float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
        const float2 scale2 = {scale, scale}, ref2 = {ref, ref};
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
          uint32_t p[32];
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int k = 0; k < 32; k += 2) {
              float2 y = fma2({__uint_as_float(x[c + e][k]), __uint_as_float(x[c + e][k + 1])},
                              scale2, ref2);
              y.x = ex2_approx(y.x);
              y.y = ex2_approx(y.y);
              sum[(k >> 1) & 1] = add2(sum[(k >> 1) & 1], y);
              const __nv_bfloat162 b = __floats2bfloat162_rn(y.x, y.y);
              p[e * 16 + (k >> 1)] = *reinterpret_cast<const uint32_t *>(&b);
            }
          tmem_st32(tS + c * 16, p);
          tmem_st_wait();
          tc_fence_before();
          warp_arrive(&sm.p_ready[w][c >> 1]);
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      }
      if (!(ok = !__any_sync(0xffffffffu, *abort))) break;
    }
    // All scores of this segment have been read, so its queries have: the next
    // segment's go in their place, and its first scores are formed while this
    // one's sums are brought out.
    more = walk.next(a, &ahead);
    if (more) put_query(ahead);
    if (active && s.t0 < s.t1) {
      if (!(ok = warp_wait(&sm.pv_done[w], pv_ph ^ 1, abort, a.dev_err))) break;
      tc_fence_after();
    }
    const bool whole = s.whole();
    float *part = nullptr;
    if (!whole) part = a.part + note_partial(a, s, cta, seg) * part_floats(M, D);
    if (!active) continue;
    const RowAt at = row_at(a, s.row0, s.r0, s.h, mine ? r : 0);
    const float inv = l == 0.f ? 0.f : unit / l;
    const float m2 = m == -INFINITY ? m : m * scale;
    const bool aligned32 = (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
    const bool bad = s.t0 < s.t1 && *reinterpret_cast<volatile int *>(&sm.any_bad) != 0;
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      float o[32];
      if (s.t0 < s.t1) {
        tmem_ld32(tO + c * 32, o);
      } else {
#pragma unroll
        for (int k = 0; k < 32; ++k) o[k] = 0.f;
      }
      if (mine && bad) {
#pragma unroll
        for (int k = 0; k < 32; k += 8) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = o[k + e];
          if constexpr (F == q8::kPlain)
            add_not_finite<D>(a, s, BN, r, c * 32 + k, v);
          else
            add_not_finite_held(a, s, BN, r, v);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[k + e] = v[e];
        }
      }
      if (mine && whole) {
        __nv_bfloat16 *to = static_cast<__nv_bfloat16 *>(a.out) + (at.token * a.Hq + at.head) * D +
                            c * 32;
#pragma unroll
        for (int k = 0; k < 32; k += 16) {
          uint32_t u[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const __nv_bfloat162 b =
                __floats2bfloat162_rn(o[k + 2 * e] * inv, o[k + 2 * e + 1] * inv);
            u[e] = *reinterpret_cast<const uint32_t *>(&b);
          }
          if (aligned32) {
            store32(to + k, u);
          } else {
            *reinterpret_cast<uint4 *>(to + k) = make_uint4(u[0], u[1], u[2], u[3]);
            *reinterpret_cast<uint4 *>(to + k + 8) = make_uint4(u[4], u[5], u[6], u[7]);
          }
        }
      } else if (mine) {
#pragma unroll
        for (int k = 0; k < 32; k += 8) {
          uint32_t u[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) u[e] = __float_as_uint(o[k + e] * unit);
          store32(part + 2 * M + r * D + c * 32 + k, u);
        }
      }
      __syncwarp();  // rows in use and others, before the warp's next TMEM load
    }
    tc_fence_before();
    if (mine && !whole) {
      part[r] = m2;
      part[M + r] = l;
    } else if (mine && a.lse) {
      a.lse[at.token * a.Hq + at.head] = l == 0.f ? -INFINITY : (m2 + log2f(l)) * kLn2;
    }
  }
}

// 4-D map of a cache of entries of `size` bytes (2: bf16, 1: codes), dimensions in the
// order of their strides: boxes of `box` tokens x 64 columns (codes: all of them) of one
// page and head. False where no such map exists.
inline bool cache_map(CUtensorMap *m, int8_t (&at)[3], const void *p, const Args &a, int D,
                      int size, int box, const pair_cache_strides &st) {
  const auto fn = tck::encode_fn();
  if (!fn) return false;
  const int64_t stride[3] = {st.for_page * size, st.for_token * size, st.for_head * size};
  const cuuint64_t sizes[3] = {(cuuint64_t)a.num_pages, (cuuint64_t)a.page, (cuuint64_t)a.Hkv};
  const cuuint32_t want[3] = {1, (cuuint32_t)box, 1};
  int order[3] = {0, 1, 2};
  for (int x = 0; x < 3; ++x)
    for (int y = 0; y < 2; ++y)
      if (stride[order[y + 1]] < stride[order[y]]) {
        const int z = order[y];
        order[y] = order[y + 1];
        order[y + 1] = z;
      }
  cuuint64_t dims[4] = {(cuuint64_t)D}, strides[3];
  cuuint32_t boxes[4] = {size == 2 ? 64u : (cuuint32_t)D}, ones[4] = {1, 1, 1, 1};
  for (int x = 0; x < 3; ++x) {
    const int64_t b = stride[order[x]];
    if (b < 16 || b >= ((int64_t)1 << 40)) return false;
    strides[x] = (cuuint64_t)b;
    dims[x + 1] = sizes[order[x]];
    boxes[x + 1] = want[order[x]];
    at[order[x]] = (int8_t)(x + 1);
  }
  return fn(m, size == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 4,
            const_cast<void *>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            size * D == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

inline bool many_maps(const Args &a, int D, int size, Maps *maps) {
  // A box is the largest power of two of tokens, up to a tile, that divides
  // the page; the swizzle's period is 8 rows.
  int box = BN;
  while (a.page % box != 0) box /= 2;
  if (D > 128 || box < 8) return false;
  maps->box = box;
  return cache_map(&maps->k, maps->k_at, a.kc, a, D, size, box, a.ks) &&
         cache_map(&maps->v, maps->v_at, a.vc, a, D, size, box, a.vs);
}

}  // namespace
}  // namespace attend
}  // namespace pairk
