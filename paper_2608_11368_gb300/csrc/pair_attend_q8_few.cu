// pair_attend_paged_q8 for chunks with few rows (single tokens, drafts), bf16 queries:
// one pass over the cached codes, bound by HBM.
//
// The products are formed the other way round, S^T = K Q^T and O^T += V^T P^T, with
// mma.sync: the keys (then the head's columns) are the 16 rows of a product and the
// query rows its 8 columns, so four rows of a single token leave half of a product
// empty and not three quarters, and every code is made a number once for all rows of
// a warp. With numbers of 8 bits that conversion is what the issue slots go to.
//
// K: codes become fp16 (exact, five instructions for four whole numbers), against
// queries in fp16 that are scaled by a power of two per row: the row's largest entry is
// brought to [2^14, 2^15), so an entry keeps its 8 bits down to 2^-31 of the largest
// and is off by 2^-39 of it below.
// V: codes become bf16 (exact), against weights exp(s - max) 2^(b - 127) in bf16: they
// carry the value's scale and want the exponent range. Each weight is off by up to 2^-8
// of itself, independently, while their sum takes them unrounded in fp32.
#include <cuda_fp16.h>

#include "pair_attend.cuh"
#include "pair_cache_q8.cuh"

namespace pairk {
namespace attend {
namespace {

using namespace tc;
using q8::kE4M3;
using q8::kI8;

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;
constexpr int BN = 128;           // keys of a tile: 32 for each warp
constexpr int kSlice = 32;        // keys that a warp works on at once

__device__ __forceinline__ uint32_t bits(__nv_bfloat162 x) {
  return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ uint32_t bits(__half2 x) {
  return *reinterpret_cast<const uint32_t *>(&x);
}
__device__ __forceinline__ __half2 half2_of(uint32_t x) {
  return *reinterpret_cast<const __half2 *>(&x);
}
__device__ __forceinline__ __nv_bfloat162 bf2_of(uint32_t x) {
  return *reinterpret_cast<const __nv_bfloat162 *>(&x);
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                        uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf(float (&d)[4], const uint32_t (&a)[4], uint32_t b0,
                                       uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit numbers, a row per four lanes, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
  uint4 u;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w)
               : "r"(at)
               : "memory");
  return u;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
  uint2 u;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(u.x), "=r"(u.y) : "r"(at) : "memory");
  return u;
}

// p + x * stride, in one instruction: a stride that fits in 32 bits.
__device__ __forceinline__ const uint8_t *wide(const uint8_t *p, int x, int64_t stride) {
  const uint8_t *q;
  asm("mad.wide.u32 %0, %1, %2, %3;" : "=l"(q) : "r"(x), "r"((uint32_t)stride), "l"(p));
  return q;
}

// The codes of a word in fp16: bytes 0, 1 and bytes 2, 3.
template <int F>
__device__ __forceinline__ void to_half(uint32_t w, uint32_t &lo, uint32_t &hi) {
  if constexpr (F == kI8) {
    w ^= 0x80808080u;  // code + 128; under 0x64 the bits of 1024 + that
    const __half2 off = __half2half2(__ushort_as_half(0x6480));  // 1152
    lo = bits(__hsub2(half2_of(__byte_perm(w, 0x64646464u, 0x4140)), off));
    hi = bits(__hsub2(half2_of(__byte_perm(w, 0x64646464u, 0x4342)), off));
  } else {
    lo = bits(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)w, __NV_E4M3)));
    hi = bits(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3)));
  }
}

// The codes in the low (hi = 0) or the high bytes of both halves of x in bf16, over
// kValueUnit.
template <int F>
constexpr float kValueUnit = F == kI8 ? 64.f : 1.f;
template <int F, int hi>
__device__ __forceinline__ uint32_t to_bf16(uint32_t x) {
  if constexpr (F == kI8) {
    // A byte u = code + 128 is as a bf16 number u 2^-133: below 128 a subnormal one, from
    // there on one of the least exponent, in the same steps. Times 2^127, less 2.
    const uint32_t y = hi ? x >> 8 : x;
    return bits(__hfma2(bf2_of((y & 0x00ff00ffu) ^ 0x00800080u), bf2_of(0x7f007f00u),
                        bf2_of(0xc000c000u)));
  } else {
    // Exponent and significand at bf16's places are the number times 2^-120 (numbers
    // below e4m3's normal ones too: bf16's multiply takes them as they are). The two
    // codes that are no numbers come out as +-480.
    const uint32_t y = hi ? x >> 4 : x << 4, z = hi ? x : x << 8;
    return bits(__hmul2(bf2_of((y & 0x07f007f0u) | (z & 0x80008000u)),
                        bf2_of(0x7b807b80u)));  // 2^120
  }
}

// Shared memory of a CTA whose units have up to M rows.
template <int D, int M>
struct Few {
  static constexpr int kStages = 2;
  static constexpr int kPart = kSlice * D;         // bytes of a slice of keys or values
  static constexpr int kPieces = D / 16;           // 16-byte pieces of a row
  static constexpr int kSteps = D / 16;            // steps of 16 columns in K Q^T
  static constexpr int kPtr = 0;                   // addresses: [kWarps][2][kSlice]
  static constexpr int kFactor = kPtr + kWarps * 2 * kSlice * 8;  // [M] scales of the queries
  static constexpr int kQ = kFactor + M * 4;       // [M / 8][kSteps / 2][32 lanes] 16 bytes
  static constexpr int kRing = kQ + M * D * 2;     // [kWarps][kStages] slices
  static constexpr int kLine = D + 4;              // floats of a row of the warps' sums, which
  static constexpr int kMl = kRing + kWarps * M * kLine * 4;  // take the ring's place: sums,
  static constexpr int kSums = kMl + kWarps * M * 8;          // statistics
  static constexpr int kEnd = kRing + kWarps * kStages * 2 * kPart;
  static constexpr int kBytes = kEnd > kSums ? kEnd : kSums;
};

// Where a 16-byte piece of a row lies in a slice, so that the reads below find all
// banks: of keys, lanes (g, t) read row g, piece t (+ 4 j); of values rows 2 t + c, piece g
// (or half a piece).
template <int D, bool value>
__device__ __forceinline__ uint32_t place(int row, int piece) {
  if constexpr (D == 64) {
    if constexpr (!value) return row * 64 + piece * 16;
    return (row >> 1) * 128 + ((row ^ (row >> 1)) & 1) * 64 + (piece ^ ((row >> 1) & 2)) * 16;
  } else {
    return row * D + (piece ^ (value ? row & 6 : (row & 1) << 2)) * 16;
  }
}

// A segment whose tile has at most 8 NT rows in use. Warp w has the slices w, w + 4, .. of
// 32 keys. The warps share nothing while they work: each brings its own slices into a
// ring of its own, by 16-byte asynchronous copies, and waits for nobody.
template <int D, int F, int M, int NT>
__device__ __forceinline__ void few_segment(const Args &a, const Segment &s, uint8_t *smem,
                                            int cta, int seg) {
  using L = Few<D, M>;
  constexpr int NST = L::kStages, MT = kSlice / 16;
  constexpr int DT = D / 16;  // tiles of 16 columns in O^T
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int g = lane >> 2, t = lane & 3;
  float *factor = reinterpret_cast<float *>(smem + L::kFactor);
  const uint32_t ring = smem_u32(smem + L::kRing) + warp * NST * 2 * L::kPart;
  const uint32_t ptrs = smem_u32(smem + L::kPtr) + warp * 2 * kSlice * 8;
  const uint8_t *kc0 = static_cast<const uint8_t *>(a.kc) + s.h * a.ks.for_head;
  const uint8_t *vc0 = static_cast<const uint8_t *>(a.vc) + s.h * a.vs.for_head;
  const uint8_t *ke0 = a.ke + s.h * a.kes.for_head, *ve0 = a.ve + s.h * a.ves.for_head;

  // This lane's key of a slice, and its way in the table.
  const int end = min(s.keys, s.t1 * BN), first = s.t0 * BN + warp * kSlice;
  const int slices = first < end ? (end - first + BN - 1) / BN : 0;
  int key = first + lane, at = key / a.page, off = key - at * a.page;
  const int by = BN / a.page, by_off = BN - by * a.page;
  const int32_t *row = a.table + (int64_t)s.i * a.width;
  int id = key < end ? row[at] : 0;
  auto look_ahead = [&] {
    key += BN;
    at += by;
    off += by_off;
    if (off >= a.page) {
      off -= a.page;
      ++at;
    }
    id = key < end ? row[at] : 0;
  };
  // Starts the copies of the slice that was looked up, and reads its exponents. Keys
  // that do not exist are the cache's first: they are masked.
  uint32_t kb = 0, vb = 0;
  auto fetch = [&](int stage) {
    int pg = id, o = off;
    if (key >= end) pg = 0, o = 0;
    if ((unsigned)pg >= (unsigned)a.num_pages) {
      flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
      pg = 0;
    }
    const uint8_t *kp, *vp;
    if (a.narrow) {
      kb = __ldg(wide(wide(ke0, pg, a.kes.for_page), o, a.kes.for_token));
      vb = __ldg(wide(wide(ve0, pg, a.ves.for_page), o, a.ves.for_token));
      kp = wide(wide(kc0, pg, a.ks.for_page), o, a.ks.for_token);
      vp = wide(wide(vc0, pg, a.vs.for_page), o, a.vs.for_token);
    } else {
      kb = __ldg(ke0 + cache_row(a, a.kes, pg, o, 0));
      vb = __ldg(ve0 + cache_row(a, a.ves, pg, o, 0));
      kp = kc0 + cache_row(a, a.ks, pg, o, 0);
      vp = vc0 + cache_row(a, a.vs, pg, o, 0);
    }
    asm volatile("st.shared.v2.b64 [%0], {%1, %2};" ::"r"(ptrs + lane * 16), "l"(kp), "l"(vp)
                 : "memory");
    __syncwarp();
    constexpr int P = L::kPieces, RP = 32 / P;  // rows of one round of copies
    const int c = lane % P;
    const uint32_t kd = ring + stage * 2 * L::kPart, vd = kd + L::kPart;
#pragma unroll
    for (int x = 0; x < kSlice / RP; ++x) {
      const int r = x * RP + lane / P;
      asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];"
                   : "=l"(kp), "=l"(vp)
                   : "r"(ptrs + r * 16)
                   : "memory");
      cp_async16(kd + place<D, false>(r, c), wide(kp, c, 16), true);
      cp_async16(vd + place<D, true>(r, c), wide(vp, c, 16), true);
    }
  };
  __syncthreads();  // the segment before is through
  if (slices > 0) fetch(0);
  cp_async_commit();
  if (slices > 1) look_ahead();

  // Queries in fp16, in the order in which the products take them: step k of 16 columns
  // takes of lane (g, t) the columns 16 (t + 4 (k / 4)) + 4 (k % 4) + {0, 1, 2, 3} of
  // row g, the places of the four codes of a word.
  for (int j = warp; j < NT; j += kWarps) {
    const __nv_bfloat16 *q = static_cast<const __nv_bfloat16 *>(a.q);
    const int r = j * 8 + g;
    uint4 u[D / 32];
    uint32_t top = 0;
    const RowAt w = row_at(a, s.row0, s.r0, s.h, r < s.rows ? r : 0);
    const __nv_bfloat16 *src = q + w.token * a.q_row + w.head * a.q_head + 16 * t;
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      u[x] = r < s.rows ? *reinterpret_cast<const uint4 *>(src + 64 * (x >> 1) + 8 * (x & 1))
                        : make_uint4(0, 0, 0, 0);
      for (const uint32_t y : {u[x].x, u[x].y, u[x].z, u[x].w})
        top = max(top, max(y & 0x7fff0000u, (y & 0x7fffu) << 16));
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // The scale that brings 2^E to 2^14, and its inverse. What is not finite stays so.
    const uint32_t e = min(max((int)(top >> 23) - 14, 1), 253);
    const float up = __uint_as_float((254 - e) << 23);
    if (t == 0) factor[r] = __uint_as_float(e << 23);
    uint4 *dst = reinterpret_cast<uint4 *>(smem + L::kQ) + j * (L::kSteps / 2) * 32 + lane;
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      const uint32_t y[4] = {u[x].x, u[x].y, u[x].z, u[x].w};
      uint32_t h[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        h[k] = bits(__floats2half2_rn(__uint_as_float(y[k] << 16) * up,
                                      __uint_as_float(y[k] & 0xffff0000u) * up));
      dst[x * 32] = make_uint4(h[0], h[1], h[2], h[3]);
    }
  }
  __syncthreads();

  float o[DT][NT][4], m[NT][2], l[NT][2], cs[NT][2];
  int seen[NT][2];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = j * 8 + 2 * t + c;
      m[j][c] = l[j][c] = 0.f;
      cs[j][c] = factor[r] * (a.scale * kLog2e);
      seen[j][c] = min(s.seen(r, a.g), s.kv);
    }
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[i][j][c] = 0.f;
  const uint32_t q_at = smem_u32(smem + L::kQ) + lane * 16;
  const int least = s.least;

#pragma unroll 1
  for (int x = 0; x < slices; ++x) {
    const float ke = q8::scale_of(kb), ve = q8::scale_of(vb);  // of this lane's key
    cp_async_wait<0>();
    __syncwarp();
    const uint32_t ks = ring + (x % NST) * 2 * L::kPart, vs = ks + L::kPart;
    const int key0 = first + x * BN;
    if (x + 1 < slices) fetch((x + 1) % NST);
    cp_async_commit();
    if (x + 2 < slices) look_ahead();
    // Scores of 32 keys with 8 NT rows.
    float sc[MT][NT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) sc[i][j][c] = 0.f;
#pragma unroll
    for (int y = 0; y < D / 64; ++y) {
      uint4 u[MT][2];
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          u[i][h] = lds128(ks + place<D, false>(i * 16 + h * 8 + g, t + 4 * y));
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        uint32_t f[2][MT][4];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            to_half<F>(p ? u[i][h].z : u[i][h].x, f[0][i][h], f[0][i][h + 2]);
            to_half<F>(p ? u[i][h].w : u[i][h].y, f[1][i][h], f[1][i][h + 2]);
          }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const uint4 b = lds128(q_at + (j * (L::kSteps / 2) + 2 * y + p) * 512);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            mma_f16(sc[i][j], f[0][i], b.x, b.y);
            mma_f16(sc[i][j], f[1][i], b.z, b.w);
          }
        }
      }
    }
    // sc[i][j][c]: key 16 i + g + 8 (c / 2), row 8 j + 2 t + c % 2. In log2 units, relative
    // to the row's reference, which is 0 at first.
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float k0 = __shfl_sync(0xffffffffu, ke, i * 16 + g);
      const float k1 = __shfl_sync(0xffffffffu, ke, i * 16 + 8 + g);
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c)
          sc[i][j][c] = fmaf(sc[i][j][c] * (c < 2 ? k0 : k1), cs[j][c & 1], -m[j][c & 1]);
    }
    const bool edge = key0 + kSlice > least;
    if (edge) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (key0 + i * 16 + g + 8 * (c >> 1) >= seen[j][c & 1]) sc[i][j][c] = -INFINITY;
    }
    float over = sc[0][0][0];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) over = fmaxf(over, sc[i][j][c]);
    // The reference is the first slice's maximum (a row that sees none of its keys sees
    // none behind it) and stays while no maximum has grown by more than 2^8 over it:
    // weights up to 256 are as good as weights up to 1.
    if (x == 0 || __any_sync(0xffffffffu, over > 8.f)) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float up = x == 0 ? -INFINITY : 0.f;
#pragma unroll
          for (int i = 0; i < MT; ++i) up = fmaxf(up, fmaxf(sc[i][j][c], sc[i][j][c + 2]));
#pragma unroll
          for (int w = 4; w < 32; w *= 2) up = fmaxf(up, __shfl_xor_sync(0xffffffffu, up, w));
          if (up == -INFINITY) up = 0.f;
          const float fix = x == 0 ? 0.f : ex2_approx(-up);
          m[j][c] += up;
          l[j][c] *= fix;
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            o[i][j][c] *= fix;
            o[i][j][c + 2] *= fix;
          }
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            sc[i][j][c] -= up;
            sc[i][j][c + 2] -= up;
          }
        }
    }
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float v0 = __shfl_sync(0xffffffffu, ve, i * 16 + g);
      const float v1 = __shfl_sync(0xffffffffu, ve, i * 16 + 8 + g);
      float w[NT][4];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float e = ex2_approx(sc[i][j][c]);
          l[j][c & 1] += e;
          w[j][c] = e * (c < 2 ? v0 : v1);
        }
      if (edge) {  // the scale of a value that a row does not see may be NaN
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (key0 + i * 16 + g + 8 * (c >> 1) >= seen[j][c & 1]) w[j][c] = 0.f;
      }
      uint32_t p[NT][2];
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        p[j][0] = transposed(bits(__floats2bfloat162_rn(w[j][0], w[j][1])));
        p[j][1] = transposed(bits(__floats2bfloat162_rn(w[j][2], w[j][3])));
      }
      // Values of the lane's keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9: 16 columns (8 for heads
      // of 64), two of a product's 16 at a time.
      constexpr int W = D == 64 ? 2 : 4;  // words
#pragma unroll
      for (int y = 0; y < (D == 256 ? 2 : 1); ++y) {
        uint32_t u[4][W];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int r = i * 16 + 2 * t + (k & 1) + 8 * (k >> 1);
          if constexpr (D == 64) {
            const uint2 z = lds64(vs + place<D, true>(r, g >> 1) + (g & 1) * 8);
            u[k][0] = z.x, u[k][1] = z.y;
          } else {
            const uint4 z = lds128(vs + place<D, true>(r, g + 8 * y));
            u[k][0] = z.x, u[k][1] = z.y, u[k][2] = z.z, u[k][3] = z.w;
          }
        }
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t sel = h ? 0x7632u : 0x5410u;
            const uint32_t z0 = __byte_perm(u[0][w], u[1][w], sel);
            const uint32_t z1 = __byte_perm(u[2][w], u[3][w], sel);
            const uint32_t f[4] = {to_bf16<F, 0>(z0), to_bf16<F, 1>(z0), to_bf16<F, 0>(z1),
                                   to_bf16<F, 1>(z1)};
#pragma unroll
            for (int j = 0; j < NT; ++j) mma_bf(o[(y * W + w) * 2 + h][j], f, p[j][0], p[j][1]);
          }
      }
    }
  }
  __syncthreads();  // nobody reads a ring any more
  // The warps' sums meet in shared memory: [warp][8 NT][kLine]. Column d is at d with
  // its bits 1 and 2 turned by its bits 5 and 6, so that the eight lanes of a row
  // find different banks.
  float *all = reinterpret_cast<float *>(smem + L::kRing);
  float2 *ml = reinterpret_cast<float2 *>(smem + L::kMl);
  constexpr int R = 8 * NT;
  const auto turned = [](int d) { return d ^ ((d >> 4) & 6); };
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = warp * R + j * 8 + 2 * t + c;
#pragma unroll
      for (int w = 4; w < 32; w *= 2) l[j][c] += __shfl_xor_sync(0xffffffffu, l[j][c], w);
      if (g == 0) ml[r] = make_float2(l[j][c] == 0.f ? -INFINITY : m[j][c], l[j][c]);
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int d = D == 64 ? 8 * g + 2 * i : 16 * (g + 8 * (i >> 3)) + 2 * (i & 7);
        *reinterpret_cast<float2 *>(all + r * L::kLine + turned(d)) =
            make_float2(o[i][j][c], o[i][j][c + 2]);
      }
    }
  __syncthreads();
  const bool whole = s.whole();
  float *part = whole ? nullptr : a.part + note_partial(a, s, cta, seg) * part_floats(M, D);
  for (int x = tid; x < s.rows * (D / 8); x += kThreads) {
    const int r = x / (D / 8), col = x % (D / 8) * 8;
    float mx = -INFINITY, sum = 0.f, v[8] = {};
#pragma unroll
    for (int k = 0; k < kWarps; ++k) mx = fmaxf(mx, ml[k * R + r].x);
    const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
    for (int k = 0; k < kWarps; ++k) {
      const float2 e = ml[k * R + r];
      const float w = ex2_approx(e.x - ref), f = kValueUnit<F> * w;
      sum = fmaf(e.y, w, sum);
#pragma unroll
      for (int c = 0; c < 8; c += 2) {
        const float2 y =
            *reinterpret_cast<const float2 *>(all + (k * R + r) * L::kLine + turned(col + c));
        v[c] = fmaf(y.x, f, v[c]);
        v[c + 1] = fmaf(y.y, f, v[c + 1]);
      }
    }
    if (whole) {
      const RowAt w = row_at(a, s.row0, s.r0, s.h, r);
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      uint4 u;
      u.x = bits(__floats2bfloat162_rn(v[0] * inv, v[1] * inv));
      u.y = bits(__floats2bfloat162_rn(v[2] * inv, v[3] * inv));
      u.z = bits(__floats2bfloat162_rn(v[4] * inv, v[5] * inv));
      u.w = bits(__floats2bfloat162_rn(v[6] * inv, v[7] * inv));
      *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(a.out) +
                                 (w.token * a.Hq + w.head) * D + col) = u;
      if (col == 0 && a.lse)
        a.lse[w.token * a.Hq + w.head] = sum == 0.f ? -INFINITY : (mx + log2f(sum)) * kLn2;
    } else {
      if (col == 0) {
        part[r] = mx;
        part[M + r] = sum;
      }
      float4 *dst = reinterpret_cast<float4 *>(part + 2 * M + r * D + col);
      dst[0] = make_float4(v[0], v[1], v[2], v[3]);
      dst[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
}

template <int D, int F, int M>
__global__ void __launch_bounds__(kThreads, M == 16 && D <= 128 ? 3 : D <= 128 ? 2 : 1)
    attend_q8_few_kernel(Args a) {
  extern __shared__ __align__(128) uint8_t smem[];
  const int cta = blockIdx.x, ctas = gridDim.x;
  if (a.rows_upto < INT32_MAX) let_next_start();  // the kernel for many rows
  clear_notes(a, cta);
  clear_spare_rows<__nv_bfloat16, D, kThreads>(a, cta, ctas);
  if (cta == ctas - 1) report_requests(a);
  Walk<M, BN> walk{find_share<kThreads>(a, M, cta, ctas, reinterpret_cast<int64_t *>(smem))};
  Segment s;
  for (int seg = 0; walk.next(a, &s); ++seg) {
    if (s.rows <= 8)
      few_segment<D, F, M, 1>(a, s, smem, cta, seg);
    else if (M == 16 || s.rows <= 16)
      few_segment<D, F, M, 2>(a, s, smem, cta, seg);
    else if (s.rows <= 24)
      few_segment<D, F, M, M / 8 < 3 ? 1 : 3>(a, s, smem, cta, seg);
    else
      few_segment<D, F, M, M / 8>(a, s, smem, cta, seg);
  }
  let_next_start();
}

template <int D, int F, int M>
pair_status run_few(Launch *l, cudaStream_t s) {
  Args &a = l->a;
  constexpr int smem = Few<D, M>::kBytes, per_sm = M == 16 && D <= 128 ? 3 : D <= 128 ? 2 : 1;
  static_assert(per_sm * (smem + 1024) <= 233472, "shared memory of an SM");
  static_assert(M <= kFewTile, "partial sums fit in the workspace");
  const auto kernel = attend_q8_few_kernel<D, F, M>;
  PAIR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  a.unit_cost = 192;
  a.narrow = true;
  for (const pair_cache_strides *x : {&a.ks, &a.vs, &a.kes, &a.ves})
    a.narrow &= (uint64_t)x->for_page <= UINT32_MAX && (uint64_t)x->for_token <= UINT32_MAX;
  const int ctas = useful_ctas(a, M, min(kMaxCtas, per_sm * sm_count()));
  PAIR_BEGIN("attend_q8_few", s);
  kernel<<<ctas, kThreads, smem, s>>>(a);
  PAIR_LAUNCH_CHECK(s);
  l->M = M;
  l->ctas = ctas;
  return PAIR_OK;
}

template <int F>
pair_status run_few(Launch *l, int D, int64_t most_rows, cudaStream_t s) {
  const bool small = most_rows <= 16;
  if (D == 64) return small ? run_few<64, F, 16>(l, s) : run_few<64, F, 32>(l, s);
  if (D == 128) return small ? run_few<128, F, 16>(l, s) : run_few<128, F, 32>(l, s);
  return run_few<256, F, 16>(l, s);
}

}  // namespace

pair_status launch_few_q8(Launch *l, int D, int fmt, int64_t most_rows, cudaStream_t s) {
  return fmt == kI8 ? run_few<kI8>(l, D, most_rows, s) : run_few<kE4M3>(l, D, most_rows, s);
}

}  // namespace attend
}  // namespace pairk
