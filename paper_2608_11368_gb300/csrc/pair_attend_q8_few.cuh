// pair_attend_paged_q8 for chunks with few rows (single tokens, drafts), and in fp32 for
// all: one pass over the cached codes.
//
// The products are formed the other way round, S^T = K Q^T and O^T += V^T P^T, with
// mma.sync: the keys (then the head's columns) are the 16 rows of a product and the
// query rows its 8 columns, so four rows of a single token leave half of a product
// empty and not three quarters, and every code is made a number once for all rows of
// a warp. mma.sync rather than tcgen05: so few rows cannot fill a tile of 128.
//
// 32 x 16 requests of 1500 tokens as the median (2.1 GB of codes, prompts of 256 tokens
// shared by 16 of them counted once): 329 us by token, 325 by head in e4m3. That is HBM's
// rate: the shared prompts come from memory again for nearly every request, 2.36 GB. Whole
// numbers leave little room beside the copies: of 715 instructions for 32 keys and 8 rows
// 350 make codes into numbers. With five rows of four heads (16 x 16 requests of 512 to
// 4096 tokens, 1.0 GB) 288 us: 1050 instructions for 32 keys and 24 rows, in two warps a
// scheduler, which issue in 0.46 of the cycles; registers (254) admit no more.
//
// K: codes become fp16 (exact, five instructions for four whole numbers), against
// queries in fp16 that are scaled by a power of two per row: the row's largest entry is
// brought to [2^14, 2^15), so an entry keeps its 8 bits down to 2^-31 of the largest
// and is off by 2^-39 of it below.
// V: codes become bf16 (exact), against weights exp(s - max) 2^(b - 127) in bf16: they
// carry the value's scale and want the exponent range. Each weight is off by up to 2^-8
// of itself, independently, while their sum takes them unrounded in fp32.
//
// fp32 queries: the stored numbers are exact in either type all the same, so only the other
// operand is split. A query entry is two fp16 numbers (22 bits, down to 2^-39 of the
// row's largest), a weight three bf16 ones (24 bits): two products for one, and three. The
// tensor cores need not round to nearest; four products at most are summed there, and
// those sums by rounded additions.
#pragma once

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
// Work is cut between tiles of BN keys, of more than one request between every kCut of them:
// a token of one request over 700 keys takes 14.6 us, cut between every 128 keys 16.5; 128
// requests of up to 640 keys in fp32 20.7, cut between all tiles 24.8 (more units fall into
// pieces, which have to be joined), between every eight 25.8 (shares differ by more). The
// rule counts entries, idle ones too: a token over 700 keys beside 1 or 15 of them takes
// 16.5, as two to eight such requests do; the finer cut was not measured there.
constexpr int BN = 32, kCut = 4;
// Keys that a warp works on at once: 16 where slices of 32 would leave an SM four warps.
template <int D>
constexpr int kSlice = D == 256 ? 16 : 32;

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
// kValueUnit. (Whole numbers by two masks and a subtraction instead of a mask and a
// multiply-add: 416 us instead of 366 for five rows of four heads.)
template <int F>
constexpr float kValueUnit = F == kI8 ? 64.f : 1.f;
template <int F, int hi>
__device__ __forceinline__ uint32_t to_bf16(uint32_t x) {
  if constexpr (F == kI8) {
    const uint32_t y = hi ? x >> 8 : x;
    return bits(q8::whole_to_bf16((y & 0x00ff00ffu) ^ 0x00800080u));
  } else {
    // Exponent and significand at bf16's places are the number times 2^-120 (numbers
    // below e4m3's normal ones too: bf16's multiply takes them as they are). The two
    // codes that are no numbers come out as +-480.
    const uint32_t y = hi ? x >> 4 : x << 4, z = hi ? x : x << 8;
    return bits(__hmul2(bf2_of((y & 0x07f007f0u) | (z & 0x80008000u)),
                        bf2_of(0x7b807b80u)));  // 2^120
  }
}

// A warp's way along its share, and its segment after the one at hand: in shared memory,
// which lane 0 writes; registers are short.
template <int M>
struct Place {
  Walk<M, BN, kCut> walk;
  Segment next;
  bool more;
  __device__ __forceinline__ void step(const Args &a) {
    if ((threadIdx.x & 31) == 0) {
      more = walk.next(a, &next);
      if (a.heads < a.Hkv) next.h = next.h * kWarps + (threadIdx.x >> 5);
    }
    __syncwarp();
  }
};

__device__ __forceinline__ void load8(const __nv_bfloat16 *p, bool there, float (&v)[8]) {
  const uint4 u = there ? *reinterpret_cast<const uint4 *>(p) : make_uint4(0, 0, 0, 0);
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = __uint_as_float(w[k] << 16);
    v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load8(const float *p, bool there, float (&v)[8]) {
#pragma unroll
  for (int k = 0; k < 8; k += 4) {
    const float4 u = there ? *reinterpret_cast<const float4 *>(p + k) : make_float4(0, 0, 0, 0);
    v[k] = u.x, v[k + 1] = u.y, v[k + 2] = u.z, v[k + 3] = u.w;
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&v)[8]) {
  *reinterpret_cast<uint4 *>(p) = make_uint4(
      bits(__floats2bfloat162_rn(v[0], v[1])), bits(__floats2bfloat162_rn(v[2], v[3])),
      bits(__floats2bfloat162_rn(v[4], v[5])), bits(__floats2bfloat162_rn(v[6], v[7])));
}
__device__ __forceinline__ void store8(float *p, const float (&v)[8]) {
  reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// Shared memory of a warp whose units have up to M rows.
template <typename T, int D, int M>
struct Few {
  static constexpr int kStages = 2;
  static constexpr int kPart = kSlice<D> * D;     // bytes of a slice of keys or values
  static constexpr int kSteps = D / 16;        // steps of 16 columns in K Q^T
  static constexpr int kRing = 0;              // [kStages][keys, values]
  static constexpr int kPtr = kRing + kStages * 2 * kPart;  // [kSlice] addresses of both
  static constexpr int kQ = kPtr + kSlice<D> * 16;  // [M / 8][kSteps / 2][32 lanes] 16 bytes
  static constexpr int kRest = M * D * 2;  // from there to what fp32 queries have beyond fp16
  static constexpr int kFactor = kQ + M * D * (int)sizeof(T);  // [M] scales of the queries
  static constexpr int kPlace = kFactor + M * 4;  // a Place
  static constexpr int kWarpBytes = (kPlace + (int)sizeof(Place<M>) + 127) / 128 * 128;
  static constexpr int kBytes = kWarps * kWarpBytes;
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

// The copies of a slice's rows, whose addresses are at `ptrs`: all addresses are read before
// the first copy (no load passes a copy, which writes shared memory: one after the other, a
// copy waits for each load, 316 us instead of 288 for five rows of four heads), two at once.
template <int D, bool value>
__device__ __forceinline__ void bring(uint32_t to, uint32_t ptrs) {
  constexpr int P = D / 16, RP = 32 / P;  // pieces of a row, rows of one round of copies
  constexpr int B = kSlice<D> / RP;       // rows of a lane
  const int lane = threadIdx.x & 31, c = lane % P;
  const auto row = [&](int x) { return x / 2 * 2 * RP + lane / P * 2 + x % 2; };
  const uint8_t *p[B];
#pragma unroll
  for (int x = 0; x < B; x += 2)
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];"
                 : "=l"(p[x]), "=l"(p[x + 1])
                 : "r"(ptrs + row(x) * 8)
                 : "memory");
#pragma unroll
  for (int x = 0; x < B; ++x)
    cp_async16(to + place<D, value>(row(x), c), wide(p[x], c, 16), true);
}

// Where a warp's copies are: this lane's key of the next slice to be brought, and that
// key's way in the block table.
struct Stream {
  const int32_t *row;
  int32_t key, end, at, off, id;
  int32_t slices;    // of the segment
  uint32_t kb, vb;   // exponent bytes of the lane's key: of the slice at hand,
  uint32_t kb1, vb1;  // of the one behind it
};

// The slices of a segment, and the page of this lane's first key.
template <int D>
__device__ __forceinline__ void begin_stream(const Args &a, const Segment &s, Stream &m) {
  const int first = s.t0 * BN;
  m.row = a.table + (int64_t)s.i * a.width;
  m.end = min(s.keys, s.t1 * BN);
  m.slices = first < m.end ? (m.end - first + kSlice<D> - 1) / kSlice<D> : 0;
  m.key = first + (threadIdx.x & 31);
  m.at = m.key / a.page;
  m.off = m.key - m.at * a.page;
  m.id = m.key < m.end ? m.row[m.at] : 0;
}
template <int D>
__device__ __forceinline__ void look_ahead(const Args &a, Stream &m) {
  m.key += kSlice<D>;
  m.at += a.slice_pages;
  m.off += a.slice_rest;
  if (m.off >= a.page) {
    m.off -= a.page;
    ++m.at;
  }
  m.id = m.key < m.end ? m.row[m.at] : 0;
}
// Starts the copies of the keys that were looked up, into half `stage` of the ring, reads
// their exponents and keeps where their values lie. Keys that do not exist are the cache's
// first: they are masked.
template <typename T, int D, int M>
__device__ __forceinline__ void bring_keys(const Args &a, const Segment &s, Stream &m, int stage,
                                           uint32_t base) {
  using L = Few<T, D, M>;
  const int lane = threadIdx.x & 31;
  int pg = m.id, o = m.off;
  if (m.key >= m.end) pg = 0, o = 0;
  if ((unsigned)pg >= (unsigned)a.num_pages) {
    flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
    pg = 0;
  }
  const uint8_t *kp = static_cast<const uint8_t *>(a.kc) + s.h * a.ks.for_head;
  const uint8_t *vp = static_cast<const uint8_t *>(a.vc) + s.h * a.vs.for_head;
  const uint8_t *ke = a.ke + s.h * a.kes.for_head, *ve = a.ve + s.h * a.ves.for_head;
  if (a.narrow) {
    ke = wide(wide(ke, pg, a.kes.for_page), o, a.kes.for_token);
    ve = wide(wide(ve, pg, a.ves.for_page), o, a.ves.for_token);
    kp = wide(wide(kp, pg, a.ks.for_page), o, a.ks.for_token);
    vp = wide(wide(vp, pg, a.vs.for_page), o, a.vs.for_token);
  } else {
    ke += cache_row(a, a.kes, pg, o, 0);
    ve += cache_row(a, a.ves, pg, o, 0);
    kp += cache_row(a, a.ks, pg, o, 0);
    vp += cache_row(a, a.vs, pg, o, 0);
  }
  m.kb1 = __ldg(ke);
  m.vb1 = __ldg(ve);
  const uint32_t ptrs = base + L::kPtr;
  if (lane < kSlice<D>) {
    asm volatile("st.shared.b64 [%0], %1;" ::"r"(ptrs + lane * 8), "l"(kp) : "memory");
    asm volatile("st.shared.b64 [%0], %1;" ::"r"(ptrs + (kSlice<D> + lane) * 8), "l"(vp)
                 : "memory");
  }
  __syncwarp();
  bring<D, false>(base + L::kRing + stage * 2 * L::kPart, ptrs);
}

// The first two slices of a segment, on their way. Copies are in groups of their own, of
// keys and of values in turn: a slice's keys have been used when its values have not, and
// are followed by those of the next slice but one (whole slices, one ahead: 382 us instead
// of 358 for five rows of four heads).
template <typename T, int D, int M>
__device__ __forceinline__ void begin_copies(const Args &a, const Segment &s, Stream &m,
                                             uint32_t base) {
  using L = Few<T, D, M>;
  Stream n = m;  // of the second slice: both slices' pages are on their way
  if (m.slices > 1) look_ahead<D>(a, n);
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    if (x < m.slices) bring_keys<T, D, M>(a, s, x ? n : m, x, base);
    cp_async_commit();
    if (x < m.slices)
      bring<D, true>(base + L::kRing + (x * 2 + 1) * L::kPart, base + L::kPtr + kSlice<D> * 8);
    cp_async_commit();
    __syncwarp();
  }
  n.kb = m.kb1, n.vb = m.vb1;
  m = n;
  if (m.slices > 2) look_ahead<D>(a, m);
}

// A warp's segment of up to 8 NT rows. Its first slices are on their way; when it ends,
// those of the segment after it are (if there is one).
template <typename T, int D, int F, int M, int NT>
__device__ __forceinline__ void few_segment(const Args &a, const Segment &s, Stream &m,
                                            const Place<M> &place_of, uint8_t *smem, float *part) {
  using L = Few<T, D, M>;
  constexpr int MT = kSlice<D> / 16;
  constexpr int DT = D / 16;  // tiles of 16 columns in O^T
  constexpr bool f32 = sizeof(T) == 4;
  constexpr int NP = f32 ? 3 : 1;  // bf16 numbers to a weight
  const int lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const uint32_t base = smem_u32(smem);
  float *factor = reinterpret_cast<float *>(smem + L::kFactor);
  const int slices = m.slices, first = s.t0 * BN;
  __syncwarp();

  // Queries in fp16, in the order in which the products take them: step k of 16 columns
  // takes of lane (g, t) the columns 16 (t + 4 (k / 4)) + 4 (k % 4) + {0, 1, 2, 3} of
  // row g, the places of the four codes of a word.
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int r = j * 8 + g;
    float v[D / 32][8];
    uint32_t top = 0;
    const RowAt w = row_at(a, s.row0, s.r0, s.h, r < s.rows ? r : 0);
    const T *src = static_cast<const T *>(a.q) + w.token * a.q_row + w.head * a.q_head + 16 * t;
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      load8(src + 64 * (x >> 1) + 8 * (x & 1), r < s.rows, v[x]);
#pragma unroll
      for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[x][k]) & 0x7fffffffu);
    }
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // The scale that brings 2^E to 2^14, and its inverse. What is not finite stays so.
    const uint32_t e = min(max((int)(top >> 23) - 14, 1), 253);
    const float up = __uint_as_float((254 - e) << 23);
    if (t == 0) factor[r] = __uint_as_float(e << 23);
    uint8_t *dst = smem + L::kQ + (j * (L::kSteps / 2) * 32 + lane) * 16;
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      uint32_t h[4], rest[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float y0 = v[x][2 * k] * up, y1 = v[x][2 * k + 1] * up;
        const __half2 z = __floats2half2_rn(y0, y1);
        h[k] = bits(z);
        if (f32) rest[k] = bits(__floats2half2_rn(y0 - __low2float(z), y1 - __high2float(z)));
      }
      *reinterpret_cast<uint4 *>(dst + x * 512) = make_uint4(h[0], h[1], h[2], h[3]);
      if (f32)
        *reinterpret_cast<uint4 *>(dst + L::kRest + x * 512) =
            make_uint4(rest[0], rest[1], rest[2], rest[3]);
    }
  }
  __syncwarp();

  float o[DT][NT][4], mx[NT][2], l[NT][2], cs[NT][2];
  int seen[NT][2];
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = j * 8 + 2 * t + c;
      mx[j][c] = l[j][c] = 0.f;
      cs[j][c] = factor[r] * (a.scale * kLog2e);
      seen[j][c] = min(s.seen(r, a.g), s.kv);
    }
#pragma unroll
  for (int i = 0; i < DT; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[i][j][c] = 0.f;
  const uint32_t q_at = base + L::kQ + lane * 16;
  const int least = s.least;

#pragma unroll 1
  for (int x = 0; x < slices; ++x) {
    const float ke = q8::scale_of(m.kb), ve = q8::scale_of(m.vb);  // of this lane's key
    cp_async_wait<3>();  // this slice's keys are there
    __syncwarp();
    const uint32_t ks = base + L::kRing + (x & 1) * 2 * L::kPart, vs = ks + L::kPart;
    const int key0 = first + x * kSlice<D>;
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
          const uint32_t b_at = q_at + (j * (L::kSteps / 2) + 2 * y + p) * 512;
          const uint4 b = lds128(b_at);
          if constexpr (f32) {
            const uint4 b1 = lds128(b_at + L::kRest);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              float part_of[4] = {};  // sums of 32 columns, joined by rounded additions
              mma_f16(part_of, f[0][i], b1.x, b1.y);
              mma_f16(part_of, f[1][i], b1.z, b1.w);
              mma_f16(part_of, f[0][i], b.x, b.y);
              mma_f16(part_of, f[1][i], b.z, b.w);
#pragma unroll
              for (int c = 0; c < 4; ++c) sc[i][j][c] += part_of[c];
            }
          } else {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              mma_f16(sc[i][j], f[0][i], b.x, b.y);
              mma_f16(sc[i][j], f[1][i], b.z, b.w);
            }
          }
        }
      }
    }
    // sc[i][j][c]: key 16 i + g + 8 (c / 2), row 8 j + 2 t + c % 2. In log2 units, relative
    // to the row's reference, which is 0 at first. The powers of two of key and query meet
    // first: a large key under small queries, whose codes alone make products of up to
    // 2^32, would leave fp32's range with one of them.
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float k0 = __shfl_sync(0xffffffffu, ke, i * 16 + g);
      const float k1 = __shfl_sync(0xffffffffu, ke, i * 16 + 8 + g);
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 4; c += 2) {  // two rows at once
          const float k = c ? k1 : k0;
          const float2 y = fma2({sc[i][j][c], sc[i][j][c + 1]}, mul2({cs[j][0], cs[j][1]}, {k, k}),
                                {-mx[j][0], -mx[j][1]});
          sc[i][j][c] = y.x, sc[i][j][c + 1] = y.y;
        }
    }
    const bool edge = key0 + kSlice<D> > least;
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
          mx[j][c] += up;
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
    __syncwarp();  // nobody reads these keys any more
    m.kb = m.kb1, m.vb = m.vb1;
    if (x + 2 < slices) bring_keys<T, D, M>(a, s, m, x & 1, base);
    cp_async_commit();
    if (x + 3 < slices) look_ahead<D>(a, m);
    cp_async_wait<3>();  // this slice's values are there
    __syncwarp();
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const float v0 = __shfl_sync(0xffffffffu, ve, i * 16 + g);
      const float v1 = __shfl_sync(0xffffffffu, ve, i * 16 + 8 + g);
      float w[NT][4];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 4; c += 2) {
          const float2 e = {ex2_approx(sc[i][j][c]), ex2_approx(sc[i][j][c + 1])};
          const float v = c ? v1 : v0;
          const float2 sum = add2({l[j][0], l[j][1]}, e), y = mul2(e, {v, v});
          l[j][0] = sum.x, l[j][1] = sum.y;
          w[j][c] = y.x, w[j][c + 1] = y.y;
        }
      if (edge) {  // the scale of a value that a row does not see may be NaN
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (key0 + i * 16 + g + 8 * (c >> 1) >= seen[j][c & 1]) w[j][c] = 0.f;
      }
      uint32_t p[NT][NP][2];
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int y = 0; y < NP; ++y)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const __nv_bfloat162 z = __floats2bfloat162_rn(w[j][2 * h], w[j][2 * h + 1]);
            p[j][y][h] = transposed(bits(z));
            if (f32) w[j][2 * h] -= __low2float(z), w[j][2 * h + 1] -= __high2float(z);
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
            for (int j = 0; j < NT; ++j) {
              float(&to)[4] = o[(y * W + w) * 2 + h][j];
              if constexpr (f32) {
                float part_of[4] = {};
#pragma unroll
                for (int z = NP - 1; z >= 0; --z) mma_bf(part_of, f, p[j][z][0], p[j][z][1]);
#pragma unroll
                for (int c = 0; c < 4; ++c) to[c] += part_of[c];
              } else {
                mma_bf(to, f, p[j][0][0], p[j][0][1]);
              }
            }
          }
      }
    }
    __syncwarp();  // nor these values
    if (x + 2 < slices) bring<D, true>(vs, base + L::kPtr + kSlice<D> * 8);
    cp_async_commit();
  }
  // The next segment's first slices, then this one's sums: lane (g, t) has 16 columns (8
  // for heads of 64) of the rows 8 j + 2 t and the one behind.
  if (place_of.more) {
    begin_stream<D>(a, place_of.next, m);
    begin_copies<T, D, M>(a, place_of.next, m, base);
  }
#pragma unroll
  for (int j = 0; j < NT; ++j)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const int r = j * 8 + 2 * t + c;
#pragma unroll
      for (int w = 4; w < 32; w *= 2) l[j][c] += __shfl_xor_sync(0xffffffffu, l[j][c], w);
      if (r >= s.rows) continue;
      const float sum = l[j][c], top = sum == 0.f ? -INFINITY : mx[j][c];
      constexpr int C = D == 64 ? 8 : 16;  // columns side by side
      if (!part) {
        const RowAt w = row_at(a, s.row0, s.r0, s.h, r);
        const float inv = sum == 0.f ? 0.f : kValueUnit<F> / sum;
        T *to = static_cast<T *>(a.out) + (w.token * a.Hq + w.head) * D + C * g;
#pragma unroll
        for (int y = 0; y < DT / 4; ++y) {
          float v[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            v[2 * k] = o[y * 4 + k][j][c] * inv;
            v[2 * k + 1] = o[y * 4 + k][j][c + 2] * inv;
          }
          store8(to + (y >> 1) * 128 + (y & 1) * 8, v);
        }
        if (g == 0 && a.lse)
          a.lse[w.token * a.Hq + w.head] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * kLn2;
      } else {
        if (g == 0) {
          part[r] = top;
          part[M + r] = sum;
        }
        float *to = part + 2 * M + r * D + C * g;
#pragma unroll
        for (int y = 0; y < DT / 2; ++y)
          *reinterpret_cast<float4 *>(to + (y >> 2) * 128 + (y & 3) * 4) = make_float4(
              o[y * 2][j][c] * kValueUnit<F>, o[y * 2][j][c + 2] * kValueUnit<F>,
              o[y * 2 + 1][j][c] * kValueUnit<F>, o[y * 2 + 1][j][c + 2] * kValueUnit<F>);
      }
    }
}

// CTAs of an SM.
template <typename T, int D, int M>
constexpr int kPerSm = 2 * (Few<T, D, M>::kBytes + 1024) > 233472 ? 1
                       : M == 8 && D * sizeof(T) <= 256           ? 3
                                                                  : 2;

// A unit is worked on by one warp from end to end, a slice of keys at a time, but where
// shares meet. Nothing waits for another warp (four warps over one unit's keys, their sums
// joined at its end: 442 us instead of 391 for the skewed requests). Every warp has a share
// of the work of its own, or, where key heads come in fours, a CTA has one of four heads at
// once: its warps then read the same tokens, whose heads lie side by side in a cache by
// token (405 us -> 351). Three CTAs an SM for up to 8 rows of at most 256 bytes (two: 419),
// two for more, one for 16 rows of 1024 bytes. The form for 32 rows, which a call takes that
// does not know its longest chunk, serves single tokens too: the skewed requests 517 us
// instead of 328, 16 x 16 with drafts 442 instead of 290.
template <typename T, int D, int F, int M>
__global__ void __launch_bounds__(kThreads, kPerSm<T, D, M>) attend_q8_few_kernel(Args a) {
  using L = Few<T, D, M>;
  extern __shared__ __align__(128) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int worker = blockIdx.x * kWarps + warp;
  if (a.rows_upto < INT32_MAX) let_next_start();  // the kernel for many rows
  if (lane < 2) a.desc[worker * 2 + lane] = {0, 0, 0, 0, 0, 0, 0, 0};
  int64_t *scratch = reinterpret_cast<int64_t *>(smem);
  const Share share =
      a.heads < a.Hkv
          ? find_share<kThreads>(a, M, blockIdx.x, gridDim.x, scratch, kMinWarp)
          : find_share<kThreads, kWarps>(a, M, worker, gridDim.x * kWarps, scratch, kMinWarp);
  __syncthreads();  // the scratch is the rings' place
  uint8_t *mine = smem + warp * L::kWarpBytes;
  Place<M> &p = *reinterpret_cast<Place<M> *>(mine + L::kPlace);
  if (lane == 0) p.walk = Walk<M, BN, kCut>(share);
  p.step(a);
  Stream m;
  m.kb = m.vb = m.kb1 = m.vb1 = 0;
  if (p.more) {
    begin_stream<D>(a, p.next, m);
    begin_copies<T, D, M>(a, p.next, m, smem_u32(mine));
  }
  clear_spare_rows<T, D, kThreads>(a, blockIdx.x, gridDim.x);
  if (blockIdx.x == gridDim.x - 1) report_requests(a);
  for (int seg = 0; p.more; ++seg) {
    const Segment s = p.next;
    __syncwarp();
    p.step(a);
    float *part = nullptr;
    if (!s.whole()) {
      const int64_t slot = worker * 2 + (seg ? 1 : 0);
      if (lane == 0) a.desc[slot] = {s.i, s.h, s.rt, s.t0, s.t1, s.tiles, s.row0, s.rows};
      part = a.part + slot * part_floats(M, D);
    }
    if (M == 8 || s.rows <= 8)
      few_segment<T, D, F, M, 1>(a, s, m, p, mine, part);
    else if (M == 16 || (M == 32 && s.rows <= 16))
      few_segment<T, D, F, M, M < 16 ? 1 : 2>(a, s, m, p, mine, part);
    else if (M == 24 || s.rows <= 24)
      few_segment<T, D, F, M, M < 24 ? 1 : 3>(a, s, m, p, mine, part);
    else
      few_segment<T, D, F, M, M < 32 ? 1 : 4>(a, s, m, p, mine, part);
    __syncwarp();  // all lanes have seen `more`
  }
  let_next_start();
}

template <typename T, int D, int F, int M>
pair_status run_few(Launch *l, int slots, cudaStream_t s) {
  Args &a = l->a;
  constexpr int smem = Few<T, D, M>::kBytes;
  static_assert(kPerSm<T, D, M> * (smem + 1024) <= 233472, "shared memory of an SM");
  const auto kernel = attend_q8_few_kernel<T, D, F, M>;
  PAIR_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  a.unit_cost = 96;  // 8 x 8 requests, a token each: 40.4 us, with 48 or 160 41.1
  a.slice_pages = kSlice<D> / a.page;
  a.slice_rest = kSlice<D> % a.page;
  a.narrow = true;
  for (const pair_cache_strides *x : {&a.ks, &a.vs, &a.kes, &a.ves})
    a.narrow &= (uint64_t)x->for_page <= UINT32_MAX && (uint64_t)x->for_token <= UINT32_MAX;
  const int fit = min(slots * (kFewTile / M) / 2,  // two partial sums each
                      min(kMaxWorkers, kPerSm<T, D, M> * kWarps * sm_count()));
  // Where key heads come in fours a CTA's warps take four of them over the same keys.
  const bool together = a.Hkv % kWarps == 0;
  if (together) a.heads = a.Hkv / kWarps;
  const int ctas = together
                       ? useful_ctas(a, M, fit / kWarps, kMinWarp)
                       : (int)ceil_div(useful_ctas(a, M, fit / kWarps * kWarps, kMinWarp), kWarps);
  PAIR_BEGIN("attend_q8_few", s);
  kernel<<<ctas, kThreads, smem, s>>>(a);
  PAIR_LAUNCH_CHECK(s);
  l->M = M;
  l->ctas = ctas * kWarps;
  return PAIR_OK;
}

template <typename T, int D, int F>
pair_status run_few(Launch *l, int64_t most_rows, int slots, cudaStream_t s) {
  if constexpr (D < 256 || sizeof(T) == 4)
    if (most_rows <= 8) return run_few<T, D, F, 8>(l, slots, s);
  if constexpr (D < 256 && sizeof(T) == 2) {
    if (most_rows > 24) return run_few<T, D, F, 32>(l, slots, s);
    if (most_rows > 16) return run_few<T, D, F, 24>(l, slots, s);
  }
  return run_few<T, D, F, 16>(l, slots, s);
}

template <typename T, int F>
pair_status run_few(Launch *l, int D, int64_t most_rows, int slots, cudaStream_t s) {
  if (D == 64) return run_few<T, 64, F>(l, most_rows, slots, s);
  if (D == 128) return run_few<T, 128, F>(l, most_rows, slots, s);
  return run_few<T, 256, F>(l, most_rows, slots, s);
}

}  // namespace
}  // namespace attend
}  // namespace pairk
