// pair_cache_append_q8, pair_cache_read_q8: rows into a paged cache of 8-bit codes
// and back.
#include "pair_cache_q8.cuh"

namespace pairk {
namespace {

using namespace q8;

constexpr int kThreads = 128;

struct Held {  // a cache of codes and exponent bytes
  uint8_t *codes;
  pair_cache_strides at;
  uint8_t *exps;
  pair_cache_strides exps_at;
};

struct Rows {
  int64_t T;
  int32_t H, D;
  void *k, *v;  // read or written, by the call
  int64_t k_row, k_head, v_row, v_head;
  const int64_t *slots;
  int64_t n_slots;
  int32_t page;
  Held kc, vc;
  int32_t *dev_err;
};

// A token's page and place in it; false where it has none (reported if its slot is
// not -1).
__device__ __forceinline__ bool find_slot(const Rows &a, int64_t t, int64_t *pg, int64_t *off) {
  const int64_t slot = a.slots[t];
  if (slot < 0 || slot >= a.n_slots) {
    if (slot != -1 && (threadIdx.x & 31) == 0) flag_error(a.dev_err, PAIR_DEV_ERR_PAGES);
    return false;
  }
  *pg = a.n_slots <= INT32_MAX ? (uint32_t)slot / (uint32_t)a.page : slot / a.page;
  *off = slot - *pg * a.page;
  return true;
}

// 32 bytes of a row: eight fp32 entries or sixteen bf16 ones.
template <typename T>
struct Piece {
  static constexpr int n = 32 / sizeof(T);
  uint4 u[2];
  __device__ __forceinline__ void words(uint32_t (&w)[8]) const {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      w[4 * k] = u[k].x, w[4 * k + 1] = u[k].y, w[4 * k + 2] = u[k].z, w[4 * k + 3] = u[k].w;
  }
  // The bits of the largest |x|, as those of an fp32 number: infinities and NaN come
  // out above all others.
  __device__ __forceinline__ uint32_t top() const {
    uint32_t w[8], m = 0;
    words(w);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if constexpr (sizeof(T) == 4)
        m = max(m, w[k] & 0x7fffffffu);
      else
        m = max(m, max(w[k] & 0x7fff0000u, (w[k] & 0x7fffu) << 16));
    }
    return m;
  }
  // Its codes, four to a word.
  template <int F>
  __device__ __forceinline__ void codes(float inv, uint32_t (&c)[n / 4]) const {
    uint32_t w[8];
    words(w);
#pragma unroll
    for (int k = 0; k < n / 4; ++k) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4)
          x[e] = __uint_as_float(w[4 * k + e]);
        else
          x[e] = __uint_as_float(e & 1 ? w[2 * k + (e >> 1)] & 0xffff0000u
                                       : w[2 * k + (e >> 1)] << 16);
      }
      c[k] = encode4<F>(x, inv);
    }
  }
};

// Lanes of a row of D entries, a piece each: a power of two.
template <typename T>
int lanes_of(int D) {
  int L = 1;
  while (L * Piece<T>::n < D) L *= 2;
  return L;
}

// A warp stores a token: L lanes a head, 32 / L heads at once, two such rounds of keys and
// of values in flight. A row is read once; its largest entry is found among its lanes
// (log2 L exchanges), its codes are formed from registers. Bound by HBM: 8192 tokens of 8
// heads of 128 stored and read back 23 us, 100 MB by both; 16 bytes of a row per lane
// instead of 32, with a division per piece in the reading: 27.
template <typename T, int F>
__global__ void __launch_bounds__(kThreads) append_kernel(Rows a, int L) {
  constexpr int n = Piece<T>::n, kAhead = 2;
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (t >= a.T) return;
  int64_t pg, off;
  if (!find_slot(a, t, &pg, &off)) return;
  const int sub = lane & (L - 1), per = 32 / L, h_lane = lane / L;
  const bool there = sub * n < a.D;
  const T *src[2] = {static_cast<const T *>(a.k) + t * a.k_row + h_lane * a.k_head + sub * n,
                     static_cast<const T *>(a.v) + t * a.v_row + h_lane * a.v_head + sub * n};
  uint8_t *to[2], *exps[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const Held &held = c ? a.vc : a.kc;
    to[c] = held.codes + pg * held.at.for_page + off * held.at.for_token +
            h_lane * held.at.for_head + sub * n;
    exps[c] = held.exps + pg * held.exps_at.for_page + off * held.exps_at.for_token +
              h_lane * held.exps_at.for_head;
  }
  for (int h0 = 0; h0 < a.H; h0 += per * kAhead) {  // alike in all lanes
    Piece<T> x[kAhead][2];
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        x[y][c].u[0] = x[y][c].u[1] = make_uint4(0, 0, 0, 0);
        if (there && h0 + y * per + h_lane < a.H) {
          const uint4 *p = reinterpret_cast<const uint4 *>(src[c]);
          x[y][c].u[0] = __ldg(p);
          x[y][c].u[1] = __ldg(p + 1);
        }
        src[c] += per * (c ? a.v_head : a.k_head);
      }
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        uint32_t top = x[y][c].top();
        for (int w = L >> 1; w > 0; w >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, w));
        const uint32_t b = exponent_of<F>(top);
        if (h0 + y * per + h_lane < a.H) {
          uint32_t w[n / 4] = {};  // a row that is not finite has no codes
          if (b != 255) x[y][c].template codes<F>(__uint_as_float((254u - b) << 23), w);
          if (there) {
            if constexpr (n == 8)
              *reinterpret_cast<uint2 *>(to[c]) = make_uint2(w[0], w[1]);
            else
              *reinterpret_cast<uint4 *>(to[c]) = make_uint4(w[0], w[1], w[2], w[3]);
          }
          if (sub == 0) *exps[c] = (uint8_t)b;
        }
        to[c] += per * (c ? a.vc : a.kc).at.for_head;
        exps[c] += per * (c ? a.vc : a.kc).exps_at.for_head;
      }
  }
}

// The values of a piece's codes.
template <typename T, int F>
__device__ __forceinline__ void values(const uint32_t (&w)[8 / sizeof(T)], uint32_t b,
                                       uint32_t (&u)[8]) {
  if constexpr (F == kI8 && sizeof(T) == 2) {
    // Codes over 64 by one multiply-add for two (whole_to_bf16), times 2^(b - 121):
    // in two factors where that is beyond bf16.
    const bool beyond = b > 248 && b != 255;
    const uint32_t f = b == 255 ? 0x7fc0u : (beyond ? b - 64 + 6 : b + 6) << 7;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t x = w[k >> 1] ^ 0x80808080u;
      __nv_bfloat162 y = whole_to_bf16(__byte_perm(x, 0, k & 1 ? 0x4342 : 0x4140));
      if (beyond) y = __hmul2(y, as_bf16x2(0x5f805f80u));  // 2^64
      y = __hmul2(y, as_bf16x2(f * 0x10001u));
      u[k] = *reinterpret_cast<const uint32_t *>(&y);
    }
  } else {
    const float s = scale_of(b);
    float x[32 / sizeof(T)];
#pragma unroll
    for (int k = 0; k < 8 / (int)sizeof(T); ++k) {
      float z[4];
      decode4<F>(w[k], z);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * k + e] = z[e] * s;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if constexpr (sizeof(T) == 4) {
        u[k] = __float_as_uint(x[k]);
      } else {
        const __nv_bfloat162 y = __floats2bfloat162_rn(x[2 * k], x[2 * k + 1]);
        u[k] = *reinterpret_cast<const uint32_t *>(&y);
      }
    }
  }
}

// 32 bytes of a row.
template <typename T, bool whole>
__device__ __forceinline__ void put32(T *to, const uint32_t (&u)[8]) {
  if constexpr (whole) {  // a sector in one piece
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(u[0]),
                 "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7])
                 : "memory");
  } else {
    reinterpret_cast<uint4 *>(to)[0] = make_uint4(u[0], u[1], u[2], u[3]);
    reinterpret_cast<uint4 *>(to)[1] = make_uint4(u[4], u[5], u[6], u[7]);
  }
}

// A warp reads a token back, laid out as in append_kernel: 65,536 tokens of 8 heads of 128
// into bf16 64 us, 6.3 TB/s (whole numbers through fp32 instead of bf16: 72). bf16 holds
// every value exactly, unless it is below its normal numbers. whole: every row of the
// outputs begins at a multiple of 32 bytes.
template <typename T, int F, bool whole>
__global__ void __launch_bounds__(kThreads) read_kernel(Rows a, int L) {
  constexpr int n = Piece<T>::n, kAhead = 2;
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (t >= a.T) return;
  int64_t pg = 0, off = 0;
  const bool there = find_slot(a, t, &pg, &off);
  const int sub = lane & (L - 1), per = 32 / L, h_lane = lane / L;
  if (sub * n >= a.D) return;
  T *out[2] = {static_cast<T *>(a.k) + t * a.k_row + h_lane * a.k_head + sub * n,
               static_cast<T *>(a.v) + t * a.v_row + h_lane * a.v_head + sub * n};
  const uint8_t *from[2], *exps[2];
#pragma unroll
  for (int c = 0; c < 2; ++c) {
    const Held &held = c ? a.vc : a.kc;
    from[c] = held.codes + pg * held.at.for_page + off * held.at.for_token +
              h_lane * held.at.for_head + sub * n;
    exps[c] = held.exps + pg * held.exps_at.for_page + off * held.exps_at.for_token +
              h_lane * held.exps_at.for_head;
  }
  for (int h0 = h_lane; h0 < a.H; h0 += per * kAhead) {
    uint32_t u[kAhead][2][n / 4], b[kAhead][2];
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        b[y][c] = 127;
#pragma unroll
        for (int k = 0; k < n / 4; ++k) u[y][c][k] = 0;
        if (there && h0 + y * per < a.H) {
          b[y][c] = __ldg(exps[c]);
          if constexpr (n == 8) {
            const uint2 z = __ldg(reinterpret_cast<const uint2 *>(from[c]));
            u[y][c][0] = z.x, u[y][c][1] = z.y;
          } else {
            const uint4 z = __ldg(reinterpret_cast<const uint4 *>(from[c]));
            u[y][c][0] = z.x, u[y][c][1] = z.y, u[y][c][2] = z.z, u[y][c][3] = z.w;
          }
        }
        from[c] += per * (c ? a.vc : a.kc).at.for_head;
        exps[c] += per * (c ? a.vc : a.kc).exps_at.for_head;
      }
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        if (h0 + y * per < a.H) {
          uint32_t x[8];
          values<T, F>(u[y][c], b[y][c], x);
          put32<T, whole>(out[c], x);
        }
        out[c] += per * (c ? a.v_head : a.k_head);
      }
  }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// What both calls check; the arguments of their kernels.
pair_status rows_of(int64_t T, int32_t H, int32_t D, pair_dtype dt, const void *k, int64_t k_row,
                    int64_t k_head, const void *v, int64_t v_row, int64_t v_head,
                    const int64_t *slots, int32_t num_pages, int32_t page_size,
                    pair_cache_format fmt, const pair_cache_q8 &kc, const pair_cache_q8 &vc,
                    int32_t *dev_err, Rows *out) {
  if (T < 1 || T > INT32_MAX || H < 1 || D < 16 || D > 256 || D % 16 != 0 ||
      (dt != PAIR_F32 && dt != PAIR_BF16) || (fmt != PAIR_CACHE_I8 && fmt != PAIR_CACHE_E4M3) ||
      !k || !v || !slots || num_pages < 1 || page_size < 1 || !kc.codes || !kc.exps || !vc.codes ||
      !vc.exps || (int64_t)H * D > INT32_MAX)
    return PAIR_ERR_INVALID_ARG;
  const int per = dt == PAIR_BF16 ? 8 : 4;  // elements of 16 bytes
  // A stride over a single entry says nothing.
  const int64_t rows[][2] = {{k_row, T}, {v_row, T}, {k_head, H}, {v_head, H}};
  for (const auto &x : rows)
    if (x[1] > 1 && x[0] % per != 0) return PAIR_ERR_INVALID_ARG;
  for (const pair_cache_q8 *c : {&kc, &vc}) {
    const int64_t codes[][2] = {{c->codes_at.for_page, num_pages},
                                {c->codes_at.for_token, page_size}, {c->codes_at.for_head, H}};
    for (const auto &x : codes)
      if (x[1] > 1 && x[0] % 16 != 0) return PAIR_ERR_INVALID_ARG;
    if (!aligned16(c->codes)) return PAIR_ERR_INVALID_ARG;
  }
  if (!aligned16(k) || !aligned16(v)) return PAIR_ERR_INVALID_ARG;
  const auto held = [](const pair_cache_q8 &c) {
    return Held{static_cast<uint8_t *>(c.codes), c.codes_at, static_cast<uint8_t *>(c.exps),
                c.exps_at};
  };
  *out = {T,      H,      D,     const_cast<void *>(k), const_cast<void *>(v),
          k_row,  k_head, v_row, v_head,                slots,
          (int64_t)num_pages * page_size, page_size,    held(kc), held(vc), dev_err};
  return check_device();
}

template <typename T, int F>
pair_status append(const Rows &a, cudaStream_t s) {
  PAIR_BEGIN("cache_append_q8", s);
  append_kernel<T, F><<<(unsigned)ceil_div(a.T, kThreads / 32), kThreads, 0, s>>>(
      a, lanes_of<T>(a.D));
  PAIR_LAUNCH_CHECK(s);
  return PAIR_OK;
}

template <typename T, int F>
pair_status read(const Rows &a, cudaStream_t s) {
  bool whole = ((reinterpret_cast<uintptr_t>(a.k) | reinterpret_cast<uintptr_t>(a.v)) & 31) == 0;
  const int64_t strides[][2] = {{a.k_row, a.T}, {a.v_row, a.T}, {a.k_head, a.H}, {a.v_head, a.H}};
  for (const auto &x : strides) whole &= x[1] == 1 || x[0] * sizeof(T) % 32 == 0;
  PAIR_BEGIN("cache_read_q8", s);
  const unsigned blocks = (unsigned)ceil_div(a.T, kThreads / 32);
  if (whole)
    read_kernel<T, F, true><<<blocks, kThreads, 0, s>>>(a, lanes_of<T>(a.D));
  else
    read_kernel<T, F, false><<<blocks, kThreads, 0, s>>>(a, lanes_of<T>(a.D));
  PAIR_LAUNCH_CHECK(s);
  return PAIR_OK;
}

}  // namespace
}  // namespace pairk

using namespace pairk;

extern "C" {

pair_status pair_cache_append_q8(int64_t T, int32_t Hkv, int32_t D, pair_dtype dt, const void *k,
                                 int64_t k_row, int64_t k_head, const void *v, int64_t v_row,
                                 int64_t v_head, const int64_t *slots, int32_t num_pages,
                                 int32_t page_size, pair_cache_format fmt, pair_cache_q8 k_cache,
                                 pair_cache_q8 v_cache, int32_t *dev_err, pair_stream_t stream) {
  reset_launches();
  Rows a;
  const pair_status st = rows_of(T, Hkv, D, dt, k, k_row, k_head, v, v_row, v_head, slots,
                                 num_pages, page_size, fmt, k_cache, v_cache, dev_err, &a);
  if (st != PAIR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (fmt == PAIR_CACHE_I8)
    return dt == PAIR_BF16 ? append<__nv_bfloat16, q8::kI8>(a, s) : append<float, q8::kI8>(a, s);
  return dt == PAIR_BF16 ? append<__nv_bfloat16, q8::kE4M3>(a, s) : append<float, q8::kE4M3>(a, s);
}

pair_status pair_cache_read_q8(int64_t T, int32_t Hkv, int32_t D, const int64_t *slots,
                               int32_t num_pages, int32_t page_size, pair_cache_format fmt,
                               pair_cache_q8 k_cache, pair_cache_q8 v_cache, pair_dtype dt, void *k,
                               int64_t k_row, int64_t k_head, void *v, int64_t v_row,
                               int64_t v_head, int32_t *dev_err, pair_stream_t stream) {
  reset_launches();
  Rows a;
  const pair_status st = rows_of(T, Hkv, D, dt, k, k_row, k_head, v, v_row, v_head, slots,
                                 num_pages, page_size, fmt, k_cache, v_cache, dev_err, &a);
  if (st != PAIR_OK) return st;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (fmt == PAIR_CACHE_I8)
    return dt == PAIR_BF16 ? read<__nv_bfloat16, q8::kI8>(a, s) : read<float, q8::kI8>(a, s);
  return dt == PAIR_BF16 ? read<__nv_bfloat16, q8::kE4M3>(a, s) : read<float, q8::kE4M3>(a, s);
}

}  // extern "C"
