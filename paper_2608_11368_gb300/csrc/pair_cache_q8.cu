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

// 16 bytes of a row: four fp32 entries or eight bf16 ones.
template <typename T>
struct Piece {
  static constexpr int n = 16 / sizeof(T);
  uint4 u;
  // The bits of the largest |x|, as those of an fp32 number: infinities and NaN come
  // out above all others.
  __device__ __forceinline__ uint32_t top() const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        m = max(m, w[k] & 0x7fffffffu);
      } else {
        m = max(m, max(w[k] & 0x7fff0000u, (w[k] & 0x7fffu) << 16));
      }
    }
    return m;
  }
  __device__ __forceinline__ void get(int from, float (&x)[4]) const {
    if constexpr (sizeof(T) == 4) {
      x[0] = __uint_as_float(u.x), x[1] = __uint_as_float(u.y);
      x[2] = __uint_as_float(u.z), x[3] = __uint_as_float(u.w);
    } else {
      const uint32_t a = from ? u.z : u.x, b = from ? u.w : u.y;
      x[0] = __uint_as_float(a << 16), x[1] = __uint_as_float(a & 0xffff0000u);
      x[2] = __uint_as_float(b << 16), x[3] = __uint_as_float(b & 0xffff0000u);
    }
  }
};

// A warp stores a token: L lanes a head, 32 / L heads at once, NP pieces of 16 bytes a
// lane, kAhead rounds of heads in flight. A row is read once; its largest entry is
// found among its lanes (log2 L exchanges), its codes are formed from registers.
// Bound by HBM: every entry is read once, every code written once.
template <typename T, int F, int NP>
__global__ void __launch_bounds__(kThreads) append_kernel(Rows a, int L) {
  constexpr int n = Piece<T>::n, kAhead = 4 / NP;
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (t >= a.T) return;
  int64_t pg, off;
  if (!find_slot(a, t, &pg, &off)) return;
  const int sub = lane & (L - 1), per = 32 / L, pieces = a.D / n;
  const T *src[2] = {static_cast<const T *>(a.k) + t * a.k_row,
                     static_cast<const T *>(a.v) + t * a.v_row};
  const int64_t head[2] = {a.k_head, a.v_head};
  for (int h0 = lane / L; h0 - lane / L < a.H; h0 += per * kAhead) {  // alike in all lanes
    Piece<T> x[kAhead][2][NP];
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const int h = h0 + y * per, at = sub + p * L;
          x[y][c][p].u = make_uint4(0, 0, 0, 0);
          if (h < a.H && at < pieces)
            x[y][c][p].u =
                __ldg(reinterpret_cast<const uint4 *>(src[c] + h * head[c] + at * n));
        }
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int h = h0 + y * per;
        uint32_t top = 0;
#pragma unroll
        for (int p = 0; p < NP; ++p) top = max(top, x[y][c][p].top());
        for (int w = L >> 1; w > 0; w >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, w));
        const uint32_t b = exponent_of<F>(top);
        const float inv = __uint_as_float(b == 255 ? 0u : (254u - b) << 23);
        if (h >= a.H) continue;
        const Held &held = c ? a.vc : a.kc;
        uint8_t *to = held.codes + pg * held.at.for_page + off * held.at.for_token +
                      h * held.at.for_head;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
          const int at = sub + p * L;
          if (at >= pieces) continue;
          uint32_t w[2] = {0, 0};  // a row that is not finite has no codes
#pragma unroll
          for (int e = 0; e < n / 4; ++e) {
            float v[4];
            x[y][c][p].get(e, v);
            if (b != 255) w[e] = encode4<F>(v, inv);
          }
          if constexpr (n == 4) {
            *reinterpret_cast<uint32_t *>(to + at * n) = w[0];
          } else {
            *reinterpret_cast<uint2 *>(to + at * n) = make_uint2(w[0], w[1]);
          }
        }
        if (sub == 0)
          held.exps[pg * held.exps_at.for_page + off * held.exps_at.for_token +
                    h * held.exps_at.for_head] = (uint8_t)b;
      }
  }
}

template <typename T>
__device__ __forceinline__ void put8(T *to, const float (&x)[4], const float (&y)[4]) {
  if constexpr (sizeof(T) == 4) {
    reinterpret_cast<float4 *>(to)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(to)[1] = make_float4(y[0], y[1], y[2], y[3]);
  } else {
    const __nv_bfloat162 u[4] = {__floats2bfloat162_rn(x[0], x[1]), __floats2bfloat162_rn(x[2], x[3]),
                                 __floats2bfloat162_rn(y[0], y[1]), __floats2bfloat162_rn(y[2], y[3])};
    *reinterpret_cast<uint4 *>(to) = *reinterpret_cast<const uint4 *>(u);
  }
}

// A warp reads a token back, eight codes per lane and step, kAhead steps of keys and of
// values in flight. bf16 holds every value exactly, unless it is below its normal
// numbers.
template <typename T, int F>
__global__ void __launch_bounds__(kThreads) read_kernel(Rows a) {
  constexpr int kAhead = 4;
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (t >= a.T) return;
  int64_t pg = 0, off = 0;
  const bool there = find_slot(a, t, &pg, &off);
  const int per = a.D / 8, pieces = a.H * per;
  T *out[2] = {static_cast<T *>(a.k) + t * a.k_row, static_cast<T *>(a.v) + t * a.v_row};
  const int64_t head[2] = {a.k_head, a.v_head};
  for (int x0 = lane; x0 < pieces; x0 += 32 * kAhead) {
    uint2 u[kAhead][2];
    uint32_t b[kAhead][2];
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int x = x0 + 32 * y, h = x / per, at = (x - h * per) * 8;
        const Held &held = c ? a.vc : a.kc;
        u[y][c] = make_uint2(0, 0);
        b[y][c] = 127;
        if (there && x < pieces) {
          u[y][c] = __ldg(reinterpret_cast<const uint2 *>(held.codes + pg * held.at.for_page +
                                                          off * held.at.for_token +
                                                          h * held.at.for_head + at));
          b[y][c] = __ldg(held.exps + pg * held.exps_at.for_page + off * held.exps_at.for_token +
                          h * held.exps_at.for_head);
        }
      }
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int x = x0 + 32 * y, h = x / per, at = (x - h * per) * 8;
        if (x >= pieces) continue;
        float lo[4] = {}, hi[4] = {};
        if (there) {
          const float s = scale_of(b[y][c]);
          decode4<F>(u[y][c].x, lo);
          decode4<F>(u[y][c].y, hi);
#pragma unroll
          for (int k = 0; k < 4; ++k) lo[k] *= s, hi[k] *= s;
        }
        put8(out[c] + h * head[c] + at, lo, hi);
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
  const unsigned blocks = (unsigned)ceil_div(a.T, kThreads / 32);
  const int pieces = a.D / Piece<T>::n;
  int L = 1;
  while (L < 32 && L < pieces) L *= 2;
  PAIR_BEGIN("cache_append_q8", s);
  if (pieces <= 32) {
    append_kernel<T, F, 1><<<blocks, kThreads, 0, s>>>(a, L);
  } else {
    if constexpr (sizeof(T) == 4)  // 256 fp32 entries are two pieces a lane
      append_kernel<T, F, 2><<<blocks, kThreads, 0, s>>>(a, L);
  }
  PAIR_LAUNCH_CHECK(s);
  return PAIR_OK;
}

template <typename T, int F>
pair_status read(const Rows &a, cudaStream_t s) {
  PAIR_BEGIN("cache_read_q8", s);
  read_kernel<T, F><<<(unsigned)ceil_div(a.T, kThreads / 32), kThreads, 0, s>>>(a);
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
