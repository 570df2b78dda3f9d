// Rows of sequences on paged caches, and what lanes do with their elements: the
// descriptions' limits, exchanges between lanes without LDS, rows of any element
// type (device code of the cache kernels), launches by sequences.
#pragma once

#include <algorithm>

#include "hh_device.h"
#include "hh_kv.h"

namespace hh {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

struct Seq {
  int row0, n, first, trow;  // rows row0 .. row0 + n - 1 at positions first ..
};

// The sequence's rows, kept inside the buffers whatever the device arrays say.
__device__ __forceinline__ Seq load_seq(const Kv4Pool& P, const Kv4Rows& R, int s) {
  // (Every pointer read, whether given or not, so that the loads go out together.)
  const int* starts = (R.row_start ? R.row_start : R.first_pos) + s;
  const int* rows = (R.table_row ? R.table_row : R.first_pos) + s;
  const int first = R.first_pos[s], a0 = starts[0], b0 = starts[R.row_start ? 1 : 0], row = rows[0];
  const int a = R.row_start ? a0 : s, b = R.row_start ? b0 : s + 1;
  Seq q;
  q.row0 = min(max(a, 0), R.n_rows);
  q.n = min(max(min(max(b, 0), R.n_rows) - q.row0, 0), R.max_rows);
  q.first = max(min(first, 1 << 30), -(1 << 30));
  q.trow = R.table_row ? row : s;
  // No such table row: every position is padding.
  if (q.trow < 0 || q.trow >= P.table_rows) {
    q.trow = 0;
    q.first = -(1 << 30);
  }
  return q;
}

// Exchanges without LDS.  The lane's number 8 lanes on in its row of 16:
__device__ __forceinline__ unsigned other8(unsigned x) { return (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, 0x128, 0xF, 0xF, false); }
__device__ __forceinline__ float other8(float x) { return __uint_as_float(other8(__float_as_uint(x))); }
// Largest of 8 lanes, ...
template <int CTRL>
__device__ __forceinline__ unsigned max_dpp(unsigned x) {
  return max(x, (unsigned)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ unsigned max8(unsigned x) { return max_dpp<0x141>(max_dpp<0x4E>(max_dpp<0xB1>(x))); }
// ... and of the lanes with one number in the wave's four rows of 16 (and their sum).
__device__ __forceinline__ unsigned rows_max(unsigned x) {
  const auto a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  const unsigned y = max((unsigned)a[0], (unsigned)a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(y, y, false, false);
  return max((unsigned)b[0], (unsigned)b[1]);
}
__device__ __forceinline__ float rows_max(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(y), __float_as_uint(y), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// x / d as a product (x < 2^31): the multiplier is 2^(31 + s) / d rounded up, s the
// least with 2^s >= d, so it is off by less than 2^s / d of 2^-31.
struct Div {
  unsigned mul, shift, d;
};
Div div_by(unsigned d) {
  unsigned s = 0;
  while ((1u << s) < d) ++s;
  return Div{(unsigned)((((uint64_t)1 << (31 + s)) + d - 1) / d), s, d};
}
__device__ __forceinline__ unsigned operator/(unsigned x, Div v) {
  return (unsigned)(((uint64_t)x * v.mul) >> 31 >> v.shift);
}
// N elements (N * size a multiple of 8 bytes, 8-byte aligned) as fp32.
template <int N>
__device__ __forceinline__ void load_row(const void* p, size_t at, int type, float* f) {
  if (type == kRowF32) {
    const f32x4* s = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const f32x4 v = s[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[4 * i + j] = v[j];
    }
    return;
  }
  unsigned w[N / 2];
  const u32x2* s = reinterpret_cast<const u32x2*>(static_cast<const unsigned short*>(p) + at);
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const u32x2 v = s[i];
    w[2 * i] = v[0];
    w[2 * i + 1] = v[1];
  }
  if (type == kRowF16) {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const f16x2 h = __builtin_bit_cast(f16x2, w[i]);
      f[2 * i] = (float)h[0];
      f[2 * i + 1] = (float)h[1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}

// 8 elements at each of two places, in flight (raw) and as fp32.
struct RawRow {
  u32x4 w[4];
};
__device__ __forceinline__ void load_raw(RawRow& r, const void* p, size_t at, size_t next, int type) {
  if (type == kRowF32) {
    const u32x4* a = reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + at);
    const u32x4* b = reinterpret_cast<const u32x4*>(static_cast<const float*>(p) + next);
    r.w[0] = a[0];
    r.w[1] = a[1];
    r.w[2] = b[0];
    r.w[3] = b[1];
  } else {
    r.w[0] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned short*>(p) + at);
    r.w[1] = *reinterpret_cast<const u32x4*>(static_cast<const unsigned short*>(p) + next);
    r.w[2] = r.w[3] = u32x4{0u, 0u, 0u, 0u};
  }
}
__device__ __forceinline__ void raw_values(const RawRow& r, int type, float* f) {
  // (One branch on the type, not one an element.)
  if (type == kRowF32) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const unsigned w = r.w[i >> 2][i & 3];
      f[i] = __uint_as_float(w);
    }
  } else if (type == kRowF16) {
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const unsigned w = r.w[i >> 3][(i >> 1) & 3];
      const f16x2 h = __builtin_bit_cast(f16x2, w);
      f[i] = (float)h[0];
      f[i + 1] = (float)h[1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; i += 2) {
      const unsigned w = r.w[i >> 3][(i >> 1) & 3];
      f[i] = __uint_as_float(w << 16);
      f[i + 1] = __uint_as_float(w & 0xffff0000u);
    }
  }
}

__device__ __forceinline__ unsigned pack16(float a, float b, int type) {
  if (type == kRowF16) return __builtin_bit_cast(unsigned, f16x2{(_Float16)a, (_Float16)b});
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, bf16x2{(__bf16)a, (__bf16)b});
}

template <int N>
__device__ __forceinline__ void store_row(void* p, size_t at, int type, const float* f) {
  if (type == kRowF32) {
    f32x4* d = reinterpret_cast<f32x4*>(static_cast<float*>(p) + at);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) d[i] = f32x4{f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]};
    return;
  }
  u32x2* d = reinterpret_cast<u32x2*>(static_cast<unsigned short*>(p) + at);
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    d[i] = u32x2{pack16(f[4 * i], f[4 * i + 1], type), pack16(f[4 * i + 2], f[4 * i + 3], type)};
}

// Magnitudes as integers have their order, and Inf and NaN above all of them.
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr unsigned kInfBits = 0x7f800000u;

// Pages that max_rows consecutive positions can touch.
int row_tiles(const Kv4Rows& R) { return (R.max_rows + kPage - 2) / kPage + 1; }

// A launch has fewer than 2^32 threads: as many sequences as fit (those with
// fewer rows than the longest have workgroups that end at once).
template <typename F>
static hipError_t by_sequences(const Kv4Rows& R, int64_t threads_each, F some) {
  Kv4Rows r = R;
  const int most = (int)std::max<int64_t>(1, std::min<int64_t>(R.n_seqs, kMaxThreads / threads_each));
  for (int s = 0; s < R.n_seqs; s += r.n_seqs) {
    r.seq0 = s;
    r.n_seqs = std::min(most, R.n_seqs - s);
    const hipError_t e = some(r);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace
}  // namespace hh
