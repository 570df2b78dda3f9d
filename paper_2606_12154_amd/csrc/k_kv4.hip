// A paged KV cache in 4 bits: quantizing rows into pages, reading them back,
// and causal grouped-query attention over the pages (gfx950).
//
// Values are c * s: c an integer in -7 .. 7, s a scale of at most 8
// significant bits for 32 dimensions of one position and head, a multiple of
// 2^-24 of at most 2720.  Hence c * s and 24 s are fp16 numbers, and with a
// code's nibble n = c + 8 in bits 6 .. 9 of 0x4c00 (16 + n as fp16) one packed
// fp16 FMA, (16 + n) s - 24 s, gives two values without a rounding: a shift, an
// and-or and an FMA for two elements.
//
// The block of a (page, head) is laid out so that a lane's 8 bytes are what it
// needs as an operand of mfma_f32_16x16x32_f16 (lane l: row or column l % 16,
// contraction elements 8 (l / 16) .. + 7), with no transposition:
//   keys    lane l holds slot l % 16, dimensions 8 (l / 16) .. + 7 of each half;
//   values  lane l holds slots 4 (l / 16) .. + 3, dimensions 4 (l % 16) .. + 3.
// The scores of two pages, S^T[slot][query] (accumulator: column l % 16, rows
// 4 (l / 16) + i), leave each lane with the slots of both pages that its value
// bytes hold; with the contraction of O^T[dim][query] += V^T P^T taken in that
// order, weights go from accumulators to operands within their lanes.
//
// Precision: a query and a weight are two fp16 terms each, 22 bits, with every
// output type (one term where a 16-bit query needs no other): bf16 results differ
// from those of fp32 products by 4e-5 of their norm, beside a rounding of 1.7e-3.
// Single terms made that 1e-3 (and an 8,192-token prompt 338 us, 32 sequences of 4,000
// positions 19.3).
//
// What bounds it (counters): vector and matrix instructions, which hardly run at once.
// A step of two pages takes a wave about 110 vector ones to unpack, 7.5 issue slots (the
// exponential four of them) a score and lane, and 18 matrix ones a column tile (14 with
// queries of one term): an 8,192-token prompt (32 query heads on 8) takes 513 us, 0.54
// PFLOP/s, 260 of vector issue and 263 of the matrix unit.
// With few rows memory does, and hides only a part of them: 32 sequences of 4,000
// positions (74 MB) take 22 us, 3.4 TB/s, the same loads alone 16 (the longest
// sequence, which one workgroup a kv head takes whole, is 1.4 times the mean); one of
// 131,072 21.8, and 18.
#include "hh_device.h"
#include "hh_kv.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace hh {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr int kKeyScales = 1024, kValueScales = 1088;  // byte offsets in a block
constexpr float kMaxScale = 2720.f;

// ------------------------------------------------------------------ rows and types

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

__device__ __forceinline__ const unsigned char* block_of(const Kv4Pool& P, const int* row, int page, int head) {
  const int id = row[page];
  // An id outside the pool reads its first page.
  return P.pool + ((size_t)((unsigned)id < (unsigned)P.n_pages ? id : 0) * P.hkv + head) * kKv4Block;
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

// ------------------------------------------------------------------ append and read

// x / s as a division rounds it, wherever that decides: a reciprocal and one
// correction by the residual.  The quotient's distance from the middle between
// two fp32 numbers is 0 or at least 1/510 of their distance (s has 8 significant bits,
// and 7 has 3), and 0 only for a power of two, whose reciprocal is exact; the
// corrected quotient is 2^-22 off.
__device__ __forceinline__ float quotient(float x, float s, float r) {
  const float q = x * r;
  return fmaf(fmaf(-q, s, x), r, q);
}

// Scale of a group whose largest magnitude is a (finite).
__device__ __forceinline__ float group_scale(float a) {
  const float t = quotient(a, 7.0f, 1.0f / 7.0f);
  const unsigned u = __float_as_uint(t);
  const float s = fminf(__uint_as_float((u + 0x7fffu + ((u >> 16) & 1u)) & 0xffff0000u), kMaxScale);
  return t < 0x1p-17f ? rintf(t * 0x1p24f) * 0x1p-24f : s;
}

// Reciprocal of a scale; 0, and hence code 0, for a zero scale or NaN.
__device__ __forceinline__ float scale_rcp(float s) { return s > 0.f ? __builtin_amdgcn_rcpf(s) : 0.f; }

// Nibbles c + 8 of four finite elements, a's the lowest: r is scale_rcp(s); s is
// finite.  (Their number, a sum of at most 30,583, is exact in fp32.)
__device__ __forceinline__ unsigned codes_of(float a, float b, float c, float d, float s, float r) {
  auto code = [&](float x) { return __builtin_amdgcn_fmed3f(rintf(quotient(x, s, r)), -7.f, 7.f); };
  return (unsigned)((int)fmaf(fmaf(fmaf(code(d), 16.f, code(c)), 16.f, code(b)), 16.f, code(a)) + 0x8888);
}

// Magnitudes as integers have their order, and Inf and NaN above all of them.
__device__ __forceinline__ unsigned magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }
constexpr unsigned kInfBits = 0x7f800000u;

__device__ __forceinline__ unsigned short half_bits(float s) {
  return __builtin_bit_cast(unsigned short, (_Float16)s);
}

// One wave has one (page, head) of one sequence: the rows of the call that lie
// in that page.  Keys: lane (slot r, quarter g) has the 16 dimensions of its 8
// code bytes, which are whole rotation pairs (i, i + 32); values: lane (r, g)
// the 4 slots x 4 dimensions of its own.  A page that the rows fill is written
// 8 bytes a lane; in one that they fill partly a lane writes its slots alone.
__global__ __launch_bounds__(256) void k_kv4_append(Kv4Pool P, Kv4Rows R, const void* __restrict__ k,
                                                    const void* __restrict__ v, int type, int64_t ks, int64_t vs,
                                                    RopeTable rope, int tiles) {
  const int lane = threadIdx.x & 63;
  const int head = blockIdx.y * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (head >= P.hkv) return;
  const unsigned sq = blockIdx.x / (unsigned)tiles;
  const int tile = blockIdx.x - sq * tiles;
  const Seq q = load_seq(P, R, R.seq0 + sq);
  const int lo = max(q.first, 0);
  int hi = min(q.first + q.n, P.max_pages * kPage);
  if (rope.at) hi = min(hi, rope.len);
  const int page = lo / kPage + tile;
  if (page >= (hi + kPage - 1) >> 4) return;  // (page * kPage may pass 31 bits)
  const int id = P.table[(size_t)q.trow * P.max_pages + page];
  if ((unsigned)id >= (unsigned)P.n_pages) return;
  unsigned char* blk = P.pool + ((size_t)id * P.hkv + head) * kKv4Block;
  const int r = lane & 15, g = lane >> 4;

  {
    const int pos = page * kPage + r;
    const bool mine = pos >= lo && pos < hi;
    float x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
    if (mine) {
      const size_t at = (size_t)(q.row0 + (pos - q.first)) * ks + head * 64 + 8 * g;
      load_row<8>(k, at, type, x);
      load_row<8>(k, at + 32, type, x + 8);
      if (rope.at) {
        const float2* cs = rope.at + (size_t)pos * 32 + 8 * g;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 t = cs[i];
          const double a = x[i], b = x[8 + i], c = t.x, s = t.y;
          x[i] = (float)(a * c - b * s);
          x[8 + i] = (float)(b * c + a * s);
        }
      }
    }
    unsigned top[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 16; ++i) top[i >> 3] = max(top[i >> 3], magnitude(x[i]));
    top[0] = rows_max(top[0]);
    top[1] = rows_max(top[1]);
    const bool bad = max(top[0], top[1]) >= kInfBits;
    unsigned word[2], sc = 0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const float s = group_scale(__uint_as_float(top[t])), rs = scale_rcp(s);
      const float* y = x + 8 * t;
      const unsigned d = codes_of(y[0], y[2], y[4], y[6], s, rs) | codes_of(y[1], y[3], y[5], y[7], s, rs) << 16;
      // (A row that is not finite: codes of 0.)
      word[t] = bad ? 0x88888888u : d;
      sc |= (bad ? 0x7e00u : (unsigned)half_bits(s)) << (16 * t);
    }
    if (mine) {
      *reinterpret_cast<u32x2*>(blk + 8 * lane) = u32x2{word[0], word[1]};
      if (g == 0) *reinterpret_cast<unsigned*>(blk + kKeyScales + 4 * r) = sc;
    }
  }

  unsigned short code[4], sc[4];
  bool mine[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * g + i, pos = page * kPage + slot;
    mine[i] = pos >= lo && pos < hi;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (mine[i]) load_row<4>(v, (size_t)(q.row0 + (pos - q.first)) * vs + head * 64 + 4 * r, type, x);
    unsigned top = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max(top, magnitude(x[j]));
    top = max8(top);
    const bool bad = max(top, other8(top)) >= kInfBits;
    const float s = group_scale(__uint_as_float(top)), rs = scale_rcp(s);
    const unsigned d = codes_of(x[0], x[1], x[2], x[3], s, rs);
    code[i] = (unsigned short)(bad ? 0x8888u : d);
    sc[i] = bad ? 0x7e00u : half_bits(s);
  }
  unsigned short* vb = reinterpret_cast<unsigned short*>(blk + 512) + 4 * lane;
  unsigned short* vsc = reinterpret_cast<unsigned short*>(blk + kValueScales) + (r >> 3) * 16 + 4 * g;
  if (mine[0] && mine[3]) {
    *reinterpret_cast<u32x2*>(vb) =
        u32x2{code[0] | (unsigned)code[1] << 16, code[2] | (unsigned)code[3] << 16};
    if ((r & 7) == 0)
      *reinterpret_cast<u32x2*>(vsc) = u32x2{sc[0] | (unsigned)sc[1] << 16, sc[2] | (unsigned)sc[3] << 16};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (mine[i]) {
        vb[i] = code[i];
        if ((r & 7) == 0) vsc[i] = sc[i];
      }
  }
}

// The same lanes the other way round.  Tiles are counted from the page of the
// first position, which may be negative: such rows, and those past the page
// table, are set to zero.
__global__ __launch_bounds__(256) void k_kv4_read(Kv4Pool P, Kv4Rows R, void* __restrict__ k, void* __restrict__ v,
                                                  int type, int64_t ks, int64_t vs, int tiles) {
  const int lane = threadIdx.x & 63;
  const int head = blockIdx.y * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (head >= P.hkv) return;
  const unsigned sq = blockIdx.x / (unsigned)tiles;
  const int tile = blockIdx.x - sq * tiles;
  const Seq q = load_seq(P, R, R.seq0 + sq);
  const int page = (q.first >> 4) + tile;  // floor
  const int hi = q.first + q.n;
  if (page >= (hi + kPage - 1) >> 4) return;  // (page * kPage may pass 31 bits)
  const bool held = page >= 0 && page < P.max_pages;
  const unsigned char* blk =
      block_of(P, P.table + (size_t)q.trow * P.max_pages, held ? page : 0, head);
  const int r = lane & 15, g = lane >> 4;

  {
    const int pos = page * kPage + r;
    if (pos >= q.first && pos < hi) {
      const u32x2 word = *reinterpret_cast<const u32x2*>(blk + 8 * lane);
      const unsigned sc = *reinterpret_cast<const unsigned*>(blk + kKeyScales + 4 * r);
      const f16x2 s = __builtin_bit_cast(f16x2, sc);
      const size_t at = (size_t)(q.row0 + (pos - q.first)) * ks + head * 64 + 8 * g;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int c = (int)(word[t] >> (4 * (e >> 1) + 16 * (e & 1)) & 15u) - 8;
          x[e] = held ? (float)c * (float)s[t] : 0.f;
        }
        store_row<8>(k, at + 32 * t, type, x);
      }
    }
  }
  const u32x2 word = *reinterpret_cast<const u32x2*>(blk + 512 + 8 * lane);
  const u32x2 sc = *reinterpret_cast<const u32x2*>(blk + kValueScales + (r >> 3) * 32 + 8 * g);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int pos = page * kPage + 4 * g + i;
    if (pos < q.first || pos >= hi) continue;
    const unsigned both = sc[i >> 1];
    const f16x2 s = __builtin_bit_cast(f16x2, both);
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int c = (int)(word[i >> 1] >> (16 * (i & 1) + 4 * j) & 15u) - 8;
      x[j] = held ? (float)c * (float)s[i & 1] : 0.f;
    }
    store_row<4>(v, (size_t)(q.row0 + (pos - q.first)) * vs + head * 64 + 4 * r, type, x);
  }
}

// Pages that max_rows consecutive positions can touch.
int row_tiles(const Kv4Rows& R) { return (R.max_rows + kPage - 2) / kPage + 1; }

// ------------------------------------------------------------------ attention

// Operand columns are (row, query head of the kv head's group) pairs, row-major:
// column c of a sequence is row c / G, head c % G.
// Pages of a split, given the pages that a column tile attends to: whole steps of two.
__device__ __forceinline__ int split_pages(int np, int splits) {
  const int pairs = (np + 1) >> 1;
  return 2 * ((pairs + splits - 1) / splits);
}

struct PageRegs {
  u32x2 k, v, vs;
  unsigned ks;
};

// The block as a buffer: its base stays in scalar registers, a lane's offset in
// one vector register (with addresses of 64 bits a lane, 2 to 5% more).
__device__ __forceinline__ void load_page(PageRegs& r, const unsigned char* blk, unsigned lane) {
  const auto b = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(blk), 0, kKv4Block, 0x00027000);
  r.k = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b, 8 * lane, 0, 0));
  r.v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b, 8 * lane + 512, 0, 0));
  r.ks = __builtin_amdgcn_raw_buffer_load_b32(b, 4 * (lane & 15) + kKeyScales, 0, 0);
  r.vs = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(b, (lane & 8) * 4 + 8 * (lane >> 4) + kValueScales, 0, 0));
}

// Nibble j of both halves of w as 16 + n.  The mask comes in a vector register:
// with both constants in scalar ones and-or would be two instructions.
template <int J>
__device__ __forceinline__ f16x2 codes16(unsigned w, unsigned mask) {
  const unsigned x = J < 2 ? w << (6 - 4 * J) : w >> (4 * J - 6);
  return __builtin_bit_cast(f16x2, (x & mask) | 0x4c004c00u);
}
__device__ __forceinline__ unsigned code_mask() {
  unsigned m;
  asm("v_mov_b32 %0, 0x03c003c0" : "=v"(m));
  return m;
}

__device__ __forceinline__ f16x2 minus24(f16x2 s) { return s * f16x2{(_Float16)-24, (_Float16)-24}; }

// The lane's 8 keys' elements of one dword under one scale.
__device__ __forceinline__ f16x8 key_frag(unsigned w, unsigned mask, f16x2 s) {
  const f16x2 b = minus24(s);
  const f16x2 x0 = __builtin_elementwise_fma(codes16<0>(w, mask), s, b), x1 = __builtin_elementwise_fma(codes16<1>(w, mask), s, b);
  const f16x2 x2 = __builtin_elementwise_fma(codes16<2>(w, mask), s, b), x3 = __builtin_elementwise_fma(codes16<3>(w, mask), s, b);
  return f16x8{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}

// Dimension 4 r + J of the lane's 4 slots; s, b: their scales, and -24 times.
template <int J>
__device__ __forceinline__ f16x4 value_frag(u32x2 w, unsigned mask, const f16x2* s, const f16x2* b) {
  const f16x2 lo = __builtin_elementwise_fma(codes16<J>(w[0], mask), s[0], b[0]);
  const f16x2 hi = __builtin_elementwise_fma(codes16<J>(w[1], mask), s[1], b[1]);
  return f16x4{lo[0], lo[1], hi[0], hi[1]};
}

// A page's operands: keys, and values.  MASK: values that no row of the tile sees
// (slots from `seen` on) may be anything, and a NaN that only some rows see must
// not reach the others as 0 x NaN: such values become 0, and bit i of `bad` says that
// the lane's value slot i is NaN, which then goes through the scores.
__device__ __forceinline__ void keys_of(u32x2 k, unsigned scales, unsigned mask, f16x8* kf) {
  const f16x2 s = __builtin_bit_cast(f16x2, scales);
  const unsigned k0 = k[0], k1 = k[1];
  kf[0] = key_frag(k0, mask, f16x2{s[0], s[0]});
  kf[1] = key_frag(k1, mask, f16x2{s[1], s[1]});
}
// In steps that mask, of two pages whose scores share an accumulator: keys that
// would make the other page's scores NaN are zeros.  Returns the lane's four slots that held NaN.
__device__ __forceinline__ unsigned mask_keys(unsigned& scales, int page, int seen) {
  const int lane = threadIdx.x & 63;
  const bool nan = (scales & 0x7c00u) == 0x7c00u || (scales & 0x7c000000u) == 0x7c000000u;
  if (nan || page * kPage + (lane & 15) >= seen) scales = 0u;
  return (unsigned)__builtin_amdgcn_ballot_w64(nan) >> (lane >> 4) * 4 & 15u;
}
template <bool MASK>
__device__ __forceinline__ void values_of(u32x2 v, u32x2 scales, unsigned mask, int page, int seen, f16x4* vf,
                                          unsigned* bad) {
  f16x2 s[2], b[2];
  unsigned nan4 = 0;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    unsigned w = scales[h];
    if constexpr (MASK) {
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int slot = page * kPage + 4 * (int)((threadIdx.x & 63) >> 4) + 2 * h + z;
        const bool nan = ((w >> (16 * z)) & 0x7c00u) == 0x7c00u;
        if (nan || slot >= seen) w &= z ? 0x0000ffffu : 0xffff0000u;
        if (nan) nan4 |= 1u << (2 * h + z);
      }
    }
    s[h] = __builtin_bit_cast(f16x2, w);
    b[h] = minus24(s[h]);
  }
  if constexpr (MASK) {
    // Either group of a value row may hold the NaN: lanes r and r ^ 8.
    *bad = nan4 | other8(nan4);
  }
  vf[0] = value_frag<0>(v, mask, s, b);
  vf[1] = value_frag<1>(v, mask, s, b);
  vf[2] = value_frag<2>(v, mask, s, b);
  vf[3] = value_frag<3>(v, mask, s, b);
}

// A weight as two fp16 terms: what its nearest fp16 number leaves goes into the second
// (two at once: two conversions of pairs and two mixed FMAs, where single
// conversions there and back take twice as many instructions).
__device__ __forceinline__ void split_weights(float a, float b, f16x2& h, f16x2& l) {
  h = f16x2{(_Float16)a, (_Float16)b};
  const unsigned w = __builtin_bit_cast(unsigned, h);
  float x, y;
  asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel_hi:[1,0,0]" : "=v"(x) : "v"(w), "v"(a));
  asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(y) : "v"(w), "v"(b));
  l = f16x2{(_Float16)x, (_Float16)y};
}

__device__ __forceinline__ f16x8 join8(f16x4 a, f16x4 b) {
  return f16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

// Weights are 2^(S qs - base): base puts a column's largest score so far at
// 2^kOffset, and is raised once a score passes 2^(kOffset + kSlack), which fp16
// still holds, so that a weight is off by 2^-37 of the row's largest at most (half
// of fp16's lowest step, 2^-25).  A higher offset would keep more and raise the base
// more often; with this one later scores of ordinary rows hardly pass the largest of a
// wave's first 32 by the slack's factor of 15, and the step needs no reductions across
// lanes (8,192-token prompt 513 us, as with an offset of 2^7 and a slack of 2^8).
constexpr float kOffset = 12.f, kSlack = 3.9f;

// Loads in flight need not land at this barrier: it orders LDS alone.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Where a wave stands: columns c0 .. c0 + 16 NQ - 1 of one (sequence, kv head).
struct Place {
  Seq s;
  int head, G, cols, c0;
  Div group;
};

// The query of the lane's column of a 16-column tile, 8 dimensions of each half:
// as loaded (with its rotation), and as operands.
struct RawQuery {
  RawRow row;
  f32x4 turn[4];
};
// QT: fp16 terms, two of fp32 and rotated queries, one of 16-bit ones that are not
// rotated.  Queries (but for fp16 ones of one term) are scaled by a power of two that puts
// a row's largest element into [2^13, 2^14), so that one term holds any 16-bit
// query and two hold 22 bits of an fp32 one.
template <int QT>
struct Query {
  f16x8 h[2], l[QT == 2 ? 2 : 1];
  float qs;  // scores to powers of two
};

// A lane's column in its tile of 16 / PACK.
template <int PACK>
__device__ __forceinline__ int column_of() { return threadIdx.x & (16 / PACK - 1); }
// Columns behind the last one repeat it (and are not written).
__device__ __forceinline__ int column_row(const Place& w, int c) { return (unsigned)min(c, w.cols - 1) / w.group; }

template <int QT, int PACK>
__device__ __forceinline__ void load_query(RawQuery& q, const Place& w, const Kv4Attend& A, int tile) {
  const int lane = threadIdx.x & 63, g = lane >> 4, c = w.c0 + 16 * tile + column_of<PACK>();
  const int rw = column_row(w, c), j = min(c, w.cols - 1) - rw * w.G;
  const size_t at = (size_t)(w.s.row0 + rw) * A.q_stride + (w.head * w.G + j) * 64 + 8 * g;
  load_raw(q.row, A.q, at, at + 32, A.q_type);
  if (QT == 2 && A.rope.at) {
    const int pos = min(max(w.s.first + rw, 0), A.rope.len - 1);
    const f32x4* cs = reinterpret_cast<const f32x4*>(A.rope.at + (size_t)pos * 32 + 8 * g);
#pragma unroll
    for (int i = 0; i < 4; ++i) q.turn[i] = cs[i];
  }
}

template <int QT>
__device__ __forceinline__ Query<QT> make_query(const RawQuery& q, const Kv4Attend& A) {
  Query<QT> z;
  if (QT == 1 && A.q_type == kRowF16) {
    z.h[0] = __builtin_bit_cast(f16x8, q.row.w[0]);
    z.h[1] = __builtin_bit_cast(f16x8, q.row.w[1]);
    z.qs = fmaxf(A.scale * 1.4426950408889634f, 1e-37f);
    return z;
  }
  float x[16];
  raw_values(q.row, A.q_type, x);
  if (QT == 2 && A.rope.at) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = x[i], v = x[8 + i], co = q.turn[i >> 1][2 * (i & 1)], si = q.turn[i >> 1][2 * (i & 1) + 1];
      x[i] = u * co - v * si;
      x[8 + i] = v * co + u * si;
    }
  }
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[i]));
  top = rows_max(top);
  int e = 0;
  if (top > 0.f && top < INFINITY) e = 14 - __builtin_amdgcn_frexp_expf(top);
  z.qs = fmaxf(__builtin_amdgcn_ldexpf(A.scale * 1.4426950408889634f, -e), 1e-37f);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float y = __builtin_amdgcn_ldexpf(x[i], e);
    const _Float16 h = (_Float16)y;
    z.h[i >> 3][i & 7] = h;
    if constexpr (QT == 2) z.l[i >> 3][i & 7] = (_Float16)(y - (float)h);
  }
  return z;
}

// A wave's NQ tiles of 16 columns.
// PACK: of up to 8 columns, two copies stand side by side, the left one for the
// first page of a step, the right one for the second, each with zeros in the
// other's operands.  A lane then has four scores a step, not eight of which half
// are of no column, and the copies are joined at the end (32 sequences of 4,000
// positions 24.1 -> 22.2 us, one of 131,072 22.7 -> 21.8, of 300 5.0 -> 4.8).
template <int NQ, int QT, int PACK>
struct Columns {
  static_assert(PACK == 1 || NQ == 1);
  static constexpr int N = 8 / PACK;  // scores of a lane, step and tile
  Query<QT> q[NQ * PACK];
  int lim[NQ];  // keys that the column sees
  f32x4 o[NQ][4], sum[NQ];
  float base[NQ];
  bool first;

  __device__ __forceinline__ void start(const Place& w, int most) {
    first = true;
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
      sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
      base[t] = 0.f;
      lim[t] = min(max(w.s.first + column_row(w, w.c0 + 16 * t + column_of<PACK>()) + 1, 0), most);
    }
  }

  static __device__ __forceinline__ bool right() { return threadIdx.x & 8; }
  __device__ __forceinline__ void pack(const Query<QT>& z) {
    const f16x8 zero = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      q[k].qs = z.qs;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        q[k].h[i] = right() == k ? z.h[i] : zero;
        if constexpr (QT == 2) q[k].l[i] = right() == k ? z.l[i] : zero;
      }
    }
  }

  // A step takes two pages: their scores, the scores' weights, the weighted values.

  // kf[page][half of the dimensions].
  __device__ __forceinline__ void scores(const f16x8 (*kf)[2], f32x4 (*sc)[2]) const {
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x4& y = sc[t][PACK == 2 ? 0 : i];
        const Query<QT>& z = q[PACK == 2 ? i : t];
        if (PACK == 1 || i == 0) y = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (QT == 2) {
          y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i][0], z.l[0], y, 0, 0, 0);
          y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i][1], z.l[1], y, 0, 0, 0);
        }
        y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i][0], z.h[0], y, 0, 0, 0);
        y = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[i][1], z.h[1], y, 0, 0, 0);
      }
  }

  // MASK: slots past a column's keys, and bad (N bits, see values_of).  The check
  // of all columns' scores is the step's only branch.
  template <bool MASK>
  __device__ __forceinline__ void weights(const f32x4 (*sc)[2], int page, unsigned bad, f16x8* ph, f16x8* pl) {
    const int g = (threadIdx.x & 63) >> 4;
    float x[NQ][N], high = -INFINITY;
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        x[t][i] = fmaf(sc[t][i >> 2][i & 3], q[t].qs, -base[t]);
        if constexpr (MASK) {
          if (bad >> i & 1u) x[t][i] = NAN;
          if ((page + (PACK == 2 ? right() : i >> 2)) * kPage + 4 * g + (i & 3) >= lim[t]) x[t][i] = -INFINITY;
        }
        high = fmaxf(high, x[t][i]);
      }
    // A wave's first pages set the base: a column that sees none of them sees
    // none of the later ones either.
    if (first || __builtin_amdgcn_ballot_w64(high > kOffset + kSlack)) {
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        float mx = x[t][0];
#pragma unroll
        for (int i = 1; i < N; ++i) mx = fmaxf(mx, x[t][i]);
        mx = rows_max(mx);
        float up = mx > -INFINITY ? mx - kOffset : 0.f;
        if (!first) up = fmaxf(up, 0.f);
        const float f = first ? 1.f : __builtin_amdgcn_exp2f(-up);
        base[t] += up;
#pragma unroll
        for (int i = 0; i < N; ++i) x[t][i] -= up;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[t][j] *= f;
        sum[t] *= f;
      }
    }
    first = false;
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        f16x2 h, l;
        split_weights(__builtin_amdgcn_exp2f(x[t][i]), __builtin_amdgcn_exp2f(x[t][i + 1]), h, l);
        ph[t][i] = h[0];
        ph[t][i + 1] = h[1];
        pl[t][i] = l[0];
        pl[t][i + 1] = l[1];
      }
    if constexpr (PACK == 2) {
      ph[0] = on_side(ph[0]);
      pl[0] = on_side(pl[0]);
    }
  }
  // A lane's four weights where its page's values are.
  static __device__ __forceinline__ f16x8 on_side(const f16x8& w) {
    const f16x4 zero = {0, 0, 0, 0}, x = {w[0], w[1], w[2], w[3]};
    return join8(right() ? zero : x, right() ? x : zero);
  }

  // vf[dimension of four].  Weights are summed as they enter the products.
  __device__ __forceinline__ void values(const f16x8* vf, const f16x8* ph, const f16x8* pl) {
    const f16x8 ones = {1, 1, 1, 1, 1, 1, 1, 1};
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
#pragma unroll
      for (int j = 0; j < 4; ++j) o[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j], pl[t], o[t][j], 0, 0, 0);
      sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, pl[t], sum[t], 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 4; ++j) o[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[j], ph[t], o[t][j], 0, 0, 0);
      sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, ph[t], sum[t], 0, 0, 0);
    }
  }

  // A column that saw no key has no base.
  __device__ __forceinline__ float base_of(int t) const { return sum[t][0] == 0.f ? -INFINITY : base[t]; }
};

// N consecutive dimensions of column col, from d0 on: the output, or (joined)
// the split's part of it, with base m and sum of weights l.
template <int N>
__device__ __forceinline__ void put(const Kv4Rows& R, const Kv4Attend& A, const Place& w, int col, int d0, const float* x,
                                    float l, float m, bool joined, int split, int splits) {
  if (col >= w.cols) return;
  const int at_row = (unsigned)col / w.group;
  const int rw = w.s.row0 + at_row, hd = w.head * w.G + col - at_row * w.G;
  if (joined) {
    const size_t at = ((size_t)split * R.n_rows + rw) * A.hq + hd;
    float* dst = A.part + at * 64 + d0;
#pragma unroll
    for (int i = 0; i < N / 4; ++i)
      *reinterpret_cast<f32x4*>(dst + 4 * i) = f32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    if (d0 == 0) {
      float2* ml = reinterpret_cast<float2*>(A.part + (size_t)splits * R.n_rows * A.hq * 64) + at;
      *ml = make_float2(m, l);
    }
    return;
  }
  float y[N];
  const float inv = l == 0.f ? 0.f : 1.0f / l;  // nothing to attend to: 0
#pragma unroll
  for (int i = 0; i < N; ++i) y[i] = x[i] * inv;
  store_row<N>(A.out, (size_t)rw * A.out_stride + hd * 64 + d0, A.out_type, y);
}

// A workgroup has a tile of 16 NQ columns; its W waves take the tile's keys in
// turn (two pages a step) and join at the end.
template <int NQ, int QT, int W, int PACK>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(waves_fit(NQ)))) void
k_kv4_attend(Kv4Pool P, Kv4Rows R, Kv4Attend A, Div heads, Div splits_, Div tiles_, Div group) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const unsigned b1 = blockIdx.x / heads, b2 = b1 / splits_, sq = b2 / tiles_;
  const int split = b1 - b2 * splits_.d, splits = splits_.d;
  // The last tiles have the most keys: they go first.
  const int tile = tiles_.d - 1 - (b2 - sq * tiles_.d);
  const Seq s = load_seq(P, R, R.seq0 + sq);
  const int G = group.d, cols = s.n * G;  // below 2^31 with a tile to spare (kv4_plan)
  const Place w{s, (int)(blockIdx.x - b1 * heads.d), G, cols, tile * (16 * NQ), group};
  if (w.c0 >= cols) return;
  // Keys of the tile's first and last row.
  const int most = P.max_pages * kPage;
  const int row_a = (unsigned)w.c0 / group, row_b = (unsigned)(min(w.c0 + 16 * NQ, cols) - 1) / group;
  const int all_see = min(max(s.first + row_a + 1, 0), most), some_see = min(max(s.first + row_b + 1, 0), most);
  const int np = (some_see + kPage - 1) / kPage;
  const int per = split_pages(np, splits);
  const int p0 = split * per, p1 = min(p0 + per, np);
  const bool joined = per < np;  // several splits have keys
  if (split > 0 && p0 >= np) return;

  // What the first step needs goes out before the queries are worked on.  Loads
  // run one step ahead; what would lie behind the wave's last step is its last
  // step again (no branch around loads, whose waits would then have to assume that it was
  // not taken).  Lane i holds the page ids of the i-th of 64 steps: a load of ids
  // in each step would be waited for there.
  const int* row = P.table + (size_t)s.trow * P.max_pages;
  constexpr int STEP = 2 * W;
  int p = p0 + 2 * wave;
  const int last = max(p + (p1 - 1 - p) / STEP * STEP, 0);
  unsigned ids[2];
  auto load_ids = [&](int q) {
    const int at = min(q + lane * STEP, last);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned x = (unsigned)row[max(min(at + i, np - 1), 0)];
      ids[i] = x < (unsigned)P.n_pages ? x : 0u;  // an id outside the pool reads its first page
    }
  };
  int ahead = 0;  // the step that is fetched next
  auto fetch = [&](PageRegs* pr) {
    if (ahead == 64) {
      load_ids(p + STEP);
      ahead = 0;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned id = (unsigned)__builtin_amdgcn_readlane((int)ids[i], ahead);
      load_page(pr[i], P.pool + ((size_t)id * (unsigned)P.hkv + (unsigned)w.head) * kKv4Block, (unsigned)lane);
    }
    ++ahead;
  };
  load_ids(p);
  // Of several tiles, each wave makes one's queries for all.
  RawQuery raw;
  if (NQ == 1 || wave < NQ) load_query<QT, PACK>(raw, w, A, NQ == 1 ? 0 : wave);
  PageRegs a[2], c[2];
  fetch(a);
  Columns<NQ, QT, PACK> C;
  C.start(w, most);
  if constexpr (PACK == 2) {
    C.pack(make_query<QT>(raw, A));
  } else if constexpr (NQ == 1) {
    C.q[0] = make_query<QT>(raw, A);
  } else {
    __shared__ f16x8 made[NQ][2 * QT][64];
    __shared__ float made_qs[NQ][64];
    if (wave < NQ) {
      const Query<QT> z = make_query<QT>(raw, A);
#pragma unroll
      for (int i = 0; i < 2 * QT; ++i) made[wave][i][lane] = i < 2 ? z.h[i] : z.l[i - 2];
      made_qs[wave][lane] = z.qs;
    }
    lds_barrier();
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
#pragma unroll
      for (int i = 0; i < 2 * QT; ++i) (i < 2 ? C.q[t].h[i] : C.q[t].l[i - 2]) = made[t][i][lane];
      C.q[t].qs = made_qs[t][lane];
    }
  }

  const unsigned mask = code_mask();
  auto step = [&](const PageRegs* pr, auto masked) {
    constexpr bool MASK = decltype(masked)::value;
    f16x8 kf[2][2], vf[4];
    f16x4 va[4], vb[4];
    unsigned bad[2] = {0u, 0u};
    unsigned ks[2] = {pr[0].ks, pr[1].ks}, bad_key[2] = {0u, 0u};
    if constexpr (MASK && PACK == 2) {
      bad_key[0] = mask_keys(ks[0], p, some_see);
      bad_key[1] = mask_keys(ks[1], p + 1, some_see);
    }
    keys_of(pr[0].k, ks[0], mask, kf[0]);
    keys_of(pr[1].k, ks[1], mask, kf[1]);
    values_of<MASK>(pr[0].v, pr[0].vs, mask, p, some_see, va, &bad[0]);
    values_of<MASK>(pr[1].v, pr[1].vs, mask, p + 1, some_see, vb, &bad[1]);
#pragma unroll
    for (int j = 0; j < 4; ++j) vf[j] = join8(va[j], vb[j]);
    f32x4 sc[NQ][2];
    f16x8 ph[NQ], pl[NQ];
    C.scores(kf, sc);
    const int side = C.right();
    C.template weights<MASK>(sc, p, PACK == 2 ? (side ? bad[1] | bad_key[1] : bad[0] | bad_key[0]) : bad[0] | bad[1] << 4, ph, pl);
    C.values(vf, ph, pl);
  };
  {
    const int full = min(all_see / kPage & ~1, p1 & ~1);  // pages below are seen by every row
    bool swapped = false;
    while (p < full) {
      fetch(c);
      step(a, std::false_type());
      p += STEP;
      if (p >= full) {
        swapped = true;
        break;
      }
      fetch(a);
      step(c, std::false_type());
      p += STEP;
    }
    if (swapped) {
      a[0] = c[0];
      a[1] = c[1];
    }
    while (p < p1) {
      fetch(c);
      step(a, std::true_type());
      a[0] = c[0];
      a[1] = c[1];
      p += STEP;
    }
  }

  // Join the waves: of four of them, wave v takes dimensions 16 g + 4 v .. + 3.
  __shared__ f32x4 lo[W][4][64];
  __shared__ float2 ls[W][64];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    if (t) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) lo[wave][i][lane] = f32x4{C.o[t][0][i], C.o[t][1][i], C.o[t][2][i], C.o[t][3][i]};
    ls[wave][lane] = make_float2(C.base_of(t), C.sum[t][0]);
    __syncthreads();
    if (wave >= 4) continue;
    float m = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < W; ++v) m = fmaxf(m, ls[v][lane].x);
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float2 z = ls[v][lane];
      const float f = z.x > -INFINITY ? __builtin_amdgcn_exp2f(z.x - m) : 0.f;
      const f32x4 y = lo[v][wave][lane];
      l += f * z.y;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] += f * y[j];
    }
    if constexpr (PACK == 2) {
      const float m2 = fmaxf(m, other8(m)), f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - m2) : 0.f;
      m = m2;
      l = f * l + other8(f * l);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = f * x[j] + other8(f * x[j]);
      if (C.right()) continue;
    }
    put<4>(R, A, w, w.c0 + 16 * t + r, 16 * g + 4 * wave, x, l, m, joined, split, splits);
  }
}

// Splits that hold keys of column c's tile in a sequence (as the attention
// kernel cut them); 1: the attention kernel wrote the output.
__device__ __forceinline__ int splits_of(const Kv4Pool& P, const Seq& s, int G, int c, int tile_cols, int splits) {
  const int cols = s.n * G, c0 = c / tile_cols * tile_cols;
  const int row_b = (min(c0 + tile_cols, cols) - 1) / G;
  const int some_see = min(max(s.first + row_b + 1, 0), P.max_pages * kPage);
  const int np = (some_see + kPage - 1) / kPage, per = split_pages(np, splits);
  return per >= np ? 1 : (np + per - 1) / per;
}

// Joins the splits of few (row, head)s, a workgroup each: lane l of wave w has
// dimensions 4 (l % 16) .. + 3 of splits 4 w + l / 16, + 16, ...: all loads are
// in flight at once.
__global__ __launch_bounds__(256) void k_kv4_join(Kv4Pool P, Kv4Rows R, Kv4Attend A, int tile_cols, int splits) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned b = blockIdx.x, row = b / (unsigned)A.hq;
  const int hd = b - row * A.hq, i = row % (unsigned)R.max_rows;
  const Seq s = load_seq(P, R, R.seq0 + row / (unsigned)R.max_rows);
  if (i >= s.n) return;
  const int G = A.hq / P.hkv;
  const int n = splits_of(P, s, G, i * G + hd % G, tile_cols, splits);
  if (n == 1) return;
  const size_t at = (size_t)(s.row0 + i) * A.hq + hd, step = (size_t)R.n_rows * A.hq;
  const float2* ml = reinterpret_cast<const float2*>(A.part + (size_t)splits * step * 64) + at;
  const float* part = A.part + at * 64 + 4 * (lane & 15);
  constexpr int N = kMaxSplits / 16;  // loads of a lane
  f32x4 y[N];
  float2 z[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int sp = k * 16 + wave * 4 + (lane >> 4);
    y[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    z[k] = make_float2(-INFINITY, 0.f);
    if (sp < n) {
      z[k] = ml[sp * step];
      y[k] = *reinterpret_cast<const f32x4*>(part + sp * step * 64);
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < N; ++k) m = fmaxf(m, z[k].x);
  m = rows_max(m);
  float x[5] = {0.f, 0.f, 0.f, 0.f, 0.f};  // 4 dimensions and the sum of weights, against m
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float f = z[k].x > -INFINITY ? __builtin_amdgcn_exp2f(z[k].x - m) : 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] += f * y[k][j];
    x[4] += f * z[k].y;
  }
#pragma unroll
  for (int j = 0; j < 5; ++j) x[j] = rows_sum(x[j]);
  __shared__ float xs[4][6][16];
  if (lane < 16) {
#pragma unroll
    for (int j = 0; j < 5; ++j) xs[wave][j][lane] = x[j];
    xs[wave][5][lane] = m;
  }
  __syncthreads();
  if (threadIdx.x >= 16) return;
  m = fmaxf(fmaxf(xs[0][5][lane], xs[1][5][lane]), fmaxf(xs[2][5][lane], xs[3][5][lane]));
#pragma unroll
  for (int j = 0; j < 5; ++j) x[j] = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float mw = xs[w][5][lane], f = mw > -INFINITY ? __builtin_amdgcn_exp2f(mw - m) : 0.f;
#pragma unroll
    for (int j = 0; j < 5; ++j) x[j] += f * xs[w][j][lane];
  }
  const float inv = x[4] == 0.f ? 0.f : 1.0f / x[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] *= inv;
  store_row<4>(A.out, (size_t)(s.row0 + i) * A.out_stride + hd * 64 + 4 * lane, A.out_type, x);
}

// Up to 16 splits of many (row, head)s, 16 lanes each: lane l of them has
// split l's statistics and dimensions 4 l .. + 3.
__global__ __launch_bounds__(256) void k_kv4_join_rows(Kv4Pool P, Kv4Rows R, Kv4Attend A, int tile_cols, int splits) {
  const int l16 = threadIdx.x & 15;
  const unsigned b = blockIdx.x * 16u + (threadIdx.x >> 4), row = b / (unsigned)A.hq;
  const int hd = b - row * A.hq, i = row % (unsigned)R.max_rows;
  const unsigned sq = row / (unsigned)R.max_rows;
  // (No early return: the lanes of a wave exchange below.)
  const bool in = sq < (unsigned)R.n_seqs;
  const Seq s = load_seq(P, R, R.seq0 + (in ? sq : 0));
  const int G = A.hq / P.hkv;
  const int n = in && i < s.n ? splits_of(P, s, G, i * G + hd % G, tile_cols, splits) : 1;
  const size_t at = (size_t)(s.row0 + (n > 1 ? i : 0)) * A.hq + hd, step = (size_t)R.n_rows * A.hq;
  const float2* ml = reinterpret_cast<const float2*>(A.part + (size_t)splits * step * 64) + at;
  const float* part = A.part + at * 64 + 4 * l16;
  float2 z = make_float2(-INFINITY, 0.f);
  if (n > 1 && l16 < n) z = ml[l16 * step];
  const float m = row_max16(z.x);
  const float f = z.x > -INFINITY ? __builtin_amdgcn_exp2f(z.x - m) : 0.f;
  const float l = row_sum16(f * z.y);
  float x[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 0; k0 < splits; k0 += 4) {
    f32x4 y[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      y[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (n > 1 && k0 + k < n) y[k] = *reinterpret_cast<const f32x4*>(part + (k0 + k) * step * 64);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float w = __shfl(f, (k0 + k) & 15, 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] += w * y[k][j];
    }
  }
  if (n == 1) return;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
  for (int j = 0; j < 4; ++j) x[j] *= inv;
  store_row<4>(A.out, (size_t)(s.row0 + i) * A.out_stride + hd * 64 + 4 * l16, A.out_type, x);
}

struct Cuts {
  unsigned groups;
  Div heads, splits, tiles, group;
};
Cuts cuts_of(const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv4Plan& p) {
  return {(unsigned)((int64_t)R.n_seqs * P.hkv * p.tiles * p.splits), div_by(P.hkv), div_by(p.splits), div_by(p.tiles),
          div_by(A.hq / P.hkv)};
}

template <int QT>
hipError_t launch_attend(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv4Plan& p) {
  const auto kernel = p.nq == 2     ? k_kv4_attend<2, QT, 4, 1>
                      : p.nq == 4   ? k_kv4_attend<4, QT, 4, 1>
                      : p.waves == 4 ? (p.packed ? k_kv4_attend<1, QT, 4, 2> : k_kv4_attend<1, QT, 4, 1>)
                                     : (p.packed ? k_kv4_attend<1, QT, 8, 2> : k_kv4_attend<1, QT, 8, 1>);
  const Cuts c = cuts_of(P, R, A, p);
  return launch(kernel, c.groups, 64 * p.waves, 0, st, P, R, A, c.heads, c.splits, c.tiles, c.group);
}

}  // namespace

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

// A wave a (page, head).  Workgroups of one wave while each CU gets a few of them,
// or else of four heads, whose rows are neighbours (append and read: 32 tokens 6.8 us
// against 8.0, 1,024 rows 8.7 and 9.0, 2,048 rows 11.6 and 10.6, 8,192 21.7 and 20.9).
static int row_heads(const Kv4Pool& P, const Kv4Rows& R) {
  return (int64_t)R.n_seqs * row_tiles(R) * P.hkv <= 1024 ? 1 : std::min(P.hkv, 4);
}
int64_t kv4_row_threads(const Kv4Pool& P, const Kv4Rows& R) { return (int64_t)row_tiles(R) * 64 * row_heads(P, R); }
static dim3 row_grid(const Kv4Pool& P, const Kv4Rows& R, int heads) {
  return dim3((unsigned)R.n_seqs * (unsigned)row_tiles(R), (unsigned)((P.hkv + heads - 1) / heads));
}

hipError_t kv4_append(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const void* k, const void* v, int type,
                      int64_t k_stride, int64_t v_stride, RopeTable rope) {
  const int h = row_heads(P, R);
  return by_sequences(R, kv4_row_threads(P, R), [&](const Kv4Rows& r) {
    return launch(k_kv4_append, row_grid(P, r, h), 64 * h, 0, st, P, r, k, v, type, k_stride, v_stride, rope, row_tiles(r));
  });
}

hipError_t kv4_read(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, void* k, void* v, int type, int64_t k_stride,
                    int64_t v_stride) {
  const int h = row_heads(P, R);
  return by_sequences(R, kv4_row_threads(P, R), [&](const Kv4Rows& r) {
    return launch(k_kv4_read, row_grid(P, r, h), 64 * h, 0, st, P, r, k, v, type, k_stride, v_stride, row_tiles(r));
  });
}

hipError_t kv4_attend(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv4Plan& p) {
  // 16-bit queries fit one fp16 term; rotated ones are fp32 numbers.
  const bool one = A.q_type != kRowF32 && !A.rope.at;
  return by_sequences(R, p.threads, [&](const Kv4Rows& r) {
    const hipError_t e = one ? launch_attend<1>(st, P, r, A, p) : launch_attend<2>(st, P, r, A, p);
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t outs = (int64_t)r.n_seqs * r.max_rows * A.hq;
    // Five and more splits of few rows are read at once by a workgroup each (rows of 32
    // heads at 3,000, with the attention: one, 16 splits, 8.2 us, by 16 lanes each 9.8; 16,
    // 8 splits, 14.8 and 15.2); fewer splits or more rows want fewer workgroups (32 rows,
    // 8 splits, 23.5 and 23.1; 64, 2 splits, 33.6 and 31.1).
    if (p.splits > 16 || (p.splits > 4 && outs <= 512))
      return launch(k_kv4_join, (unsigned)outs, 256, 0, st, P, r, A, 16 * p.nq, p.splits);
    return launch(k_kv4_join_rows, (unsigned)((outs + 15) / 16), 256, 0, st, P, r, A, 16 * p.nq, p.splits);
  });
}

}  // namespace hh
