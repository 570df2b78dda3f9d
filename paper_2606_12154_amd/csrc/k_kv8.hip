// A paged KV cache in 8 bits: quantizing rows into pages, reading them back, and
// causal grouped-query attention over the pages or over listed ones (gfx950).
//
// Values are c * s: c an integer in -127 .. 127, s a power of two of the page's and head's
// keys, or of its values.  So a code's byte n = c + 128 behind the byte 0x64 (1024 + n as
// fp16) becomes c * s / 16 by one packed fp16 FMA, (1024 + n) t - 1152 t with t = s / 16,
// without a rounding (1152 s itself would pass fp16's range): a byte permutation
// and an FMA for two elements.  The sixteens go into the scale of the scores and out of the sums.
//
// The block of a (page, head) is laid out so that a lane's 16 bytes are what it needs
// as operands of mfma_f32_16x16x32_f16 (lane l: row or column l % 16, contraction elements
// 8 (l / 16) .. + 7), with no transposition:
//   keys    lane l holds slot l % 16, dimensions 8 (l / 16) .. + 7 of each half;
//   values  lane l holds dimensions 4 (l % 16) .. + 3, of each its slots 4 (l / 16) .. + 3.
// The scores of two pages, S^T[slot][query], leave each lane with the slots of both pages
// that its value bytes hold (see kv_attend.h for what follows).  An int8 product of 64
// dimensions takes the same key bytes as they are.
//
// Precision: weights are two fp16 terms each (22 bits), and so are queries of prompts (one term
// where 16-bit ones are not rotated); those of few columns are whole numbers of 23 bits.
//
// What bounds it.  Few columns over all keys: the loads.  32 sequences of 4,000 positions (132
// MB) take 27 us, 4.9 TB/s, the same loads alone 24: blocks of 2 KiB in no order, and the
// longest sequence, which one workgroup a kv head takes whole, is 1.4 times the mean.  Listed
// blocks of prompts: vector instructions, 106 a step of two blocks beside 14 matrix ones (85%
// of the cycles; 4,000 rows of 32 160 us, the same loads alone 96).  Prompts: both, hardly at
// once, as in the 4-bit cache's kernel (8,192 rows 488 us).  There four column tiles of queries of two
// terms take all 256 registers that two waves a SIMD leave each, and 20 bytes of scratch a lane.
#include "kv_attend.h"

#include <type_traits>

namespace hh {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ append and read

// The least e with a <= 127 * 2^e, within the format's; a is finite and not negative.
__device__ __forceinline__ int scale_exponent(float a) {
  const int e = __builtin_amdgcn_frexp_expf(a) - (__builtin_amdgcn_frexp_mantf(a) <= 127.f / 128.f ? 7 : 6);
  return a > 0.f ? min(max(e, kKv8Low), kKv8High) : kKv8Low;
}
__device__ __forceinline__ float power2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
__device__ __forceinline__ float from_half(unsigned bits) { return (float)__builtin_bit_cast(_Float16, (unsigned short)bits); }
__device__ __forceinline__ unsigned half_bits(float s) { return __builtin_bit_cast(unsigned short, (_Float16)s); }
// A held scale's exponent, whatever the bytes say.
__device__ __forceinline__ int held_exponent(unsigned bits) {
  return min(max((int)(__float_as_uint(from_half(bits & 0x7fffu)) >> 23) - 127, kKv8Low), kKv8High);
}

// Four codes as bytes c + 128, a's the lowest.
__device__ __forceinline__ unsigned bytes_of(float a, float b, float c, float d) {
  const unsigned lo = (unsigned)((int)fmaf(b, 256.f, a) + 0x8080), hi = (unsigned)((int)fmaf(d, 256.f, c) + 0x8080);
  return lo | hi << 16;
}
__device__ __forceinline__ float code_at(unsigned w, int i) { return (float)((int)(w >> (8 * i) & 255u) - 128); }
__device__ __forceinline__ float clamp127(float c) { return __builtin_amdgcn_fmed3f(c, -127.f, 127.f); }

__device__ __forceinline__ unsigned max16(unsigned x) { return max_dpp<0x128>(max_dpp<0x124>(max_dpp<0x4E>(max_dpp<0xB1>(x)))); }

// One wave has the keys, or the values, of one (page, head) of one sequence: the rows of the
// call that lie in that page, and what the page held in front of them.  The scale becomes the
// one that the largest of the new rows needs, and never less than the kept ones' own: codes that
// stay are divided by the power of two between, to nearest even, so that a value that was
// held through several such steps is off by less than one step of the last scale.
// The page is written whole: slots behind the rows hold zeros.
struct PageRows {
  Seq q;
  int page, from, to;  // the page's new slots
  unsigned char* blk;
  size_t row;  // the buffer's, of slot 0
};

__device__ __forceinline__ void put_keys(const PageRows& z, int head, const void* __restrict__ k, int type, int64_t stride, RopeTable rope) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, from = z.from;
  unsigned char* blk = z.blk;
  u32x4 old = {0u, 0u, 0u, 0u};
  unsigned old_s = 0u, old_bad = 0u;
  if (from > 0) {
    old = *reinterpret_cast<const u32x4*>(blk + 16 * lane);
    old_s = *reinterpret_cast<const unsigned short*>(blk + kKv8Scales);
    old_bad = *reinterpret_cast<const unsigned short*>(blk + kKv8Scales + 4) & ((1u << from) - 1u);
  }
  // Lane (slot r, quarter g) has whole rotation pairs (i, i + 32).
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.f;
  if (r >= from && r < z.to) {
    const size_t at = (z.row + r) * stride + head * 64 + 8 * g;
    load_row<8>(k, at, type, x);
    load_row<8>(k, at + 32, type, x + 8);
    if (rope.at) {
      const float2* cs = rope.at + (size_t)(z.page * kPage + r) * 32 + 8 * g;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float2 t = cs[i];
        const double a = x[i], b = x[8 + i], c = t.x, s = t.y;
        x[i] = (float)(a * c - b * s);
        x[8 + i] = (float)(b * c + a * s);
      }
    }
  }
  // Rows that are not finite: marked, codes of 0.
  unsigned top = 0u;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, magnitude(x[i]));
  top = rows_max(top);
  const bool bad = top >= kInfBits;
  const unsigned marks = ((unsigned)__builtin_amdgcn_ballot_w64(bad) & 0xffffu) | old_bad;
  if (bad) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
    top = 0u;
  }
  int e = scale_exponent(__uint_as_float(max16(top)));
  const int before = held_exponent(old_s);
  if (from > 0) e = max(e, before);
  const float down = power2(-e);
  float c[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) c[i] = clamp127(rintf(x[i] * down));
  if (from > 0) {
    const float shrink = power2(before - e);
#pragma unroll
    for (int i = 0; i < 16; ++i) c[i] = r < from ? clamp127(rintf(code_at(old[i >> 2], i & 3) * shrink)) : c[i];
  }
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = bytes_of(c[4 * i], c[4 * i + 1], c[4 * i + 2], c[4 * i + 3]);
  *reinterpret_cast<u32x4*>(blk + 16 * lane) = w;

  // The summary: sums of codes over the slots, a lane's 16 dimensions in pairs
  // a + 4096 b (both at most 2,032, so the pair is exact), in 8 bits.
  float high = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = row_sum16(fmaf(c[8 + i], 4096.f, c[i]));
    c[8 + i] = rintf(t * (1.f / 4096.f));
    c[i] = fmaf(c[8 + i], -4096.f, t);
    high = fmaxf(high, fmaxf(fabsf(c[i]), fabsf(c[8 + i])));
  }
  high = rows_max(high);
  const int less = (high > 127.f) + (high > 254.f) + (high > 508.f) + (high > 1016.f);
  const float part = power2(-less);
  if (r == 0) {
    unsigned* m = reinterpret_cast<unsigned*>(blk + kKv8Sums + 8 * g);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = rintf(c[8 * h + i] * part);
      *reinterpret_cast<u32x2*>(m + 8 * h) = u32x2{bytes_of(y[0], y[1], y[2], y[3]) ^ 0x80808080u,
                                                   bytes_of(y[4], y[5], y[6], y[7]) ^ 0x80808080u};
    }
  }
  if (lane == 0) {
    *reinterpret_cast<unsigned short*>(blk + kKv8Scales) = (unsigned short)half_bits(power2(e));
    *reinterpret_cast<unsigned short*>(blk + kKv8Scales + 4) = (unsigned short)marks;
    // The summary's scale, for means, and nothing behind it.
    *reinterpret_cast<u32x2*>(blk + kKv8Scales + 8) = u32x2{half_bits(power2(e + less - 4)), 0u};
  }
}

__device__ __forceinline__ void put_values(const PageRows& z, int head, const void* __restrict__ v, int type, int64_t stride) {
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4, from = z.from;
  unsigned char* blk = z.blk;
  u32x4 old = {0u, 0u, 0u, 0u};
  unsigned old_s = 0u, old_bad = 0u;
  if (from > 0) {
    old = *reinterpret_cast<const u32x4*>(blk + kKv8Values + 16 * lane);
    old_s = *reinterpret_cast<const unsigned short*>(blk + kKv8Scales + 2);
    old_bad = *reinterpret_cast<const unsigned short*>(blk + kKv8Scales + 6) & ((1u << from) - 1u);
  }
  // Lane (r, g) has slots 4 g .. + 3, dimensions 4 r .. + 3.
  float y[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * g + i;
#pragma unroll
    for (int j = 0; j < 4; ++j) y[i][j] = 0.f;
    if (slot >= from && slot < z.to) load_row<4>(v, (z.row + slot) * stride + head * 64 + 4 * r, type, y[i]);
  }
  unsigned all = 0u, marks = 0u;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned top = 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max(top, magnitude(y[i][j]));
    top = max16(top);
    if (top >= kInfBits) {
      marks |= 1u << (4 * g + i);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[i][j] = 0.f;
      top = 0u;
    }
    all = max(all, top);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) old_bad |= (unsigned)__builtin_amdgcn_readlane((int)marks, 16 * i);
  int e = scale_exponent(__uint_as_float(rows_max(all)));
  const int before = held_exponent(old_s);
  if (from > 0) e = max(e, before);
  const float down = power2(-e), shrink = power2(before - e);
  u32x4 w;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = clamp127(rintf(y[i][j] * down));
    if (from > 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) c[i] = 4 * g + i < from ? clamp127(rintf(code_at(old[j], i) * shrink)) : c[i];
    }
    w[j] = bytes_of(c[0], c[1], c[2], c[3]);
  }
  *reinterpret_cast<u32x4*>(blk + kKv8Values + 16 * lane) = w;
  if (lane == 0) {
    *reinterpret_cast<unsigned short*>(blk + kKv8Scales + 2) = (unsigned short)half_bits(power2(e));
    *reinterpret_cast<unsigned short*>(blk + kKv8Scales + 6) = (unsigned short)old_bad;
  }
}

__global__ __launch_bounds__(256) void k_kv8_append(Kv4Pool P, Kv4Rows R, const void* __restrict__ k,
                                                    const void* __restrict__ v, int type, int64_t ks, int64_t vs,
                                                    RopeTable rope, int tiles) {
  const int head = blockIdx.y * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (head >= P.hkv) return;
  const unsigned sq = blockIdx.x / (unsigned)tiles;
  const int tile = blockIdx.x - sq * tiles;
  PageRows z;
  z.q = load_seq(P, R, R.seq0 + sq);
  const int lo = max(z.q.first, 0);
  int hi = min(z.q.first + z.q.n, P.max_pages * kPage);
  if (rope.at) hi = min(hi, rope.len);
  z.page = lo / kPage + tile;
  // (page * kPage may pass 31 bits.)  Without rows the page stays as it is.
  if (lo >= hi || z.page >= (hi + kPage - 1) >> 4) return;
  const int id = P.table[(size_t)z.q.trow * P.max_pages + z.page];
  if ((unsigned)id >= (unsigned)P.n_pages) return;
  z.blk = P.pool + ((size_t)id * P.hkv + head) * kKv8Block;
  z.from = max(lo - z.page * kPage, 0);
  z.to = min(hi - z.page * kPage, kPage);
  z.row = (size_t)((int64_t)z.q.row0 + z.page * kPage - z.q.first);  // (that of slot `from` on is in the buffer)
  if (blockIdx.z == 0)
    put_keys(z, head, k, type, ks, rope);
  else
    put_values(z, head, v, type, vs);
}

// The same lanes the other way round.  Tiles are counted from the page of the
// first position, which may be negative: such rows, and those past the page
// table, are set to zero.
__global__ __launch_bounds__(256) void k_kv8_read(Kv4Pool P, Kv4Rows R, void* __restrict__ k, void* __restrict__ v,
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
  const unsigned id = (unsigned)P.table[(size_t)q.trow * P.max_pages + (held ? page : 0)];
  // An id outside the pool reads its first page.
  const unsigned char* blk = P.pool + ((size_t)(id < (unsigned)P.n_pages ? id : 0u) * P.hkv + head) * kKv8Block;
  const int r = lane & 15, g = lane >> 4;
  const u32x4 kw = *reinterpret_cast<const u32x4*>(blk + 16 * lane);
  const u32x4 vw = *reinterpret_cast<const u32x4*>(blk + kKv8Values + 16 * lane);
  const u32x2 sc = *reinterpret_cast<const u32x2*>(blk + kKv8Scales);
  const unsigned bad = sc[1];
  const float k_scale = from_half(sc[0] & 0xffffu), v_scale = from_half(sc[0] >> 16);

  {
    const int pos = page * kPage + r;
    if (pos >= q.first && pos < hi) {
      const float s = bad >> r & 1u ? NAN : k_scale;
      const size_t at = (size_t)(q.row0 + (pos - q.first)) * ks + head * 64 + 8 * g;
      float x[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = held ? code_at(kw[i >> 2], i & 3) * s : 0.f;
      store_row<8>(k, at, type, x);
      store_row<8>(k, at + 32, type, x + 8);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int slot = 4 * g + i, pos = page * kPage + slot;
    if (pos < q.first || pos >= hi) continue;
    const float s = bad >> (16 + slot) & 1u ? NAN : v_scale;
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = held ? code_at(vw[j], i) * s : 0.f;
    store_row<4>(v, (size_t)(q.row0 + (pos - q.first)) * vs + head * 64 + 4 * r, type, x);
  }
}

// ------------------------------------------------------------------ attention

struct PageRegs {
  u32x4 k, v;
  u32x2 s;  // scales, marks
};

// The block as a buffer: its base stays in scalar registers, a lane's offset in one
// vector register; its scales are the wave's, read by the scalar unit (by vector loads, with
// 8 more registers, the longest prompt 493 -> 516, 131,072 positions 30.0 -> 33.1).  ONCE:
// no other workgroup reads the block, whose lines then stay out of the caches' way (32
// sequences of 4,000 positions 31.5 -> 27.9 us, one of 131,072 33.4 -> 31.1; but the longest
// prompt 501 -> 509).
template <bool ONCE>
__device__ __forceinline__ void load_page(PageRegs& r, const unsigned char* blk, unsigned lane) {
  constexpr int AUX = ONCE ? 2 : 0;
  const auto b = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(blk), 0, kKv8Block, 0x00027000);
  r.k = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, 16 * lane, 0, AUX));
  r.v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(b, 16 * lane + kKv8Values, 0, AUX));
  r.s = *reinterpret_cast<const __attribute__((address_space(4))) u32x2*>(
      reinterpret_cast<uintptr_t>(blk + kKv8Scales));
}

// Bytes 2 J and 2 J + 1 of w as 1024 + n.
template <int J>
__device__ __forceinline__ f16x2 codes16(unsigned w) {
  return __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, J ? 0x04030402u : 0x04010400u));
}
// A scale's sixteenth and -1152 times that, each twice.
struct Scale {
  f16x2 s, b;
};
__device__ __forceinline__ Scale scale_of(unsigned both) {
  Scale z;
  z.s = __builtin_bit_cast(f16x2, both) * f16x2{(_Float16)0.0625f, (_Float16)0.0625f};
  z.b = z.s * f16x2{(_Float16)-1152, (_Float16)-1152};
  return z;
}
__device__ __forceinline__ f16x4 four(unsigned w, Scale z) {
  const f16x2 lo = __builtin_elementwise_fma(codes16<0>(w), z.s, z.b), hi = __builtin_elementwise_fma(codes16<1>(w), z.s, z.b);
  return f16x4{lo[0], lo[1], hi[0], hi[1]};
}

// A page's operands: keys of each half, and the values of each dimension of four.
// Without MASK every column sees every slot, so that a page with a marked one makes all
// of them NaN; with it the marks go through the scores, to the rows that see them.
template <bool MASK>
__device__ __forceinline__ void operands(const PageRegs& p, f16x8* kf, f16x4* vf) {
  unsigned sk = __builtin_amdgcn_perm(p.s[0], p.s[0], 0x01000100u), sv = __builtin_amdgcn_perm(p.s[0], p.s[0], 0x03020302u);
  if constexpr (!MASK)
    if (p.s[1]) sk = 0x7e007e00u;
  const Scale a = scale_of(sk), b = scale_of(sv);
  kf[0] = join8(four(p.k[0], a), four(p.k[1], a));
  kf[1] = join8(four(p.k[2], a), four(p.k[3], a));
#pragma unroll
  for (int j = 0; j < 4; ++j) vf[j] = four(p.v[j], b);
}

constexpr int kNowhere = 1 << 30;  // a listed block that is none: behind every column's keys

// ---- few columns: a token's query heads, or a row's that lists its blocks
//
// A tile of 16 columns holds 16 / P query heads P times, side by side (P: 2 for up to 8 heads
// a kv head).  Copy i has its queries in page i's product and zeros in the other's, so that a lane's
// four scores of a step of two pages are of both, not of one and half of them of no column.
//
// Scores are products of whole numbers: a query in three signed digits of 8 bits (23 bits of
// its largest element: a score is off by 2^-16 of the largest |q| times the block's largest |k| at
// most, where a code's own rounding, half a step of |k| / 127, is worth 2^-8 of that in the largest
// |q|'s dimension alone; a fourth digit took 28.8 us for 26.6 at 32 tokens of 4,000 positions, 33.0 for
// 28.9 at one of 131,072) times the page's codes as they lie, mfma_i32_16x16x64_i8; three
// conversions and two FMAs a score take the place of unpacking the keys (4,000 prompt rows of 32
// listed blocks 177 -> 164 us, 64 sequences of 1,500 positions 22.7 -> 21.7; 16-bit queries
// that need one term and no scaling lose 0.4 us at the start).  P = 4 takes fewer exponentials
// a page, but 165 to 195 registers (170 and 25.6).
// Where a query's factor would be less than 2^-100, scores are below 2^-56, and all weights 1.
constexpr float kLeastFactor = 0x1p-100f;

template <int P>
__device__ __forceinline__ int copy_of() { return (threadIdx.x & 15) / (16 / P); }

struct Digits {
  i32x4 d[3];
};
__device__ __forceinline__ i32x4 no_digits() { return i32x4{0, 0, 0, 0}; }
// The lane's 16 dimensions as digits, and the power of two that scores take.
__device__ __forceinline__ float make_digits(const RawQuery& q, const Kv4Attend& A, Digits& z) {
  float x[16];
  raw_values(q.row, A.q_type, x);
  if (A.rope.at) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float u = x[i], v = x[8 + i], co = q.turn[i >> 1][2 * (i & 1)], si = q.turn[i >> 1][2 * (i & 1) + 1];
      x[i] = u * co - v * si;
      x[8 + i] = v * co + u * si;
    }
  }
  // The scores' factor to powers of two, but for a power of two itself, goes into the query: then
  // a whole number times what is left is exact, and equal scores stay equal whatever their base.
  const float to_powers = A.scale * (1.4426950408889634f / 16.f), part = __builtin_amdgcn_frexp_mantf(to_powers);
  unsigned top = 0u;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = max(top, magnitude(x[i]));
  top = rows_max(top);
  // The largest becomes a number from 2^21 to 2^22.
  const int e = top > 0u && top < kInfBits ? 22 - __builtin_amdgcn_frexp_expf(__uint_as_float(top) * part) : 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    unsigned y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      y[i] = ((unsigned)(int)rintf(__builtin_amdgcn_ldexpf(top < kInfBits ? x[4 * w + i] : 0.f, e) * part) + 0x808080u) ^ 0x808080u;
    const unsigned a = __builtin_amdgcn_perm(y[1], y[0], 0x05010400u), b = __builtin_amdgcn_perm(y[3], y[2], 0x05010400u);
    const unsigned c = __builtin_amdgcn_perm(y[1], y[0], 0x0c0c0602u), d = __builtin_amdgcn_perm(y[3], y[2], 0x0c0c0602u);
    z.d[0][w] = (int)__builtin_amdgcn_perm(b, a, 0x05040100u);
    z.d[1][w] = (int)__builtin_amdgcn_perm(b, a, 0x07060302u);
    z.d[2][w] = (int)__builtin_amdgcn_perm(d, c, 0x05040100u);
  }
  // (A query that is not finite makes every score NaN.)
  const float f = __builtin_amdgcn_ldexpf(1.f, __builtin_amdgcn_frexp_expf(to_powers) - e);
  return top < kInfBits ? __builtin_amdgcn_fmed3f(f, kLeastFactor, kMostFactor) : NAN;
}

// A wave's columns: their queries, bases, sums (of a lane's own slots) and outputs.
template <int P>
struct Few {
  static constexpr int N = 8 / P;  // scores of a lane and step of two pages
  struct Places {
    int v[2];
  };
  Digits q[P];
  float qs, base, sum;
  float limit;  // scores above it raise the base
  int lim;  // keys that the column sees
  f32x4 o[4];
  bool fresh;      // the column has seen no key yet
  bool any_fresh;  // one of the wave's may not have

  __device__ __forceinline__ void start(const Place& w, int most, const RawQuery& raw, const Kv4Attend& A) {
    Digits z;
    qs = make_digits(raw, A, z);
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int j = 0; j < 3; ++j) q[i].d[j] = P == 1 || copy_of<P>() == i ? z.d[j] : no_digits();
    base = sum = limit = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    lim = min(max(w.s.first + column_row(w, w.c0 + column_of<P>()) + 1, 0), most);
    fresh = any_fresh = true;
  }

  // Two pages, from positions `at` on.  MASK: slots past a column's keys, and marked ones.
  template <bool MASK>
  __device__ __forceinline__ void step(const PageRegs (&x)[2], const Places& at) {
    const int g = (threadIdx.x & 63) >> 4, side = copy_of<P>();
    float scale[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // (Marks as in operands.  Where a block is none, whatever is read in its place may have any scale.)
      const unsigned held = MASK && at.v[i] == kNowhere ? 0u : x[i].s[0];
      const unsigned s = !MASK && x[i].s[1] ? 0x7e00u : held & 0xffffu;
      scale[i] = qs * from_half(s);
    }
    i32x4 acc[P == 1 ? 2 : 1][3];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u32x4 codes = x[i].k ^ 0x80808080u;
      const i32x4 a = __builtin_bit_cast(i32x4, codes);
#pragma unroll
      for (int j = 0; j < 3; ++j) {
        i32x4& y = acc[P == 1 ? i : 0][j];
        y = __builtin_amdgcn_mfma_i32_16x16x64_i8(a, q[P == 1 ? 0 : i].d[j], P == 1 || i == 0 ? no_digits() : y, 0, 0, 0);
      }
    }
    const float mine = P == 2 && side ? scale[1] : scale[0];
    // Scores as whole numbers, and the largest of those that are neither hidden nor marked.
    // Weights are taken against the base that it leaves (see base_for).
    float s[N], high = -INFINITY;
    bool hidden[N], marked[N];
    if constexpr (MASK) {
      unsigned bad[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) bad[i] = x[i].s[1] | x[i].s[1] >> 16;
      const unsigned of = P == 2 && side ? bad[1] : bad[0];
      const int from = P == 2 && side ? at.v[1] : at.v[0];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        marked[i] = (P == 1 ? bad[i >> 2] : of) >> (4 * g + (i & 3)) & 1u;
        hidden[i] = (P == 1 ? at.v[i >> 2] : from) + 4 * g + (i & 3) >= lim;
      }
    }
#pragma unroll
    for (int u = 0; u < N / 4; ++u) {
      const i32x4* y = acc[u];
      float most = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = 4 * u + j;
        s[i] = fmaf((float)y[2][j], 65536.f, fmaf((float)y[1][j], 256.f, (float)y[0][j]));
        most = fmaxf(most, MASK && (hidden[i] || marked[i]) ? -INFINITY : s[i]);
      }
      high = u ? fmaxf(high, most * scale[u]) : most * (P == 1 ? scale[0] : mine);
    }
    if (any_fresh || __builtin_amdgcn_ballot_w64(high > limit)) {
      const float mx = rows_max(fmaxf(high, -INFINITY));  // (NaN, of what is not finite, counts as none)
      float to = mx > -INFINITY ? base_for(mx) : base;
      if (!fresh) to = fmaxf(to, base);
      const float f = fresh ? 1.f : __builtin_amdgcn_exp2f(base - to);
      base = to;
      limit = fabsf(base) < kLarge ? base + (kOffset + kSlack) : base;
      sum *= f;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] *= f;
      fresh = fresh && !(mx > -INFINITY);
      any_fresh = __builtin_amdgcn_ballot_w64(fresh);
    }
    float sc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sc[i] = fmaf(s[i], P == 1 ? scale[i >> 2] : mine, -base);
    if constexpr (MASK) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (marked[i]) sc[i] = NAN;
        if (hidden[i]) sc[i] = -INFINITY;
      }
    }
    f16x2 h[N / 2], l[N / 2];
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      const float a = __builtin_amdgcn_exp2f(sc[i]), b = __builtin_amdgcn_exp2f(sc[i + 1]);
      sum += a + b;
      split_weights(a, b, h[i / 2], l[i / 2]);
    }
    // A lane's weights where their page's values are.
    auto weights = [&](const f16x2* y) {
      const f16x4 z = {y[0][0], y[0][1], y[1][0], y[1][1]}, none = {0, 0, 0, 0};
      if constexpr (P == 1) return join8(z, f16x4{y[2][0], y[2][1], y[3][0], y[3][1]});
      return join8(side ? none : z, side ? z : none);
    };
    const f16x8 ph = weights(h), pl = weights(l);
    Scale vs[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned s = MASK && at.v[i] == kNowhere ? 0u : x[i].s[0];
      vs[i] = scale_of(__builtin_amdgcn_perm(s, s, 0x03020302u));
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const f16x8 v = join8(four(x[0].v[d], vs[0]), four(x[1].v[d], vs[1]));
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, pl, o[d], 0, 0, 0);
      o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, ph, o[d], 0, 0, 0);
    }
  }
};

// Copies of a column side by side (16 / P lanes apart), joined.
template <int P, int N>
__device__ __forceinline__ void join_copies(float& m, float& l, float (&x)[N]) {
  if constexpr (P == 1) return;
  const float top = fmaxf(m, other8(m)), f = m > -INFINITY ? __builtin_amdgcn_exp2f(m - top) : 0.f;
  m = top;
  l = f * l + other8(f * l);
#pragma unroll
  for (int j = 0; j < N; ++j) x[j] = f * x[j] + other8(f * x[j]);
}

// A workgroup has a sequence's columns of one kv head (LIST: a row's, or 16 of them); its W
// waves take the pages (the listed blocks) in turn, NP a step, and join at the end.
template <int P, int W, bool LIST, bool ONCE>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(4))) void
k_kv8_few(Kv4Pool Q, Kv4Rows R, Kv4Attend A, Kv8List B, Div heads, Div splits_, Div tiles_, Div group, Div row_tiles_) {
  constexpr int NP = 2, STEP = NP * W;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const unsigned b1 = blockIdx.x / heads, b2 = b1 / splits_, sq = b2 / tiles_;
  const int split = b1 - b2 * splits_.d, splits = splits_.d;
  const int tile = b2 - sq * tiles_.d;
  const Seq s = load_seq(Q, R, R.seq0 + sq);
  const int G = group.d, own = LIST ? (unsigned)tile / row_tiles_ : 0;  // LIST: the row
  if (LIST && own >= s.n) return;
  const int cols = LIST ? (own + 1) * G : s.n * G;
  const Place w{s, (int)(blockIdx.x - b1 * heads.d), G, cols, LIST ? own * G + 16 * (tile - own * (int)row_tiles_.d) : 0, group};
  if (w.c0 >= cols) return;
  // Keys of the first and last row.
  const int most = Q.max_pages * kPage;
  const int row_b = (unsigned)(min(w.c0 + 16, cols) - 1) / group;
  const int all_see = min(max(s.first + (LIST ? row_b : 0) + 1, 0), most), some_see = min(max(s.first + row_b + 1, 0), most);
  const int np = LIST ? B.n : (some_see + kPage - 1) / kPage;
  const int per = split_pages(np, splits);
  const int p0 = split * per, p1 = min(p0 + per, np);
  const bool joined = per < np;  // several splits have keys
  if (split > 0 && p0 >= np) return;

  // What the first step needs goes out before the queries are worked on.  Loads run one
  // step ahead; what would lie behind the wave's last step is its last step again (no branch
  // around loads, whose waits would then have to assume that it was not taken).  Lane i holds
  // the page ids of the i-th of 64 steps.
  const int* row = Q.table + (size_t)s.trow * Q.max_pages;
  const int* list = LIST ? B.blocks + ((size_t)(s.row0 + own) * Q.hkv + w.head) * B.n : nullptr;
  int p = p0 + NP * wave;
  const int last = max(p + (p1 - 1 - p) / STEP * STEP, 0);
  unsigned ids[NP];
  int at[NP];                   // LIST: the blocks' first positions
  uint64_t full = 0, part = 0;  // LIST: steps that the row sees whole, other ones with a block
  auto load_ids = [&](int q) {
    const int from = LIST ? q + lane * STEP : min(q + lane * STEP, last);
    int low = kNowhere, high = 0;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      int page = max(min(from + i, np - 1), 0);
      if constexpr (LIST) {
        const int b = list[page];
        const bool in = from + i < p1 && b >= 0 && b <= (some_see - 1) >> 4;
        at[i] = in ? b * kPage : kNowhere;
        page = in ? b : 0;
        low = min(low, at[i]);
        high = max(high, at[i]);
      }
      const unsigned x = (unsigned)row[page];
      ids[i] = x < (unsigned)Q.n_pages ? x : 0u;  // an id outside the pool reads its first page
    }
    if constexpr (LIST) {
      full = __builtin_amdgcn_ballot_w64(high + kPage <= some_see);
      part = __builtin_amdgcn_ballot_w64(low < kNowhere) & ~full;
    }
  };
  int ahead = 0;  // the step that is fetched next
  auto fetch = [&](PageRegs* x) {
    if constexpr (LIST) {
      // First the steps that the row sees whole.  (Behind the last one any other is fetched.)
      uint64_t& of = full ? full : part;
      ahead = of ? __builtin_ctzll(of) : 0;
      of &= of - 1;
    } else if (ahead == 64) {
      load_ids(p + STEP);
      ahead = 0;
    }
#pragma unroll
    for (int j = 0; j < NP; ++j) {
      const unsigned id = (unsigned)__builtin_amdgcn_readlane((int)ids[j], ahead);
      load_page<ONCE>(x[j], Q.pool + ((size_t)id * (unsigned)Q.hkv + (unsigned)w.head) * kKv8Block, (unsigned)lane);
    }
    if constexpr (!LIST) ++ahead;
  };
  load_ids(p);
  RawQuery raw;
  load_query<2, P>(raw, w, A, 0);
  PageRegs a[NP], c[NP];
  int n_full = __builtin_popcountll(full), n_part = __builtin_popcountll(part);
  fetch(a);
  Few<P> C;
  C.start(w, most, raw, A);
  auto to_a = [&] {
#pragma unroll
    for (int i = 0; i < NP; ++i) a[i] = c[i];
  };
  if constexpr (LIST) {
    while (true) {
      bool swapped = false;
      while (n_full > 0) {
        fetch(c);
        C.template step<false>(a, {});
        if (--n_full == 0) {
          swapped = true;
          break;
        }
        fetch(a);
        C.template step<false>(c, {});
        --n_full;
      }
      if (swapped) to_a();
      for (; n_part > 0; --n_part) {
        typename Few<P>::Places from;
#pragma unroll
        for (int i = 0; i < NP; ++i) from.v[i] = __builtin_amdgcn_readlane(at[i], ahead);
        fetch(c);
        C.template step<true>(a, from);
        to_a();
      }
      p += 64 * STEP;
      if (p >= p1) break;
      load_ids(p);
      n_full = __builtin_popcountll(full);
      n_part = __builtin_popcountll(part);
      fetch(a);
    }
  } else {
    const int whole = min(all_see / kPage, p1);  // pages below are seen by every row
    bool swapped = false;
    while (p + NP <= whole) {
      fetch(c);
      C.template step<false>(a, {});
      p += STEP;
      if (p + NP > whole) {
        swapped = true;
        break;
      }
      fetch(a);
      C.template step<false>(c, {});
      p += STEP;
    }
    if (swapped) to_a();
    while (p < p1) {
      typename Few<P>::Places from;
#pragma unroll
      for (int i = 0; i < NP; ++i) from.v[i] = p + i < p1 ? (p + i) * kPage : kNowhere;
      fetch(c);
      C.template step<true>(a, from);
      to_a();
      p += STEP;
    }
  }

  const float total = rows_sum(C.sum), base = total == 0.f ? -INFINITY : C.base;  // (no key, no base)
  const bool writes = P == 1 || copy_of<P>() == 0;
  // Without neighbours a lane writes its 16 dimensions from 16 g on.
  if constexpr (W == 1) {
    float m = base, l = total, x[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 16.f * C.o[i & 3][i >> 2];  // (16: of the values' scale)
    join_copies<P>(m, l, x);
    if (writes) put<16>(R, A, w, w.c0 + r, 16 * g, x, l, m, joined, split, splits);
    return;
  }
  // Join the waves: wave v takes dimensions 16 g + 4 v .. + 3, of two waves v + 2 too.
  __shared__ f32x4 lo[W][4][64];
  __shared__ float2 ls[W][64];
#pragma unroll
  for (int i = 0; i < 4; ++i) lo[wave][i][lane] = f32x4{C.o[0][i], C.o[1][i], C.o[2][i], C.o[3][i]};
  ls[wave][lane] = make_float2(base, total);
  __syncthreads();
  float top = -INFINITY;
#pragma unroll
  for (int v = 0; v < W; ++v) top = fmaxf(top, ls[v][lane].x);
  for (int part4 = wave; part4 < 4; part4 += W) {
    float m = top, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float2 z = ls[v][lane];
      const float f = z.x > -INFINITY ? 16.f * __builtin_amdgcn_exp2f(z.x - m) : 0.f;  // (as above)
      const f32x4 y = lo[v][part4][lane];
      l += f * z.y;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] += f * y[j];
    }
    l *= 0.0625f;
    join_copies<P>(m, l, x);
    if (writes) put<4>(R, A, w, w.c0 + r, 16 * g + 4 * part4, x, l, m, joined, split, splits);
  }
}

// ---- many columns: prompts
//
// A workgroup has a tile of 16 NQ columns; its four waves take the tile's pages in turn, two a
// step, and join at the end.
template <int NQ, int QT>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(waves_fit(NQ)))) void
k_kv8_attend(Kv4Pool P, Kv4Rows R, Kv4Attend A, Div heads, Div splits_, Div tiles_, Div group) {
  constexpr int W = 4;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, g = lane >> 4;
  const unsigned b1 = blockIdx.x / heads, b2 = b1 / splits_, sq = b2 / tiles_;
  const int split = b1 - b2 * splits_.d, splits = splits_.d;
  // The last tiles have the most keys: they go first.
  const int tile = tiles_.d - 1 - (b2 - sq * tiles_.d);
  const Seq s = load_seq(P, R, R.seq0 + sq);
  const int G = group.d, cols = s.n * G;  // below 2^31 with a tile to spare (kv8_plan)
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

  // (Loads and page ids as above.)
  const int* row = P.table + (size_t)s.trow * P.max_pages;
  constexpr int STEP = 2 * W;
  int p = p0 + 2 * wave;
  const int from = p < p1 ? p * kPage : INT_MAX - kPage;
  const int last = max(p + (p1 - 1 - p) / STEP * STEP, 0);
  unsigned ids[2];
  auto load_ids = [&](int q) {
    const int from = min(q + lane * STEP, last);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned x = (unsigned)row[max(min(from + i, np - 1), 0)];
      ids[i] = x < (unsigned)P.n_pages ? x : 0u;  // an id outside the pool reads its first page
    }
  };
  int ahead = 0;  // the step that is fetched next
  auto fetch = [&](PageRegs* x) {
    if (ahead == 64) {
      load_ids(p + STEP);
      ahead = 0;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned id = (unsigned)__builtin_amdgcn_readlane((int)ids[i], ahead);
      load_page<false>(x[i], P.pool + ((size_t)id * (unsigned)P.hkv + (unsigned)w.head) * kKv8Block, (unsigned)lane);
    }
    ++ahead;
  };
  load_ids(p);
  // Of several tiles, each wave makes one's queries for all.
  RawQuery raw;
  if (NQ == 1 || wave < NQ) load_query<QT, 1>(raw, w, A, NQ == 1 ? 0 : wave);
  PageRegs a[2], c[2];
  fetch(a);
  Columns<NQ, QT, 1> C;
  C.start(w, most);
  if constexpr (NQ == 1) {
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

  auto step = [&](const PageRegs* x, auto masked) {
    constexpr bool MASK = decltype(masked)::value;
    f16x8 kf[2][2], vf[4];
    f16x4 va[4], vb[4];
    operands<MASK>(x[0], kf[0], va);
    operands<MASK>(x[1], kf[1], vb);
#pragma unroll
    for (int j = 0; j < 4; ++j) vf[j] = join8(va[j], vb[j]);
    unsigned bad[2] = {0u, 0u};
    if constexpr (MASK) {
#pragma unroll
      for (int i = 0; i < 2; ++i) bad[i] = (x[i].s[1] | x[i].s[1] >> 16) >> (4 * g) & 15u;
    }
    f32x4 sc[NQ][2];
    f16x8 ph[NQ], pl[NQ];
    C.scores(kf, sc);
    C.template weights<MASK>(sc, p * kPage, (p + 1) * kPage, bad[0] | bad[1] << 4, ph, pl);
    C.values(vf, ph, pl);
  };
  const int whole = min(all_see / kPage & ~1, p1 & ~1);  // pages below are seen by every row
  bool swapped = false;
  while (p < whole) {
    fetch(c);
    step(a, std::false_type());
    p += STEP;
    if (p >= whole) {
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

  C.finish(from);

  // Join the waves: wave v takes dimensions 16 g + 4 v .. + 3.
  __shared__ f32x4 lo[W][4][64];
  __shared__ float2 ls[W][64];
#pragma unroll
  for (int t = 0; t < NQ; ++t) {
    if (t) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) lo[wave][i][lane] = f32x4{C.o[t][0][i], C.o[t][1][i], C.o[t][2][i], C.o[t][3][i]};
    ls[wave][lane] = make_float2(C.base_of(t), C.sum[t][0]);
    __syncthreads();
    float m = -INFINITY, l = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < W; ++v) m = fmaxf(m, ls[v][lane].x);
#pragma unroll
    for (int v = 0; v < W; ++v) {
      const float2 z = ls[v][lane];
      const float f = z.x > -INFINITY ? 16.f * __builtin_amdgcn_exp2f(z.x - m) : 0.f;  // (16: of the values' scale)
      const f32x4 y = lo[v][wave][lane];
      l += f * z.y;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] += f * y[j];
    }
    put<4>(R, A, w, w.c0 + 16 * t + r, 16 * g + 4 * wave, x, l * 0.0625f, m, joined, split, splits);
  }
}

typedef void (*FewKernel)(Kv4Pool, Kv4Rows, Kv4Attend, Kv8List, Div, Div, Div, Div, Div);
template <int W, bool LIST>
FewKernel pick_few(int columns) {
  return columns <= 8 ? k_kv8_few<2, W, LIST, !LIST> : k_kv8_few<1, W, LIST, !LIST>;
}
template <int QT>
hipError_t launch_prompt(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv8Plan& p, unsigned groups) {
  const auto kernel = p.nq == 1 ? k_kv8_attend<1, QT> : p.nq == 2 ? k_kv8_attend<2, QT> : k_kv8_attend<4, QT>;
  return launch(kernel, groups, 256, 0, st, P, R, A, div_by(P.hkv), div_by(p.splits), div_by(p.tiles), div_by(A.hq / P.hkv));
}

// Waves a (page, head), as in the 4-bit cache's calls: workgroups of one head while each CU
// gets a few of them, or else of four, whose rows are neighbours (8,192 rows appended and
// read 23.0 us; of one head 22.7, two 22.4, eight 23.0).  A wave of its own for the keys and one
// for the values: 32 tokens 9.3 -> 8.1 us, 8,192 rows 24.1 -> 23.1.
int row_heads(const Kv4Pool& P, const Kv4Rows& R) {
  return (int64_t)R.n_seqs * row_tiles(R) * P.hkv <= 1024 ? 1 : std::min(P.hkv, 4);
}
dim3 row_grid(const Kv4Pool& P, const Kv4Rows& R, int heads) {
  return dim3((unsigned)R.n_seqs * (unsigned)row_tiles(R), (unsigned)((P.hkv + heads - 1) / heads));
}

}  // namespace

int64_t kv8_row_threads(const Kv4Pool& P, const Kv4Rows& R) { return (int64_t)row_tiles(R) * 64 * row_heads(P, R); }

hipError_t kv8_append(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const void* k, const void* v, int type,
                      int64_t k_stride, int64_t v_stride, RopeTable rope) {
  const int h = row_heads(P, R);
  return by_sequences(R, kv8_row_threads(P, R), [&](const Kv4Rows& r) {
    dim3 grid = row_grid(P, r, h);
    grid.z = 2;  // keys, and values
    return launch(k_kv8_append, grid, 64 * h, 0, st, P, r, k, v, type, k_stride, v_stride, rope, row_tiles(r));
  });
}

hipError_t kv8_read(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, void* k, void* v, int type, int64_t k_stride,
                    int64_t v_stride) {
  const int h = row_heads(P, R);
  return by_sequences(R, kv8_row_threads(P, R), [&](const Kv4Rows& r) {
    return launch(k_kv8_read, row_grid(P, r, h), 64 * h, 0, st, P, r, k, v, type, k_stride, v_stride, row_tiles(r));
  });
}

hipError_t kv8_attend(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv8Plan& p) {
  // 16-bit queries fit one fp16 term; rotated ones are fp32 numbers.
  const bool one = A.q_type != kRowF32 && !A.rope.at;
  const int group = A.hq / P.hkv;
  return by_sequences(R, p.threads, [&](const Kv4Rows& r) {
    const unsigned groups = (unsigned)((int64_t)r.n_seqs * P.hkv * p.tiles * p.splits);
    hipError_t e;
    if (p.tiles == 1 && p.nq == 1)
      e = launch(p.waves == 4 ? pick_few<4, false>(r.max_rows * group) : pick_few<8, false>(r.max_rows * group), groups,
                 64 * p.waves, 0, st, P, r, A, Kv8List{nullptr, 0}, div_by(P.hkv), div_by(p.splits), div_by(1), div_by(group), div_by(1));
    else
      e = one ? launch_prompt<1>(st, P, r, A, p, groups) : launch_prompt<2>(st, P, r, A, p, groups);
    return e != hipSuccess || p.splits == 1 ? e : launch_join(st, P, r, A, 16 * p.nq, p.splits, 0);
  });
}

hipError_t kv8_attend_list(hipStream_t st, const Kv4Pool& P, const Kv4Rows& R, const Kv4Attend& A, const Kv8List& B,
                           const Kv8ListPlan& p) {
  const int group = A.hq / P.hkv, tiles = R.max_rows * p.tiles;
  const int per = 2 * (((B.n + 1) / 2 + p.splits - 1) / p.splits), used = (B.n + per - 1) / per;
  const auto kernel = p.waves == 1   ? pick_few<1, true>(group)
                      : p.waves == 2 ? pick_few<2, true>(group)
                      : p.waves == 4 ? pick_few<4, true>(group)
                                     : pick_few<8, true>(group);
  return by_sequences(R, p.threads, [&](const Kv4Rows& r) {
    const unsigned groups = (unsigned)((int64_t)r.n_seqs * P.hkv * tiles * p.splits);
    const hipError_t e = launch(kernel, groups, 64 * p.waves, 0, st, P, r, A, B, div_by(P.hkv), div_by(p.splits), div_by(tiles),
                                div_by(group), div_by(p.tiles));
    return e != hipSuccess || used == 1 ? e : launch_join(st, P, r, A, 16, p.splits, used);
  });
}

}  // namespace hh
