// What the gradient kernels on the bf16 matrix cores share: operands and accumulators of 32x32x16 products, rows and
// tiles in LDS and their transposing reads.
//
// Layouts.  A lane of a 32x32 accumulator holds 16 values of one column, rows 8 (r / 4) + 4 hf + r % 4 (hf = lane / 32); an
// operand holds 8 values of one row (A) or column (B) for each slice of 16 of the contraction, and any order of these is
// fine as long as both operands use it.  So an accumulator, rounded and packed, is an operand over its rows.
#pragma once

#include "common.hpp"
#include "grad.hpp"

namespace vista {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;

namespace {

// f(0), ..., f(N - 1) with constants: register arrays keep to registers whatever the body's size.
template <int V>
struct Int { static constexpr int value = V; };
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each(F f) {
  if constexpr (I < N) {
    f(Int<I>{});
    each<N, I + 1>(f);
  }
}

union Pack8 {
  bf16x8 v;
  u32x4 u;
  u32x2 d[2];
  uint32_t w[4];
};

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// An accumulator as two operands over its rows.
__device__ __forceinline__ void pack(const f32x16& v, bf16x8 (&out)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    Pack8 p;
#pragma unroll
    for (int i = 0; i < 4; ++i) p.w[i] = pair_to_bf16(v[8 * t + 2 * i], v[8 * t + 2 * i + 1]);
    out[t] = p.v;
  }
}
// The same in two terms: hi + lo has 16 bits.
__device__ __forceinline__ void pack2(const f32x16& v, bf16x8 (&hi)[2], bf16x8 (&lo)[2]) {
  pack(v, hi);
  f32x16 rest;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    Pack8 p;
    p.v = hi[r / 8];
    const uint32_t w = p.w[r % 8 / 2];
    rest[r] = v[r] - __uint_as_float(r % 2 ? w & 0xFFFF0000u : w << 16);
  }
  pack(rest, lo);
}

// LDS by address.  A lane's addresses are formed once and kept opaque, so that the blocks of an unrolled loop differ by the
// instruction's own offset and not by a register each.
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const char*)(p)));
}
__device__ __forceinline__ uint32_t kept(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}
template <typename T>
__device__ __forceinline__ T lds_read(uint32_t at) {
  return *(__attribute__((address_space(3))) const T*)(uintptr_t(at));
}
template <typename T>
__device__ __forceinline__ void lds_write(uint32_t at, const T& v) {
  *(__attribute__((address_space(3))) T*)(uintptr_t(at)) = v;
}
// Transposing read of four rows x 16 columns by 16 lanes: lane i gives the address of row i / 4, columns 4 (i % 4), and
// receives column i, the four rows in its registers.
__device__ __forceinline__ u32x2 read_turned(uint32_t at) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(uintptr_t(at))));
}

// Rows of 32 bf16 (64 bytes) in LDS.  Chunk c of 16 bytes of row r sits at c ^ (r / 4 % 4): 16 rows' chunks of one index, and four
// rows' 32 bytes, spread over all banks.  Blocks of 32 rows are alike, 2048 bytes apart.
__device__ __forceinline__ uint32_t chunk_at(int row, int c) { return row * 64 + ((c ^ ((row >> 2) & 3)) << 4); }
constexpr uint32_t kBlockBytes = 2048;

// Q and dO rows are stored with the channels of each 16 in the order 0-3, 8-11, 4-7, 12-15: a 16-byte chunk is then the
// operand's slice (t, hf) = chunk 2 t + hf, and in a product whose rows are these channels a lane's registers 0..7 and
// 8..15 are eight consecutive channels each, 8 hf and 16 + 8 hf on.
__device__ __forceinline__ void put_row_chunk(char* base, int row, int cn, u32x4 v) {
  const int t = cn >> 1, half = cn & 1;
  *reinterpret_cast<u32x2*>(base + chunk_at(row, 2 * t) + 8 * half) = u32x2{v.x, v.y};
  *reinterpret_cast<u32x2*>(base + chunk_at(row, 2 * t + 1) + 8 * half) = u32x2{v.z, v.w};
}

// A lane's addresses in the array of such rows.
struct RowReader {
  uint32_t row[2];      // slice t of the operand whose rows are the block's rows
  uint32_t turned[2];   // the operand whose rows are the 32 positions, contracted over the rows in an accumulator's order
  __device__ __forceinline__ RowReader(const void* base, int lane) {
    const int i = lane & 15, cb = (lane >> 4) & 1, hf = lane >> 5, l32 = lane & 31;
    const int r = 4 * hf + (i >> 2), c = 2 * cb + ((i >> 1) & 1), sub = (i & 1) * 8;
    const uint32_t b = lds_address(base);
    row[0] = kept(b + chunk_at(l32, hf));
    row[1] = kept(b + chunk_at(l32, 2 + hf));
    turned[0] = kept(b + chunk_at(r, c) + sub);
    turned[1] = kept(b + chunk_at(r + 8, c) + sub);
  }
  __device__ __forceinline__ bf16x8 rows(uint32_t offset, int t) const { return lds_read<bf16x8>(row[t] + offset); }
  __device__ __forceinline__ bf16x8 columns(uint32_t offset, int t) const {
    Pack8 p;
    p.d[0] = read_turned(turned[0] + offset + 1024 * t);
    p.d[1] = read_turned(turned[1] + offset + 1024 * t);
    return p.v;
  }
};

// A wave's own patch: a 32 x 32 tile [item][column], written from an accumulator whose lanes are the items and read
// as an operand whose lanes are the columns, contracted over the items (natural order).
__device__ __forceinline__ uint32_t patch_at(int row, int c, int sub) {
  return chunk_at(row, c) + ((sub ^ ((row >> 4) & 1)) << 3);
}
struct Patch {
  uint32_t put_at[4], get_at[2][2];
  __device__ __forceinline__ Patch(const void* base, int lane) {
    const int i = lane & 15, cb = (lane >> 4) & 1, hf = lane >> 5, item = lane & 31;
    const uint32_t b = lds_address(base);
#pragma unroll
    for (int g = 0; g < 4; ++g) put_at[g] = kept(b + patch_at(item, g, hf));
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int k = 0; k < 2; ++k)
        get_at[t][k] = kept(b + patch_at(16 * t + 8 * hf + 4 * k + (i >> 2), 2 * cb + ((i >> 1) & 1), i & 1));
  }
  __device__ __forceinline__ void put(uint32_t offset, const bf16x8 (&v)[2]) const {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      Pack8 p;
      p.v = v[g / 2];
      lds_write(put_at[g] + offset, p.d[g % 2]);
    }
  }
  __device__ __forceinline__ bf16x8 get(uint32_t offset, int t) const {
    Pack8 p;
    p.d[0] = read_turned(get_at[t][0] + offset);
    p.d[1] = read_turned(get_at[t][1] + offset);
    return p.v;
  }
};

}  // namespace
}  // namespace vista
