// Microscaled 4-bit floating point: blocks of 32 consecutive numbers of a row share a scale 2^s, held as the byte s + 127;
// a number is a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (two exponent bits, one mantissa bit).  The scale puts the block's
// largest magnitude between 4 and 8; what exceeds 6 becomes 6.  A block with an infinity or a NaN gets the scale byte 255,
// which reads as NaN for the whole block.  Byte i of a row's codes holds number 2 i in its lower half and 2 i + 1 above.
//
// The matrix instruction with scales takes exactly that: a lane's 16 bytes are one block of one row, its scale one byte, so
// rows go from memory to the matrix cores without a change of layout.
#include "kernels.h"
#include "product_tile.h"

namespace lshmoe {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = 32;   // numbers that share a scale

// Scale byte of a block whose largest magnitude has these bits.  The magnitude's exponent less 2; blocks of numbers below
// 2^-125 use the smallest scale.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits) {
  const uint32_t exponent = top_bits >> 23;
  return exponent == 255u ? 255u : exponent < 2u ? 0u : exponent - 2u;
}

// Binary32 whose exponent field is the scale byte: 2^s, and for byte 0 the number that the conversions take for 2^-127.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte == 0u ? 0x00400000u : byte << 23); }

// A thread has one block: its elements, 16 bytes of codes, one scale byte.
template <typename DT>
__global__ __launch_bounds__(256) void quantize_kernel(const char* __restrict__ x, char* __restrict__ codes,
                                                       uint8_t* __restrict__ scales, uint64_t blocks) {
  constexpr int kElems = Piece<DT>::kElems, kPieces = kBlock / kElems;
  const uint64_t b = linear_block() * 256 + threadIdx.x;
  if (b >= blocks) return;
  float v[kBlock];
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    float e[kElems];
    Piece<DT>::widen(load16(x + (b * kPieces + i) * 16), e);
#pragma unroll
    for (int j = 0; j < kElems; ++j) {
      v[i * kElems + j] = e[j];
      top = max(top, __float_as_uint(e[j]) & 0x7fffffffu);
    }
  }
  const uint32_t byte = scale_byte(top);
  const float scale = scale_value(byte == 255u ? 127u : byte);
  uint32_t word[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t q = 0u;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * i], v[8 * i + 1], scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * i + 2], v[8 * i + 3], scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * i + 4], v[8 * i + 5], scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[8 * i + 6], v[8 * i + 7], scale, 3);
    word[i] = byte == 255u ? 0u : q;
  }
  store16(codes + b * 16, make_uint4(word[0], word[1], word[2], word[3]));
  scales[b] = (uint8_t)byte;
}

template <typename DT>
__global__ __launch_bounds__(256) void dequantize_kernel(const char* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                         char* __restrict__ out, uint64_t blocks) {
  constexpr int kElems = Piece<DT>::kElems, kPieces = kBlock / kElems;
  const uint64_t b = linear_block() * 256 + threadIdx.x;
  if (b >= blocks) return;
  const uint4 q = load16(codes + b * 16);
  const uint32_t word[4] = {q.x, q.y, q.z, q.w}, byte = scales[b];
  const float scale = scale_value(byte == 255u ? 127u : byte);
  float v[kBlock];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 0);
    const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 1);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 2);
    const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 3);
    v[8 * i] = a[0]; v[8 * i + 1] = a[1]; v[8 * i + 2] = c[0]; v[8 * i + 3] = c[1];
    v[8 * i + 4] = d[0]; v[8 * i + 5] = d[1]; v[8 * i + 6] = e[0]; v[8 * i + 7] = e[1];
  }
#pragma unroll
  for (int i = 0; i < kBlock; ++i) v[i] = byte == 255u ? __uint_as_float(0x7fc00000u) : v[i];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    float e[kElems];
#pragma unroll
    for (int j = 0; j < kElems; ++j) e[j] = v[i * kElems + j];
    store16(out + (b * kPieces + i) * 16, Piece<DT>::narrow(e));
  }
}

constexpr int kTile = 64;   // outputs of a workgroup in either direction

template <typename DT> __device__ __forceinline__ float widen_at(const void* p, int64_t i);
template <> __device__ __forceinline__ float widen_at<F32>(const void* p, int64_t i) { return ((const float*)p)[i]; }
template <> __device__ __forceinline__ float widen_at<BF16>(const void* p, int64_t i) { return (float)((const __bf16*)p)[i]; }
template <typename DT> __device__ __forceinline__ void store_at(void* p, int64_t i, float v);
template <> __device__ __forceinline__ void store_at<F32>(void* p, int64_t i, float v) { ((float*)p)[i] = v; }
template <> __device__ __forceinline__ void store_at<BF16>(void* p, int64_t i, float v) { ((__bf16*)p)[i] = (__bf16)v; }

// 16 bytes of codes and the scale byte of block `block` of a row; a block behind the row's end is zeros.
__device__ __forceinline__ void load_block(const char* codes, const uint8_t* scales, int64_t row, int blocks, int block,
                                           i32x8& v, int& scale) {
  uint4 q = make_uint4(0u, 0u, 0u, 0u);
  scale = 127;
  if (block < blocks) {
    q = load16(codes + (row * blocks + block) * 16);
    scale = scales[row * blocks + block];
  }
  v = (i32x8){(int)q.x, (int)q.y, (int)q.z, (int)q.w, 0, 0, 0, 0};
}

// out = act(x W_e^T + b_e) of quantised x and W_e.  A wave has 64 columns of 16 rows; operands come straight from memory.
template <typename DT>
__global__ __launch_bounds__(256) void direct_kernel(const char* __restrict__ x_codes, const uint8_t* __restrict__ x_scales,
                                                      const char* __restrict__ w_codes, const uint8_t* __restrict__ w_scales,
                                                      const void* bias, const int32_t* __restrict__ offsets, int64_t rows,
                                                      int d_in, int d_out, int E, int act, void* out) {
  const int ptiles = (d_out + kTile - 1) / kTile;
  const RowTiles tiles(offsets, E, (int)rows, kTile);
  if (linear_block() >= (uint64_t)tiles.total * ptiles) return;
  const RowTile t = tiles.find((int)linear_block(), ptiles);
  const int p0 = t.column * kTile;
  const int lane = (int)threadIdx.x % 64, wave = (int)threadIdx.x / 64, r = lane % 16, g = lane / 16;
  const int blocks = d_in / kBlock;
  const int64_t q = (int64_t)t.first + 16 * wave + r, end = (int64_t)t.first + t.rows;
  f32x4 acc[4] = {};
  for (int k = 0; k < blocks; k += 4) {
    i32x8 b, a;
    int sb, sa;
    load_block(x_codes, x_scales, min(q, end - 1), blocks, k + g, b, sb);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      load_block(w_codes, w_scales, (int64_t)t.expert * d_out + min(p0 + 16 * i + r, d_out - 1), blocks, k + g, a, sa);
      acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[i], 4, 4, 0, sa, 0, sb);
    }
  }
  if (q >= end) return;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = p0 + 16 * i + 4 * g + j;
      if (p >= d_out) continue;
      float v = acc[i][j];
      if (bias) v += widen_at<DT>(bias, (int64_t)t.expert * d_out + p);
      store_at<DT>(out, q * d_out + p, activate(v, act));
    }
}

}  // namespace

hipError_t launch_mx4_quantize(const void* x, int64_t rows, int d, bool bf16, void* codes, uint8_t* scales, hipStream_t stream) {
  const uint64_t blocks = (uint64_t)rows * (d / kBlock);
  const dim3 grid = grid_of_blocks((blocks + 255) / 256);
  if (bf16)
    quantize_kernel<BF16><<<grid, 256, 0, stream>>>((const char*)x, (char*)codes, scales, blocks);
  else
    quantize_kernel<F32><<<grid, 256, 0, stream>>>((const char*)x, (char*)codes, scales, blocks);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const void* codes, const uint8_t* scales, int64_t rows, int d, bool bf16, void* out,
                                 hipStream_t stream) {
  const uint64_t blocks = (uint64_t)rows * (d / kBlock);
  const dim3 grid = grid_of_blocks((blocks + 255) / 256);
  if (bf16)
    dequantize_kernel<BF16><<<grid, 256, 0, stream>>>((const char*)codes, scales, (char*)out, blocks);
  else
    dequantize_kernel<F32><<<grid, 256, 0, stream>>>((const char*)codes, scales, (char*)out, blocks);
  return hipGetLastError();
}

namespace {

template <typename DT>
hipError_t forward_mx4(const void* x_codes, const uint8_t* x_scales, const void* w_codes, const uint8_t* w_scales,
                       const void* bias, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E, int act, void* out,
                       hipStream_t stream) {
  if (d_in % 128 == 0 && rows >= 64 * (int64_t)E) {
    typedef Tile<MX4, DT, false, false, 256, 256, 2, 4> TILE;
    auto kernel = forward_kernel<MX4, DT, TILE, 256, 256>;
    if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
    const uint64_t tiles = (uint64_t)most_row_tiles(rows, E, 256) * ((d_out + 255) / 256);
    kernel<<<blocks_for(tiles, 1), TILE::kThreads, TILE::kLds, stream>>>(
        (const char*)x_codes, (const char*)w_codes, (const char*)x_scales, (const char*)w_scales, (const char*)bias, offsets,
        (int)rows, d_in, d_out, E, act, nullptr, (char*)out);
    return hipGetLastError();
  }
  const dim3 grid = grid_of_blocks((uint64_t)most_row_tiles(rows, E, kTile) * ((d_out + kTile - 1) / kTile));
  direct_kernel<DT><<<grid, 256, 0, stream>>>((const char*)x_codes, x_scales, (const char*)w_codes, w_scales, bias, offsets, rows,
                                              d_in, d_out, E, act, out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_expert_forward_mx4(const void* x_codes, const uint8_t* x_scales, const void* w_codes, const uint8_t* w_scales,
                                     const void* bias, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E,
                                     bool bf16, int act, void* out, hipStream_t stream) {
  return bf16 ? forward_mx4<BF16>(x_codes, x_scales, w_codes, w_scales, bias, offsets, rows, d_in, d_out, E, act, out, stream)
              : forward_mx4<F32>(x_codes, x_scales, w_codes, w_scales, bias, offsets, rows, d_in, d_out, E, act, out, stream);
}

}  // namespace lshmoe
