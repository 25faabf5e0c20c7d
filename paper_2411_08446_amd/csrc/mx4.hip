// Microscaled 4-bit floating point: blocks of 32 consecutive numbers of a row share a scale 2^s, held as the byte s + 127;
// a number is a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (two exponent bits, one mantissa bit).  The scale puts the block's
// largest magnitude between 4 and 8; what exceeds 6 becomes 6.  A block with an infinity or a NaN gets the scale byte 255,
// which reads as NaN for the whole block.  Byte i of a row's codes holds number 2 i in its lower half and 2 i + 1 above.
//
// The matrix instruction with scales takes exactly that: a lane's 16 bytes are one block of one row, its scale one byte, so
// rows go from memory to the matrix cores without a change of layout.
#include "kernels.h"
#include "product_direct.h"
#include "product_tile.h"

namespace lshmoe {

namespace {

constexpr int kBlock = 32;   // numbers that share a scale

// Scale byte of a block whose largest magnitude has these bits.  The magnitude's exponent less 2; blocks of numbers below
// 2^-125 use the smallest scale.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top_bits) {
  const uint32_t exponent = top_bits >> 23;
  return exponent == 255u ? 255u : exponent < 2u ? 0u : exponent - 2u;
}

// Binary32 whose exponent field is the scale byte: 2^s, and for byte 0 the number that the conversions take for 2^-127.
__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte == 0u ? 0x00400000u : byte << 23); }

// A thread has pieces of 16 bytes, 256 pieces apart; the 4 or 8 lanes of a block find its largest magnitude together, so that
// loads and stores are whole lines.  Bound by the read.  The loads are streaming ones: 131072 x 1024 bf16 53 us, 6.4 TB/s with
// the codes, and 59 us behind kernels that filled the last-level cache with written lines (plain loads 57 and 89; four pieces to a
// thread 52 and 61, one 57 and 60; a thread per block, plain loads 59 and 91).
constexpr int kQuantPieces = 2;
template <typename DT>
__global__ __launch_bounds__(256) void quantize_kernel(const char* __restrict__ x, char* __restrict__ codes,
                                                       uint8_t* __restrict__ scales, uint64_t pieces) {
  constexpr int kElems = Piece<DT>::kElems, kPieces = kBlock / kElems;
  const uint64_t first = linear_block() * (256 * kQuantPieces) + threadIdx.x;
  uint4 data[kQuantPieces];
#pragma unroll
  for (int i = 0; i < kQuantPieces; ++i) data[i] = load16_stream(x + (first + 256 * i < pieces ? first + 256 * i : pieces - 1) * 16);
#pragma unroll
  for (int i = 0; i < kQuantPieces; ++i) {
    const uint64_t p = first + 256 * i;
    float v[kElems];
    Piece<DT>::widen(data[i], v);
    uint32_t top = 0u;
#pragma unroll
    for (int j = 0; j < kElems; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
    top = max(top, other_half<1>(top));
    top = max(top, other_half<2>(top));
    if (kPieces == 8) top = max(top, other_half<4>(top));
    const uint32_t byte = scale_byte(top);
    const float scale = scale_value(byte == 255u ? 127u : byte);
    uint32_t word = 0u;
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0], v[1], scale, 0);
    word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2], v[3], scale, 1);
    if constexpr (kElems == 8) {
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4], v[5], scale, 2);
      word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6], v[7], scale, 3);
    }
    if (byte == 255u) word = 0u;
    if (p >= pieces) continue;
    if (kElems == 8) *reinterpret_cast<uint32_t*>(codes + p * 4) = word;
    else *reinterpret_cast<uint16_t*>(codes + p * 2) = (uint16_t)word;
    if (p % kPieces == 0) scales[p / kPieces] = (uint8_t)byte;
  }
}

// A thread has pieces of 16 bytes of the result, 256 pieces apart: its neighbours' stores are next to its own.  Bound by the
// stores: 131072 x 1024 bf16 48 us, 7.0 TB/s with the codes (a thread per block, 64 bytes to a lane: 89; stores that stay in the caches: 60).
constexpr int kReadPieces = 4;
template <typename DT>
__global__ __launch_bounds__(256) void dequantize_kernel(const char* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                         char* __restrict__ out, uint64_t pieces) {
  constexpr int kElems = Piece<DT>::kElems, kPieces = kBlock / kElems;
  const uint64_t first = linear_block() * (256 * kReadPieces) + threadIdx.x;
  uint32_t word[kReadPieces], byte[kReadPieces];
#pragma unroll
  for (int i = 0; i < kReadPieces; ++i) {
    const uint64_t p = first + 256 * i < pieces ? first + 256 * i : pieces - 1;
    word[i] = kElems == 8 ? *reinterpret_cast<const uint32_t*>(codes + p * 4) : *reinterpret_cast<const uint16_t*>(codes + p * 2);
    byte[i] = scales[p / kPieces];
  }
#pragma unroll
  for (int i = 0; i < kReadPieces; ++i) {
    const float scale = scale_value(byte[i] == 255u ? 127u : byte[i]);
    float v[kElems];
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 1);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
    if constexpr (kElems == 8) {
      const f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 2);
      const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word[i], scale, 3);
      v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
    }
#pragma unroll
    for (int j = 0; j < kElems; ++j) v[j] = byte[i] == 255u ? __uint_as_float(0x7fc00000u) : v[j];
    if (first + 256 * i < pieces) store16_stream(out + (first + 256 * i) * 16, Piece<DT>::narrow(v));
  }
}

}  // namespace

hipError_t launch_mx4_quantize(const void* x, int64_t rows, int d, bool bf16, void* codes, uint8_t* scales, hipStream_t stream) {
  const uint64_t pieces = (uint64_t)rows * (d / (bf16 ? 8 : 4));
  const dim3 grid = grid_of_blocks((pieces + 256 * kQuantPieces - 1) / (256 * kQuantPieces));
  if (bf16)
    quantize_kernel<BF16><<<grid, 256, 0, stream>>>((const char*)x, (char*)codes, scales, pieces);
  else
    quantize_kernel<F32><<<grid, 256, 0, stream>>>((const char*)x, (char*)codes, scales, pieces);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const void* codes, const uint8_t* scales, int64_t rows, int d, bool bf16, void* out,
                                 hipStream_t stream) {
  const uint64_t pieces = (uint64_t)rows * (d / (bf16 ? 8 : 4));
  const dim3 grid = grid_of_blocks((pieces + 256 * kReadPieces - 1) / (256 * kReadPieces));
  if (bf16)
    dequantize_kernel<BF16><<<grid, 256, 0, stream>>>((const char*)codes, scales, (char*)out, pieces);
  else
    dequantize_kernel<F32><<<grid, 256, 0, stream>>>((const char*)codes, scales, (char*)out, pieces);
  return hipGetLastError();
}

namespace {

template <typename DT, typename S>
hipError_t forward_on_tiles(const void* x_codes, const uint8_t* x_scales, const void* w_codes, const uint8_t* w_scales,
                            const void* bias, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E, int act,
                            void* out, hipStream_t stream) {
  typedef Tile<MX4, DT, false, false, S::BP, S::BQ, S::WP, S::WQ> TILE;
  auto kernel = forward_kernel<MX4, DT, TILE, S::BP, S::BQ>;
  if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
  const uint64_t tiles = (uint64_t)most_row_tiles(rows, E, S::BQ) * ((d_out + S::BP - 1) / S::BP);
  kernel<<<blocks_for(tiles, S::kPerUnit), TILE::kThreads, TILE::kLds, stream>>>(
      (const char*)x_codes, (const char*)w_codes, (const char*)x_scales, (const char*)w_scales, (const char*)bias, offsets,
      (int)rows, d_in, d_out, E, act, nullptr, (char*)out);
  return hipGetLastError();
}

// Tiles move scales by 4 bytes, and so take rows of whole 128 numbers.  Others go through the few-row kernel whatever their number, which
// is several times as long for many of them: 131072 rows of 64 experts, 1056 -> 4096 columns 3826 us (1024: 418, 1152: 478),
// 2880 -> 2048 4081 (2816: 531, 2944: 620); 8192 rows, 1056 -> 4096 236 (1024: 41).
template <typename DT>
hipError_t forward_mx4(const void* x_codes, const uint8_t* x_scales, const void* w_codes, const uint8_t* w_scales,
                       const void* bias, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E, int act, void* out,
                       hipStream_t stream) {
  if (d_in % 128 != 0 || few_rows(rows, E, d_out, 8))
    return launch_direct<MX4, DT>((const char*)x_codes, (const char*)w_codes, (const char*)x_scales, (const char*)w_scales,
                                  (const char*)bias, offsets, rows, d_in / 2, d_out, E, act, nullptr, (char*)out, stream);
  if (small_tiles(rows, E, d_out))
    return forward_on_tiles<DT, Small>(x_codes, x_scales, w_codes, w_scales, bias, offsets, rows, d_in, d_out, E, act, out, stream);
  return forward_on_tiles<DT, Large>(x_codes, x_scales, w_codes, w_scales, bias, offsets, rows, d_in, d_out, E, act, out, stream);
}

}  // namespace

hipError_t launch_expert_forward_mx4(const void* x_codes, const uint8_t* x_scales, const void* w_codes, const uint8_t* w_scales,
                                     const void* bias, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E,
                                     bool bf16, int act, void* out, hipStream_t stream) {
  return bf16 ? forward_mx4<BF16>(x_codes, x_scales, w_codes, w_scales, bias, offsets, rows, d_in, d_out, E, act, out, stream)
              : forward_mx4<F32>(x_codes, x_scales, w_codes, w_scales, bias, offsets, rows, d_in, d_out, E, act, out, stream);
}

}  // namespace lshmoe
