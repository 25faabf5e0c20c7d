// Products of rows that are grouped by expert, on the matrix cores: the tiles that experts.hip and mx4.hip are made of.
//
// All products are out[q][p] = sum_k Q[q][k] P[p][k], p the index that is contiguous in the output:
//   forward      q = row, p = d_out, k = d_in       Q = x, P = W_e, both contiguous in k (4-bit numbers too)
//   input        q = row, p = d_in,  k = d_out      Q = grad_out contiguous in k, P = W_e contiguous in p
//   weight       q = d_out, p = d_in, k = row       Q = grad_out contiguous in q, P = x contiguous in p
// The matrix instruction takes P as its first operand: a lane then holds runs of 4 consecutive p of one q.
//
// A workgroup computes tiles of BQ x BP outputs, one after the other.  k goes by chunks: 128 bytes of every row of an operand
// that is contiguous in k ("rows"), as many k of one that is not ("columns").  Chunks go from memory straight into LDS, into
// rings of three chunks of P and two of Q (160 KB for two workgroups of binary32 or one of bf16), one barrier to a chunk.
// A wave spreads its loads between its products: a chunk's loads all at once fill the address units' queue, and the
// products behind them wait.  The chunks of all tiles of a workgroup are one stream: while a tile's results are
// stored, the first chunks of the next are on their way.
//
// Measured, as many rows to every expert (no tile partly empty) where nothing else is said.  131072 rows of 32 experts, 4096 -> 4096
// columns of bf16: 3334 to 3494 us, 1.26 to 1.32 PFLOP/s; bound by the matrix cores (busy two thirds of the time; the loop's
// barriers and the clock on real data take the rest).  1024 -> 4096 columns of 64 experts with values kept before the
// activation: 1267 to 1294 us with ReLU, 0.85 to 0.87 PFLOP/s, and 1361 to 1376 with GELU (ReLU, 1557 to 2667 rows to an expert:
// 1314).  A tile's results are as many bytes as its operands there, and their stores, 14 us to a round of tiles, do not overlap
// with products: the 256 x 256 forward kernels do not have registers enough (bf16 keeps 17 words of a lane in scratch memory, two of the
// table of tiles among them, 4 bits 4 to 8), and the wait for what is fetched from there, in front of the next tile, is one for the
// stores too, since operations count as done in their order.  4 bits: 4096 -> 4096 columns 1433 to 1457 us, 3.0 to 3.1 PFLOP/s;
// 1024 -> 4096 columns 418 us, with 1557 to 2667 rows to an expert 445, and 553 behind the quantisation of rows that are new each time.
// binary32, 15011 rows of 6 experts, 1000 -> 1500 columns, GELU: 393 to 402 us, 112 to 115 TFLOP/s.
#pragma once

#include <type_traits>
#include <utility>

#include "kernels.h"
#include "rows_by_expert.h"

namespace lshmoe {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunkBytes = 128;   // of a row per chunk
constexpr int kPieces = kChunkBytes / 16;
constexpr int kSteps = kPieces / 2;   // steps of two 16-byte pieces, one per lane half, per chunk

// Piece s of row i of a chunk of rows lies in slot s ^ row_shift(i): 16 lanes reading a piece of 16 rows cover 256 bytes once.
__device__ __forceinline__ int row_shift(int i) { return i / (256 / kChunkBytes) % kPieces; }

// c += P Q of one step: 8 elements of k (bf16, one instruction of 16 with the other lane half) or 4 (binary32, four of 2).
template <typename OT> __device__ __forceinline__ void mma(const u32x4& a, const u32x4& b, f32x16& c);
template <> __device__ __forceinline__ void mma<BF16>(const u32x4& a, const u32x4& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma<F32>(const u32x4& a, const u32x4& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[0]), __uint_as_float(b[0]), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[1]), __uint_as_float(b[1]), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[2]), __uint_as_float(b[2]), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[3]), __uint_as_float(b[3]), c, 0, 0, 0);
}

// c += P Q of one step of 4-bit numbers, 32 to a lane, one instruction of 64: S is the step within a chunk.  A lane's scales are the bytes
// 0 and 2 of a word per two steps.
typedef int i32x8 __attribute__((ext_vector_type(8)));
template <int S> __device__ __forceinline__ void mma_scaled(const u32x4& a, const u32x4& b, uint32_t scale_a, uint32_t scale_b, f32x16& c) {
  const i32x8 wide_a = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8 wide_b = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide_a, wide_b, c, 4, 4, S % 2 * 2, (int)scale_a, S % 2 * 2, (int)scale_b);
}

// 16 bytes per lane from a buffer straight into LDS: lane l's piece, offset + ahead bytes into the buffer, lands at dst + 16 l (ahead
// and dst are wave-uniform); a lane whose piece is behind the buffer's end gets zeros.  Inline assembly, because behind the compiler's own builtin every LDS read
// waits until the load has landed; the caller waits for these loads itself.  Between m0's write and its use is one wait state.
__device__ __forceinline__ void load16_to_lds(const i32x4& buffer, uint32_t offset, uint32_t ahead, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %2, %3 offen lds"
               : : "v"(offset), "s"(dst), "s"(buffer), "s"(ahead) : "memory", "m0");
}

// The same with 4 bytes per lane.
__device__ __forceinline__ void load4_to_lds(const i32x4& buffer, uint32_t offset, uint32_t ahead, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dword %0, %2, %3 offen lds"
               : : "v"(offset), "s"(dst), "s"(buffer), "s"(ahead) : "memory", "m0");
}

__device__ __forceinline__ i32x4 buffer_of(const char* base, int64_t bytes) {
  const uint64_t at = (uint64_t)base;
  const uint32_t size = bytes <= 0 ? 0u : bytes > 0x7fffffff ? 0x7fffffffu : (uint32_t)bytes;
  return (i32x4){__builtin_amdgcn_readfirstlane((int)(uint32_t)at), __builtin_amdgcn_readfirstlane((int)(uint32_t)(at >> 32) & 0xffff),
                 __builtin_amdgcn_readfirstlane((int)size), 0x00020000};
}

constexpr uint32_t kNowhere = 0x80000000u;   // an offset behind the end of every buffer

// One operand of a tile: B indices, COLUMNS: contiguous in the index and not in k.
//
// LDS holds a chunk of rows as [index][kPieces].  A chunk of columns is [k][B elements]; the pieces of bf16 are moved by 64 bytes times k % 4
// (a transposing read takes 32 bytes each of 4 consecutive k, 16 lanes at a time), of binary32 by 128 bytes times k / 4 % 2.
template <typename OT, bool COLUMNS, int B, int WAVES> struct Operand {
  static constexpr int kItem = ItemSize<OT>::value;
  static constexpr int kChunk = kChunkBytes / kItem;              // k of a chunk
  static constexpr int kBytes = B * kChunkBytes;                  // LDS of a chunk
  static constexpr int kLoads = kBytes / (1024 * WAVES);          // instructions of a wave per chunk
  static constexpr int kRowPieces = COLUMNS ? B * kItem / 16 : kPieces;   // pieces of a line of LDS
  static_assert(kLoads * 1024 * WAVES == kBytes, "whole instructions");

  uint32_t offset[kLoads];   // of the lane's pieces from the chunk's first element
  uint32_t k_piece;          // rows: the lane's piece within the chunk, in bytes
  uint32_t stride;           // bytes from one index (rows) or k (columns) to the next
  i32x4 buffer;              // descriptor of what may be read from the tile's first element (or from further on) to its end
  uint32_t ahead;            // of the next chunk's first element from there
  uint32_t now;              // of the chunk being loaded
  int left;                  // rows: bytes of k from the next chunk on
  uint32_t cut;              // rows: kNowhere where the lane's piece of a chunk that is not whole is behind the end of the rows
  uint32_t away;             // the same for the chunk being loaded
  const char* base;          // columns: where the buffer starts, the bytes to its end
  int64_t bytes;

  __device__ __forceinline__ explicit Operand(uint32_t stride_) : k_piece(0), stride(stride_) {
    const int lane = (int)threadIdx.x % 64, wave = (int)threadIdx.x / 64;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int slot = (i * WAVES + wave) * 64 + lane, line = slot / kRowPieces, s = slot % kRowPieces;
      if (COLUMNS) {
        const int shift = kItem == 2 ? (line & 3) << 2 : (line >> 2 & 1) << 3;
        offset[i] = (uint32_t)line * stride + (uint32_t)(s ^ shift) * 16;
      } else {
        k_piece = (uint32_t)(s ^ row_shift(line)) * 16;           // the same for every i: lines are 8 WAVES apart
        offset[i] = (uint32_t)line * stride + k_piece;
      }
    }
  }

  // A tile's operand: element (index i, k) is at first + i * stride + k * item (rows) or first + k * stride + i * item
  // (columns); `indices` of the tile and K of k exist.
  __device__ __forceinline__ void start(const char* first, int indices, int K) {
    base = first;
    left = K * kItem;
    bytes = COLUMNS ? (int64_t)(K - 1) * stride + indices * kItem : (int64_t)(indices - 1) * stride + K * kItem;
    if (K == 0 || indices == 0) bytes = 0;
    cut = !COLUMNS && (int)k_piece >= left % kChunkBytes ? kNowhere : 0u;
    restart();
  }
  __device__ __forceinline__ void restart() {
    buffer = buffer_of(base, bytes);
    ahead = 0;
    // the descriptor may come from vector instructions: five cycles before its use
    asm volatile("s_nop 4" : "+s"(buffer));
  }
  // The next chunk's loads begin.  Behind the last chunk they bring zeros and read nothing.
  __device__ __forceinline__ void next() {
    if (COLUMNS && ahead >= 1u << 30) {             // offsets are 32 bits and a buffer ends below 2^31
      base += ahead;
      bytes -= ahead;
      restart();
    }
    now = ahead;
    ahead += COLUMNS ? kChunk * stride : (uint32_t)kChunkBytes;
    if (!COLUMNS) away = left < kChunkBytes ? cut : 0u;
    left -= kChunkBytes;
    asm volatile("s_nop 4" : "+s"(buffer), "+s"(now));   // as in restart
  }
  // Starts load i of the chunk; lds: where the ring's slot has the wave's first 1024 bytes.
  __device__ __forceinline__ void load(int i, uint32_t lds) const {
    load16_to_lds(buffer, COLUMNS ? offset[i] : offset[i] | away, now, lds + i * WAVES * 1024);
  }
};

// The scales of two operands of 4-bit numbers, B indices each: 8 bytes of a row to a chunk, in LDS as two words of [P's index, then
// Q's].  The first half of the waves load P's, the others Q's.  Rows of whole 4 bytes.
template <int B, int WAVES> struct ScaleOperand {
  static constexpr int kBytes = 2 * B * 8;
  static_assert(kBytes == 512 * WAVES, "two loads of 4 bytes a lane to a wave");
  uint32_t offset, ahead, now, away, stride;
  i32x4 buffer;
  bool mine_p;

  __device__ __forceinline__ explicit ScaleOperand(uint32_t stride_) : stride(stride_) {
    offset = (uint32_t)((int)threadIdx.x % (32 * WAVES)) * stride;
    mine_p = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64) < WAVES / 2;
  }
  __device__ __forceinline__ void start(const char* first_p, const char* first_q, int np, int nq, int K) {
    const int n = K == 0 ? 0 : mine_p ? np : nq;
    buffer = buffer_of(mine_p ? first_p : first_q, (int64_t)n * stride);
    ahead = 0;
    asm volatile("s_nop 4" : "+s"(buffer));
  }
  __device__ __forceinline__ void next() {
    now = ahead;
    ahead += 8;
    away = ahead > stride ? kNowhere : 0u;      // half a chunk: the second word is behind the row's end
    asm volatile("s_nop 4" : "+s"(buffer), "+s"(now));
  }
  __device__ __forceinline__ void load(int i, uint32_t lds) const {
    load4_to_lds(buffer, i == 0 ? offset : offset + 4 | away, now, lds + i * 256 * WAVES);
  }
};

typedef __attribute__((address_space(3))) char lds_char;

// Compile-time loop: f is called with std::integral_constant<int, 0> .. <int, N - 1>.
template <typename F, int... I> __device__ __forceinline__ void static_for_impl(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F> __device__ __forceinline__ void static_for(F&& f) {
  static_for_impl(f, std::make_integer_sequence<int, N>{});
}

// Fragments of a wave: T tiles of 32 indices from `first` on.
template <typename OT, bool COLUMNS, int B, int T> struct Fragments {
  static constexpr int kLine = B * ItemSize<OT>::value;   // columns: bytes of a line
  static constexpr int kAddresses = COLUMNS ? T : kSteps;
  uint32_t at[kAddresses];

  __device__ __forceinline__ explicit Fragments(int first) {
    const int lane = (int)threadIdx.x % 64, r = lane % 32, h = lane / 32;
#pragma unroll
    for (int i = 0; i < kAddresses; ++i) {
      if (!COLUMNS) {
        at[i] = (uint32_t)((first + r) * kChunkBytes + ((2 * i + h) ^ row_shift(r)) * 16);
      } else if (ItemSize<OT>::value == 2) {
        // lane l of 16 supplies 8 bytes of k l / 4 and receives 4 k of index l % 16
        const int kk = lane % 16 / 4;
        at[i] = (uint32_t)((8 * h + kk) * kLine + ((first / 32 + i) ^ kk) * 64 + (lane / 16 & 1) * 32 + lane % 4 * 8);
      } else {
        at[i] = (uint32_t)(4 * h * kLine + ((first / 32 + i) ^ h) * 128 + r * 4);
      }
    }
  }

  // Fragment of step s (a constant) of tile t.
  __device__ __forceinline__ u32x4 read(lds_char* lds, int s, int t) const {
    if (!COLUMNS) return *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>(lds + at[s] + t * 32 * kChunkBytes);
    if (ItemSize<OT>::value == 2) {
      lds_char* p = lds + at[COLUMNS ? t : 0] + s * 16 * kLine;
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)p);
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p + 4 * kLine));
      const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
      return (u32x4){a.x, a.y, b.x, b.y};
    }
    typedef __attribute__((address_space(3))) const uint32_t* word;
    lds_char* p = lds + at[COLUMNS ? t : 0] + s * 8 * kLine;
    return (u32x4){*(word)p, *(word)(p + kLine), *(word)(p + 2 * kLine), *(word)(p + 3 * kLine)};
  }
};

struct TileEntry { int v[5]; };

// OT: type of the operands, DT: of the results.
template <typename OT, typename DT, bool P_COLUMNS, bool Q_COLUMNS, int BP, int BQ, int WP, int WQ> struct Tile {
  static constexpr int kWaves = WP * WQ, kThreads = 64 * kWaves;
  static constexpr int TP = BP / WP / 32, TQ = BQ / WQ / 32;     // 32 x 32 tiles of a wave
  typedef Operand<OT, P_COLUMNS, BP, kWaves> OpP;
  typedef Operand<OT, Q_COLUMNS, BQ, kWaves> OpQ;
  static constexpr int kPieceReads = std::is_same<OT, BF16>::value ? 8 : 4;   // bytes that one read of columns gives a lane
  // Chunks in LDS.  Operands of 4-bit numbers have their scales there too, which take the room of P's third chunk.
  static constexpr bool kScaled = std::is_same<OT, MX4>::value;
  static constexpr int kRingP = kScaled ? 2 : 3, kRingQ = 2;
  static constexpr int kAtQ = kRingP * OpP::kBytes, kAtScales = kAtQ + kRingQ * OpQ::kBytes;
  static_assert(!kScaled || BP == BQ, "the waves share the scales' loads evenly");
  typedef ScaleOperand<32 * kWaves, kWaves> Scales;
  static constexpr size_t kLds = kAtScales + (kScaled ? 2 * Scales::kBytes : 0);
  static_assert(OpP::kLoads == 4 && OpQ::kLoads == 4 && kSteps == 4 && TP % 2 == 0, "a load to a half step");

  struct Feed {
    OpP P;
    OpQ Q;
    Scales S;
    lds_char* lds;
    uint32_t to_p, to_q, to_s;   // where a wave's loads go
    int slot_p, slot_q;          // ring slots of the chunk at work
    int chunks_p, chunks_q;      // of the tiles being loaded, still to be loaded

    // The next chunk's loads begin.
    __device__ __forceinline__ void next_p() {
      P.next();
      if constexpr (kScaled) S.next();
      --chunks_p;
    }
    __device__ __forceinline__ void next_q() {
      Q.next();
      --chunks_q;
    }
  };

  f32x16 acc[TP][TQ];
  float sums[TQ];           // where wanted: Q summed over the k that the lane half holds
  uint32_t scale_p[TP][2], scale_q[TQ][2];   // scales of the chunk, of this lane half in bytes 0 and 2
  u32x4 a[2][TP / 2], b[2][TQ];   // fragments: of half a step and the next half; of a step and the next one

  __device__ __forceinline__ static void add_elements(const u32x4& q, float& sum) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (ItemSize<DT>::value == 2) sum += __uint_as_float(q[i] << 16);
      sum += __uint_as_float(ItemSize<DT>::value == 2 ? q[i] & 0xffff0000u : q[i]);
    }
  }

  typedef Fragments<OT, P_COLUMNS, BP, TP> FragP;
  typedef Fragments<OT, Q_COLUMNS, BQ, TQ> FragQ;

  // The scales of the chunk at work.
  __device__ __forceinline__ void read_scales(const Feed& f) {
    typedef __attribute__((address_space(3))) const uint32_t* word;
    const int lane = (int)threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64), shift = lane / 32 * 8;
    lds_char* const at = f.lds + kAtScales + f.slot_q * Scales::kBytes + lane % 32 * 4;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int t = 0; t < TP; ++t) scale_p[t][i] = *(word)(at + i * Scales::kBytes / 2 + (wave % WP * TP + t) * 128) >> shift;
#pragma unroll
      for (int u = 0; u < TQ; ++u) scale_q[u][i] = *(word)(at + i * Scales::kBytes / 2 + BP * 4 + (wave / WP * TQ + u) * 128) >> shift;
    }
  }

  // One chunk's products, the loads of a chunk ahead, the first fragments of the next chunk.  A half step is the products of half
  // of P's tiles: fragments of P are read half a step ahead, of Q a step ahead.  In front of the last half step is the
  // chunk's barrier.  While chunk c is at work, Q's loads of chunk c + 1, which is needed first, are started behind the first
  // half step's products, P's of chunk c + 2 one by one behind the next ones' (Q's one by one too: 6 to 9 % more time); Q's of
  // the next tile's second chunk are started at the end of the last one, in front of the results' stores.  With scales:
  // everything of chunk c + 1, two or three to a half step.
  template <bool SUMS, bool FIRST, bool LAST, typename SwitchP, typename SwitchQ>
  __device__ __forceinline__ void chunk(const FragP& fp, const FragQ& fq, Feed& f, SwitchP&& switch_p, SwitchQ&& switch_q,
                                        int stores) {
    lds_char* const now_p = f.lds + f.slot_p * OpP::kBytes;
    lds_char* const now_q = f.lds + kAtQ + f.slot_q * OpQ::kBytes;
    const int slot_next = f.slot_p == kRingP - 1 ? 0 : f.slot_p + 1, slot_free = f.slot_p == 0 ? kRingP - 1 : f.slot_p - 1;
    lds_char* const next_p_at = f.lds + slot_next * OpP::kBytes;
    lds_char* const next_q_at = f.lds + kAtQ + (f.slot_q ^ 1) * OpQ::kBytes;
    constexpr bool kLoadQ = !FIRST, kLoadP = !kScaled || !FIRST;
    // everything that branches is in front of the products: they are one straight line
    if (kLoadQ) switch_q();
    if (kLoadP) switch_p();
    if constexpr (kScaled) read_scales(f);
    auto load_scales = [&](int slot) {
      if constexpr (kScaled) {
        f.S.load(0, f.to_s + slot * Scales::kBytes);
        f.S.load(1, f.to_s + slot * Scales::kBytes);
      }
    };
    static_for<2 * kSteps>([&](auto ic) {
      constexpr int i = decltype(ic)::value, s = i / 2, half = i % 2;
      constexpr bool kEnd = i == 2 * kSteps - 1;
      if (kEnd) {
        // The last fragments of this chunk are in registers, this wave's share of the next one has landed (P's of the one after it and a
        // finished tile's stores may be under way, as far as this wait goes: in the kernels that fetch spilled registers in front
        // of a tile the stores have ended there).  Behind the barrier that is so for all waves: this chunk's slots are free, the
        // next one may be read.
        constexpr int kUnderWay = kScaled ? 0 : 4;
        static_assert(kScaled || kUnderWay + 2 * kStores < 64, "what a wait can name");
        if (FIRST) {
          if (!kScaled && stores == 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(kScaled ? 0 : kUnderWay + 2 * kStores) : "memory");
          else if (stores) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(kUnderWay + kStores) : "memory");
          else asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(kUnderWay) : "memory");
        } else {
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" : : "n"(kUnderWay) : "memory");
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" : : : "memory");
      }
      // reads for the next half step
      constexpr int sn = kEnd ? 0 : (i + 1) / 2, halfn = (i + 1) % 2;
#pragma unroll
      for (int t = 0; t < TP / 2; ++t) a[halfn][t] = fp.read(kEnd ? next_p_at : now_p, sn, halfn * TP / 2 + t);
      constexpr int kFirstQ = kEnd ? 0 : s == kSteps - 1 ? TQ : half * TQ / 2;
      constexpr int kLastQ = kEnd ? TQ : s == kSteps - 1 ? TQ : (half + 1) * TQ / 2;
#pragma unroll
      for (int u = kFirstQ; u < kLastQ; ++u) b[(s + 1) & 1][u] = fq.read(kEnd ? next_q_at : now_q, (s + 1) % kSteps, u);
#pragma unroll
      for (int t = 0; t < TP / 2; ++t)
#pragma unroll
        for (int u = 0; u < TQ; ++u) {
          constexpr int t0 = half * TP / 2;
          if constexpr (kScaled) {
            mma_scaled<s>(a[half][t], b[s & 1][u], scale_p[t0 + t][s / 2], scale_q[u][s / 2], acc[t0 + t][u]);
            // the compiler may move this instruction behind later branches, which keeps all fragments alive until there
            asm volatile("" : "+v"(acc[t0 + t][u]));
          } else {
            mma<OT>(a[half][t], b[s & 1][u], acc[t0 + t][u]);
          }
        }
      if constexpr (SUMS) {
#pragma unroll
        for (int u = half * TQ / 2; u < (half + 1) * TQ / 2; ++u) add_elements(b[s & 1][u], sums[u]);
      }
      // reads and products take turns
      constexpr int kReads = TP / 2 * (P_COLUMNS ? 16 / kPieceReads : 1) + (kLastQ - kFirstQ) * (Q_COLUMNS ? 16 / kPieceReads : 1);
      constexpr int kTurns = TP / 2 * TQ;
      constexpr int kProducts = kTurns * (std::is_same<OT, F32>::value ? 4 : 1);
      static_for<kTurns>([&](auto jc) {
        constexpr int n = decltype(jc)::value;
        __builtin_amdgcn_sched_group_barrier(0x100, kReads * (n + 1) / kTurns - kReads * n / kTurns, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, kProducts * (n + 1) / kTurns - kProducts * n / kTurns, 0);
      });
      __builtin_amdgcn_sched_barrier(0);
      // loads, in the shadow of the products just started
      if constexpr (kScaled) {
        constexpr int kFrom[5] = {0, 1, 4, 6, 8};      // loads 0 .. 3 are Q's, 4 .. 7 P's
        if (kLoadQ && i == 0) {
          f.next_q();
          f.next_p();
          load_scales(f.slot_q ^ 1);
        }
        if constexpr (kLoadQ && i < 4) {
#pragma unroll
          for (int j = kFrom[i]; j < kFrom[i + 1]; ++j) {
            if (j < 4) f.Q.load(j, f.to_q + (f.slot_q ^ 1) * OpQ::kBytes);
            else f.P.load(j - 4, f.to_p + slot_free * OpP::kBytes);
          }
        }
      } else {
        if (kLoadQ && i == 0) f.next_q();
        if (i == 2) f.next_p();
        if (kLoadQ && i == 0) f.Q.load(0, f.to_q + (f.slot_q ^ 1) * OpQ::kBytes);
        if (kLoadQ && i == 0) f.Q.load(1, f.to_q + (f.slot_q ^ 1) * OpQ::kBytes);
        if (kLoadQ && i == 0) f.Q.load(2, f.to_q + (f.slot_q ^ 1) * OpQ::kBytes);
        if (kLoadQ && i == 0) f.Q.load(3, f.to_q + (f.slot_q ^ 1) * OpQ::kBytes);
        if (i == 2) f.P.load(0, f.to_p + slot_free * OpP::kBytes);
        if (i == 3) f.P.load(1, f.to_p + slot_free * OpP::kBytes);
        if (i == 4) f.P.load(2, f.to_p + slot_free * OpP::kBytes);
        if (i == 5) f.P.load(3, f.to_p + slot_free * OpP::kBytes);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if (LAST) {
      switch_q();
      f.next_q();
      if constexpr (kScaled) {
        switch_p();
        f.next_p();
        load_scales(f.slot_q);
#pragma unroll
        for (int j = 0; j < 4; ++j) f.P.load(j, f.to_p + f.slot_p * OpP::kBytes);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) f.Q.load(j, f.to_q + f.slot_q * OpQ::kBytes);
    }
    f.slot_p = slot_next;
    f.slot_q ^= 1;
  }

  // All chunks of a tile.
  template <bool SUMS, typename SwitchP, typename SwitchQ>
  __device__ __forceinline__ void products(const FragP& fp, const FragQ& fq, Feed& f, SwitchP&& switch_p, SwitchQ&& switch_q,
                                           int chunks, int stores) {
    if (chunks == 1) {
      chunk<SUMS, true, true>(fp, fq, f, switch_p, switch_q, stores);
      return;
    }
    chunk<SUMS, true, false>(fp, fq, f, switch_p, switch_q, stores);
    for (int c = chunks - 2; c > 0; --c) chunk<SUMS, false, false>(fp, fq, f, switch_p, switch_q, stores);
    chunk<SUMS, false, true>(fp, fq, f, switch_p, switch_q, stores);
  }

  // The tiles n, n + step, .. below end.  JOB: entry(n) says which tile n is, each lane of another one; place(entry) gives a
  // tile's operands and where its results go; finish(place, tile) stores them, with kStores stores to a wave or more, or
  // twice that where job.twice().
  // Lane i of a wave has the entry of the tile i steps on: looked up one by one between the products, they cost
  // 3 of a tile's 40 us at K = 1024.
  template <typename JOB> __device__ __forceinline__ void run(const JOB& job, int n, int end, int step) {
    extern __shared__ uint4 lds[];
    if (n >= end) return;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const FragP fp(wave % WP * TP * 32);
    const FragQ fq(wave / WP * TQ * 32);
    Feed f = {OpP(job.p_stride()), OpQ(job.q_stride()), Scales(job.s_stride()), (lds_char*)lds, 0, 0, 0, 0, 0, 0, 0};
    f.to_p = (uint32_t)(uintptr_t)f.lds + wave * 1024;
    f.to_q = f.to_p + kAtQ;
    f.to_s = (uint32_t)(uintptr_t)f.lds + kAtScales + wave * 256;
    const int count = (end - n + step - 1) / step;       // tiles
    int at = 0, table_at = 0;                              // the tile at work, the first of the table's
    TileEntry table = job.template entry<false>(n + (int)(threadIdx.x % kWave) * step);
    auto place = [&](int i) {
      if (i - table_at >= kWave) {
        table_at = at;
        table = job.template entry<true>(n + (at + (int)(threadIdx.x % kWave)) * step);
      }
      TileEntry e;
#pragma unroll
      for (int j = 0; j < 5; ++j) e.v[j] = __builtin_amdgcn_readlane(table.v[j], i - table_at);
      return job.place(e);
    };
    typename JOB::Place here = place(0);
    int at_p = 0, at_q = 0;                                // the tiles that P's and Q's loads are at
    auto start_p = [&](const typename JOB::Place& x) {
      f.P.start(x.p, x.np, x.K);
      if constexpr (kScaled) f.S.start(x.w_scales, x.x_scales, x.np, x.nq, x.K);
      f.chunks_p = x.chunks();
    };
    auto start_q = [&](const typename JOB::Place& x) {
      f.Q.start(x.q, x.nq, x.K);
      f.chunks_q = x.chunks();
    };
    auto switch_p = [&] {
      if (f.chunks_p == 0) start_p(++at_p < count ? place(at_p) : JOB::Place::none(here));
    };
    auto switch_q = [&] {
      if (f.chunks_q == 0) start_q(++at_q < count ? place(at_q) : JOB::Place::none(here));
    };
    start_p(here);
    start_q(here);
    auto load_q = [&](int slot) {
      switch_q();
      f.next_q();
#pragma unroll
      for (int i = 0; i < 4; ++i) f.Q.load(i, f.to_q + slot * OpQ::kBytes);
    };
    auto load_p = [&](int slot) {
      switch_p();
      f.next_p();
#pragma unroll
      for (int i = 0; i < 4; ++i) f.P.load(i, f.to_p + slot * OpP::kBytes);
      if constexpr (kScaled) {
        f.S.load(0, f.to_s + slot * Scales::kBytes);
        f.S.load(1, f.to_s + slot * Scales::kBytes);
      }
    };
    load_q(0);
    load_p(0);
    load_p(1);
    asm volatile("s_waitcnt vmcnt(%0)" : : "n"(kScaled ? 6 : 4) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
    load_q(1);
    int stores = 0;          // of the tile before, in units of kStores
    for (;;) {
      // the first fragments and scales (again behind a finished tile: they would take registers that its results need)
#pragma unroll
      for (int t = 0; t < TP / 2; ++t) a[0][t] = fp.read(f.lds + f.slot_p * OpP::kBytes, 0, t);
#pragma unroll
      for (int u = 0; u < TQ; ++u) b[0][u] = fq.read(f.lds + kAtQ + f.slot_q * OpQ::kBytes, 0, u);
#pragma unroll
      for (int u = 0; u < TQ; ++u) {
#pragma unroll
        for (int t = 0; t < TP; ++t) acc[t][u] = (f32x16){};
        sums[u] = 0.0f;
      }
      if (JOB::kSums && job.sums(here)) products<JOB::kSums>(fp, fq, f, switch_p, switch_q, here.chunks(), stores);
      else products<false>(fp, fq, f, switch_p, switch_q, here.chunks(), stores);
      job.finish(here, *this);
      stores = job.twice() ? 2 : 1;
      if (++at == count) break;
      here = place(at);
    }
    asm volatile("s_waitcnt vmcnt(0)" : : : "memory");   // nothing is on its way to LDS when the workgroup ends
  }

  // ---- results: lanes and memory.  Of the 32 x 32 results of tiles t, u a lane has q = r = lane % 32 and, h = lane / 32, p = 8 j + 4 h
  // + 0 .. 3 for j = 0 .. 3.  Three exchanges between lanes make that 16 bytes of consecutive p to a lane and whole lines of 128
  // bytes of 8 rows to an instruction: a group, 128 bytes of p (one tile of binary32, two of bf16) by 32 q, is four pieces
  // to a lane, of q = 8 i + lane % 8.  (64 bytes of 16 rows: 1578 us in place of 1326 at K = 1024
  // with two results stored.)
  static constexpr int kItemsPerWord = 4 / ItemSize<DT>::value;
  static constexpr int kGroupTiles = kItemsPerWord, kGroups = TP / kGroupTiles;
  static constexpr int kStores = kGroups * TQ * 4;

  struct Lines {
    __amdgpu_buffer_rsrc_t buffer;
    uint32_t at, ld;     // the lane's first piece of the wave's part; bytes of a line
    int p, np;           // its column; columns that exist
  };
  // first: the tile's first element in an array of lines of ld bytes; nq by np of it exist.
  __device__ __forceinline__ static Lines lines(const char* first, uint32_t ld, int nq, int np) {
    return lines(first, ld, nq, np, __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64));
  }
  __device__ __forceinline__ static Lines lines(const char* first, uint32_t ld, int nq, int np, int wave) {
    const int lane = (int)threadIdx.x % 64;
    const int64_t bytes = nq == 0 ? 0 : (int64_t)(nq - 1) * ld + np * ItemSize<DT>::value;
    Lines l;
    l.buffer = __builtin_amdgcn_make_buffer_rsrc((void*)first, 0, (int)min(bytes, (int64_t)0x7fffffff), 0x00020000);
    l.ld = ld;
    l.p = wave % WP * TP * 32 + (lane / 8 % 2 * 32 + lane / 16 % 2 * 16 + lane / 32 * 8) * kItemsPerWord / 2;
    l.np = np;
    l.at = (uint32_t)(wave / WP * TQ * 32 + lane % 8) * ld + (uint32_t)l.p * ItemSize<DT>::value;
    return l;
  }
  // Offset of the lane's piece i of group g and tile u; behind the end of the buffer where there is no such column (or line).
  __device__ __forceinline__ static uint32_t piece_at(const Lines& l, int g, int u, int i) {
    return l.p + 32 * kGroupTiles * g < l.np ? l.at + (uint32_t)(32 * u + 8 * i) * l.ld + 128u * g : kNowhere;
  }
  // Lanes 32 .. 63 of x and 0 .. 31 of y change places; lanes 16 .. 31 of 32 of x and 0 .. 15 of y; lanes 8 .. 15 of 16 of x and 0 .. 7
  // of y.  Each is its own inverse.
  __device__ __forceinline__ static void swap32(uint32_t& x, uint32_t& y) {
    const auto v = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    x = v[0];
    y = v[1];
  }
  __device__ __forceinline__ static void swap16(uint32_t& x, uint32_t& y) {
    const auto v = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    x = v[0];
    y = v[1];
  }
  __device__ __forceinline__ static void swap8(uint32_t& x, uint32_t& y) {
    constexpr int kRotateBy8 = 0x128;
    const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)y, kRotateBy8, 0xf, 0xc, false);
    y = (uint32_t)__builtin_amdgcn_update_dpp((int)y, (int)x, kRotateBy8, 0xf, 0x3, false);
    x = a;
  }
  // From the lanes' results to pieces, w[4 i .. 4 i + 3] piece i, or back.  Before: bf16 w[8 t + 2 j + i] is the pair of p 32 t + 8 j + 4 h +
  // 2 i, binary32 w[4 j + i] is p 8 j + 4 h + i.
  __device__ __forceinline__ static void exchange(uint32_t (&w)[16], bool back) {
    auto halves = [&] {
      if (ItemSize<DT>::value != 2) return;
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        swap32(w[i], w[i + 2]);
        swap32(w[i + 1], w[i + 3]);
      }
    };
    auto rows16 = [&] {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        swap16(w[i], w[4 + i]);
        swap16(w[8 + i], w[12 + i]);
      }
    };
    auto rows8 = [&] {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        swap8(w[i], w[8 + i]);
        swap8(w[4 + i], w[12 + i]);
      }
    };
    if (!back) {
      halves();
      rows16();
      rows8();
    } else {
      rows8();
      rows16();
      halves();
    }
  }
  struct Pieces { u32x4 v[4]; };
  // A group's pieces of results v, element 16 t + 4 j + i.  Pieces 1 and 2 come out of the exchanges in each other's place.
  __device__ __forceinline__ static Pieces pack(const float (&v)[16 * kGroupTiles]) {
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (ItemSize<DT>::value == 2) w[i] = f32_to_bf16_pair(v[2 * i], v[2 * i + 1]);
      else w[i] = __float_as_uint(v[i]);
    }
    exchange(w, false);
    Pieces x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i % 2 * 2 + i / 2] = (u32x4){w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    return x;
  }
  // STREAM: the lines are not kept in the caches.
  template <bool STREAM = false> __device__ __forceinline__ static void put(const Lines& l, int g, int u, const Pieces& x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) __builtin_amdgcn_raw_buffer_store_b128(x.v[i], l.buffer, (int)piece_at(l, g, u, i), 0, STREAM ? 2 : 0);
  }
  __device__ __forceinline__ static Pieces get(const Lines& l, int g, int u) {
    Pieces x;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(l.buffer, (int)piece_at(l, g, u, i), 0, 0));
    return x;
  }
  __device__ __forceinline__ static void spread(const Pieces& x, float (&v)[16 * kGroupTiles]) {
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = x.v[i / 4 % 2 * 2 + i / 8][i % 4];
    exchange(w, true);
#pragma unroll
    for (int i = 0; i < 16 * kGroupTiles; ++i) {
      if constexpr (ItemSize<DT>::value == 2) v[i] = __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
      else v[i] = __uint_as_float(w[i]);
    }
  }
  __device__ __forceinline__ void results(int g, int u, float (&v)[16 * kGroupTiles]) const {
#pragma unroll
    for (int i = 0; i < 16 * kGroupTiles; ++i) v[i] = acc[g * kGroupTiles + i / 16][u][i % 16];
  }
  // Four elements for each j of tile t from a line (bias); behind its end zeros.
  struct Fours { uint32_t v[4][4 / kItemsPerWord]; };
  __device__ __forceinline__ static Fours get_line(const char* line, int np, int t) {
    const int lane = (int)threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const __amdgpu_buffer_rsrc_t buffer = __builtin_amdgcn_make_buffer_rsrc((void*)line, 0, np * ItemSize<DT>::value, 0x00020000);
    Fours x;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = (wave % WP * TP * 32 + 32 * t + 8 * j + 4 * (lane / 32)) * ItemSize<DT>::value;
      if constexpr (ItemSize<DT>::value == 2) {
        const u32x2 q = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(buffer, at, 0, 0));
        x.v[j][0] = q[0];
        x.v[j][1] = q[1];
      } else {
        const u32x4 q = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(buffer, at, 0, 0));
#pragma unroll
        for (int i = 0; i < 4; ++i) x.v[j][i] = q[i];
      }
    }
    return x;
  }
  __device__ __forceinline__ static float four(const Fours& x, int i) {
    const uint32_t w = x.v[i / 4][i % 4 / kItemsPerWord];
    return __uint_as_float(ItemSize<DT>::value == 4 ? w : i % 2 ? w & 0xffff0000u : w << 16);
  }
};

// Tiles of a workgroup out of `total`: workgroups go round the 8 XCDs, each XCD has a run of consecutive tiles, dealt to its
// workgroups one by one, so that what neighbouring tiles share is fetched into one L2.
struct Share { int first, end, step; };
__device__ __forceinline__ Share share_of_block(int total) {
  const int xcd = (int)(blockIdx.x % 8), mine = (int)(blockIdx.x / 8), blocks = (int)(gridDim.x / 8);
  const int per = total / 8, more = total % 8;                // the first `more` XCDs have one tile more
  const int first = xcd * per + min(xcd, more);
  return {first + mine, first + per + (xcd < more ? 1 : 0), blocks};
}

// A tile as Tile::run takes it.
struct PlaceOfRows {
  const char *p, *q, *w_scales, *x_scales;
  int np, nq, K, chunk, expert, first, p0;
  __device__ __forceinline__ int chunks() const { return max((K + chunk - 1) / chunk, 1); }
  __device__ __forceinline__ static PlaceOfRows none(const PlaceOfRows& like) {
    PlaceOfRows x = like;
    x.np = x.nq = x.K = 0;
    return x;
  }
};

// x W_e^T + b_e through the activation; OT: type of x and W, DT: of the rest.
template <typename OT, typename DT, typename TILE, int BP, int BQ> struct ForwardJob {
  typedef PlaceOfRows Place;
  static constexpr bool kSums = false;
  static constexpr int kItem = ItemSize<DT>::value;
  const char *x, *w, *x_scales, *w_scales, *bias;
  char *pre, *out;
  int d_in, d_out, act, ptiles;
  const RowTiles& tiles;

  static constexpr bool kScaled = std::is_same<OT, MX4>::value;
  __device__ __forceinline__ int line() const { return kScaled ? d_in / 2 : d_in * ItemSize<OT>::value; }   // bytes of a row
  __device__ __forceinline__ uint32_t p_stride() const { return line(); }
  __device__ __forceinline__ uint32_t q_stride() const { return line(); }
  __device__ __forceinline__ uint32_t s_stride() const { return d_in / 32; }
  template <bool AGAIN> __device__ __forceinline__ TileEntry entry(int n) const {
    const RowTile t = tiles.template tile<AGAIN>(n, ptiles);
    return {{t.expert, t.first, t.rows, t.column * BP, 0}};
  }
  __device__ __forceinline__ Place place(const TileEntry& t) const {
    const int expert = t.v[0], first = t.v[1], nq = t.v[2], p0 = t.v[3];
    const int64_t column = (int64_t)expert * d_out + p0;
    return {w + column * line(), x + (int64_t)first * line(), kScaled ? w_scales + column * s_stride() : nullptr,
            kScaled ? x_scales + (int64_t)first * s_stride() : nullptr, min(BP, d_out - p0), nq, kScaled ? d_in / 2 : d_in,
            TILE::OpP::kChunk, expert, first, p0};
  }
  __device__ __forceinline__ bool sums(const Place&) const { return false; }
  __device__ __forceinline__ bool twice() const { return !kScaled && pre != nullptr; }
  template <int ACT, bool KEEP> __device__ __forceinline__ void store(const Place& at, const TILE& tile) const {
    const int64_t first = ((int64_t)at.first * d_out + at.p0) * kItem;
    const typename TILE::Lines o = TILE::lines(out + first, (uint32_t)d_out * kItem, at.nq, at.np);
    const typename TILE::Lines k = TILE::lines((KEEP ? pre : out) + first, (uint32_t)d_out * kItem, at.nq, at.np);
    // all loads in front of the stores: operations count as done in their order, and a load behind a store would wait until
    // that has reached memory (they wait for the next tile's first loads, which are in front of them)
    typename TILE::Fours b[TILE::TP] = {};
    if (bias) {
#pragma unroll
      for (int t = 0; t < TILE::TP; ++t) b[t] = TILE::get_line(bias + ((int64_t)at.expert * d_out + at.p0) * kItem, at.np, t);
      asm volatile("" : : : "memory");
    }
#pragma unroll
    for (int g = 0; g < TILE::kGroups; ++g) {
#pragma unroll
      for (int u = 0; u < TILE::TQ; ++u) {
        float v[16 * TILE::kGroupTiles];
        tile.results(g, u, v);
#pragma unroll
        for (int i = 0; i < 16 * TILE::kGroupTiles; ++i) v[i] += TILE::four(b[g * TILE::kGroupTiles + i / 16], i % 16);
        if (KEEP) TILE::put(k, g, u, TILE::pack(v));
#pragma unroll
        for (int i = 0; i < 16 * TILE::kGroupTiles; ++i) v[i] = activate<DT>(v[i], ACT);
        // Streaming stores of 4-bit products, which write many times what they read: 1024 -> 4096 columns, 131072 rows of 64 experts,
        // 2048 each, 573 -> 416 us, 16384 rows of 32 61 -> 60, 2048 of 16 17 -> 15; a kernel that reads the results next takes as
        // much longer as they gain, or less.  bf16 products: 1264 and 1277 us, 1027 and 1031, 180 and 175.
        TILE::template put<kScaled>(o, g, u, TILE::pack(v));
      }
    }
  }
  template <int ACT> __device__ __forceinline__ void store(const Place& at, const TILE& tile) const {
    if (!kScaled && pre) store<ACT, !kScaled>(at, tile);
    else store<ACT, false>(at, tile);
  }
  __device__ __forceinline__ void finish(const Place& at, const TILE& tile) const {
    if (act == LSHMOE_ACT_RELU) store<LSHMOE_ACT_RELU>(at, tile);
    else if (act == LSHMOE_ACT_GELU) store<LSHMOE_ACT_GELU>(at, tile);
    else store<LSHMOE_ACT_NONE>(at, tile);
  }
};

template <typename OT, typename DT, typename TILE, int BP, int BQ>
__global__ __launch_bounds__(TILE::kThreads, 2) void forward_kernel(const char* __restrict__ x, const char* __restrict__ w,
                                                                    const char* __restrict__ x_scales,
                                                                    const char* __restrict__ w_scales,
                                                                    const char* __restrict__ bias,
                                                                    const int32_t* __restrict__ offsets, int rows, int d_in,
                                                                    int d_out, int E, int act, char* __restrict__ pre,
                                                                    char* __restrict__ out) {
  const RowTiles tiles(offsets, E, rows, BQ);
  const int ptiles = (d_out + BP - 1) / BP;
  const ForwardJob<OT, DT, TILE, BP, BQ> job = {x, w, x_scales, w_scales, bias, pre, out, d_in, d_out, act, ptiles, tiles};
  const Share s = share_of_block(tiles.total * ptiles);
  TILE tile;
  tile.run(job, s.first, s.end, s.step);
}

constexpr int kUnits = 256;   // compute units

// Tiles: 256 x 256 by 8 waves, one workgroup to a compute unit, or 128 x 128 by 4 waves, two of them (binary32 always).
struct Large { static constexpr int BP = 256, BQ = 256, WP = 2, WQ = 4, kPerUnit = 1; };
struct Small { static constexpr int BP = 128, BQ = 128, WP = 2, WQ = 2, kPerUnit = 2; };

// Both rules go by the rows of the call's buffer: how many of them belong to experts is known to the device only.
//
// Small tiles where a call has at most 128 rows per expert on average or fewer large tiles than compute units (1024 -> 4096 columns
// of 16 experts: 2048 rows 28.7 us and 34 on large tiles, 4096 rows 43.3 and 39.5; 4 bits 14.5 and 17.9, 23.6 and 21.1;
// 512 -> 512 columns of 8 experts, 16384 rows, 4 bits: 10.9 and 14.1; with work enough large ones are 20 % faster).
inline bool small_tiles(int64_t rows, int E, int columns) {
  return rows <= 128 * (int64_t)E || (uint64_t)most_row_tiles(rows, E, Large::BQ) * ((columns + Large::BP - 1) / Large::BP) < (uint64_t)kUnits;
}

// Waves that read the weights for themselves (product_direct.h) where a call has at most `few` rows per expert on average and no more
// small tiles than run at a time (16 experts, 74 rows: 768 -> 2048 columns 13.1 and 13.9 us on tiles, 2048 -> 768 13.1 and
// 22.9; 4 bits 9.1 and 10.5, 9.0 and 11.6; 256 rows 15.6 and 13.8; 64 experts, 256 rows, 1024 -> 4096 columns 100 and 96, 4 bits
// 47 and 33).
inline bool few_rows(int64_t rows, int E, int columns, int few) {
  return rows <= few * (int64_t)E && (uint64_t)most_row_tiles(rows, E, Small::BQ) * ((columns + Small::BP - 1) / Small::BP) <=
                                         (uint64_t)kUnits * Small::kPerUnit;
}

// More than 64 KB of LDS has to be asked for, once per kernel and device; asking again is harmless.
template <typename K> hipError_t allow_lds(K kernel, size_t bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

// Workgroups for at most this many tiles: as many as run at a time, a multiple of the 8 XCDs.
inline uint32_t blocks_for(uint64_t tiles, int per_unit) {
  const uint64_t most = (uint64_t)kUnits * per_unit, want = (tiles + 7) / 8 * 8;
  return (uint32_t)(want < most ? want : most);
}

}  // namespace

}  // namespace lshmoe
