// The experts' products on rows that are grouped by expert: rows expert_offsets[e] .. expert_offsets[e+1] - 1 belong to
// expert e.  The offsets are in device memory, so a launch is sized for the worst case and a workgroup finds its expert
// and its rows from the offsets itself.
//
//   forward      pre = x W_e^T + b_e,  out = act(pre)          W_e [d_out, d_in]
//   input        grad_x = (grad_out W_e) * act'(pre)
//   weight       grad_W_e = grad_out_e^T x_e,  grad_b_e = sum of grad_out_e
//
// All three are out[q][p] = sum_k Q[q][k] P[p][k], p the index that is contiguous in the output:
//   forward      q = row, p = d_out, k = d_in       Q = x, P = W_e, both contiguous in k
//   input        q = row, p = d_in,  k = d_out      Q = grad_out contiguous in k, P = W_e contiguous in p
//   weight       q = d_out, p = d_in, k = row       Q = grad_out contiguous in q, P = x contiguous in p
// The matrix instruction takes P as its first operand: a lane then holds runs of 4 consecutive p of one q.
//
// A workgroup computes a tile of BQ x BP outputs.  k goes by chunks: 128 bytes of every row of an operand that is
// contiguous in k ("rows"), as many k of one that is not ("columns").  Chunks go from memory straight into LDS, into rings of
// three chunks of P and two of Q (160 KB for two workgroups of binary32 or one of bf16), one barrier to a chunk.  A wave
// starts one load per half step, between its products: a chunk's loads all at once fill the address units' queue, and the
// products behind them wait.
#include <type_traits>
#include <utility>

#include "kernels.h"
#include "rows_by_expert.h"

namespace lshmoe {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kChunkBytes = 128;   // of a row per chunk
constexpr int kPieces = kChunkBytes / 16;
constexpr int kSteps = kPieces / 2;   // steps of two 16-byte pieces, one per lane half, per chunk

// Piece s of row i of a chunk of rows lies in slot s ^ row_shift(i): 16 lanes reading a piece of 16 rows cover 256 bytes once.
__device__ __forceinline__ int row_shift(int i) { return i / (256 / kChunkBytes) % kPieces; }

// c += P Q of one step: 8 elements of k (bf16, one instruction of 16 with the other lane half) or 4 (binary32, four of 2).
template <typename DT> __device__ __forceinline__ void mma(const u32x4& a, const u32x4& b, f32x16& c);
template <> __device__ __forceinline__ void mma<BF16>(const u32x4& a, const u32x4& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma<F32>(const u32x4& a, const u32x4& b, f32x16& c) {
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[0]), __uint_as_float(b[0]), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[1]), __uint_as_float(b[1]), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[2]), __uint_as_float(b[2]), c, 0, 0, 0);
  c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[3]), __uint_as_float(b[3]), c, 0, 0, 0);
}

// 16 bytes per lane from a buffer straight into LDS: lane l's piece lands at dst + 16 l (dst is wave-uniform); a lane whose
// offset is behind the buffer's end gets zeros.  Inline assembly, because behind the compiler's own builtin every LDS read
// waits until the load has landed; the caller waits for these loads itself.
__device__ __forceinline__ void load16_to_lds(const i32x4& buffer, uint32_t offset, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %1\n\tbuffer_load_dwordx4 %0, %2, 0 offen lds" : : "v"(offset), "s"(dst), "s"(buffer) : "memory", "m0");
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
template <typename DT, bool COLUMNS, int B, int WAVES> struct Operand {
  static constexpr int kItem = ItemSize<DT>::value;
  static constexpr int kChunk = kChunkBytes / kItem;              // k of a chunk
  static constexpr int kBytes = B * kChunkBytes;                  // LDS of a chunk
  static constexpr int kLoads = kBytes / (1024 * WAVES);          // instructions of a wave per chunk
  static constexpr int kRowPieces = COLUMNS ? B * kItem / 16 : kPieces;   // pieces of a line of LDS
  static_assert(kLoads * 1024 * WAVES == kBytes, "whole instructions");

  const char* base;       // the tile's first element, chunk 0
  int64_t bytes;          // from there to the end of what may be read
  int64_t chunk_step;     // bytes from one chunk to the next
  uint32_t offset[kLoads];
  uint32_t k_piece;       // rows: the lane's piece within the chunk, in bytes

  // element (index i, k) is at first + i * stride + k * item (rows) or first + k * stride + i * item (columns); `indices` of the
  // tile and K of k exist; columns: a line has `line` bytes behind the tile's first index
  __device__ __forceinline__ Operand(const char* first, uint32_t stride, int indices, int64_t K) {
    const int lane = (int)threadIdx.x % 64, wave = (int)threadIdx.x / 64;
    base = first;
    k_piece = 0;
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
    if (COLUMNS) {
      bytes = K == 0 ? 0 : (K - 1) * (int64_t)stride + indices * kItem;
      chunk_step = (int64_t)kChunk * stride;
    } else {
      bytes = indices == 0 ? 0 : (int64_t)(indices - 1) * stride + K * kItem;
      chunk_step = kChunkBytes;
    }
  }

  i32x4 buffer;           // descriptor of the chunk being loaded
  bool cut;               // the lane's piece is behind the end of the rows

  // Prepares the loads of the next chunk; k_bytes: what is left of a row (may be nothing: the loads then bring zeros).
  __device__ __forceinline__ void next(int64_t k_bytes) {
    buffer = buffer_of(base, bytes);
    // the descriptor may come from vector instructions: five cycles before its use
    asm volatile("s_nop 4" : "+s"(buffer));
    cut = !COLUMNS && (int64_t)k_piece >= k_bytes;
    base += chunk_step;
    bytes -= chunk_step;
  }
  // Starts load i of the chunk; lds: where the ring's slot has the wave's first 1024 bytes.
  __device__ __forceinline__ void load(int i, uint32_t lds) const {
    load16_to_lds(buffer, cut ? kNowhere : offset[i], lds + i * WAVES * 1024);
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
template <typename DT, bool COLUMNS, int B, int T> struct Fragments {
  static constexpr int kLine = B * ItemSize<DT>::value;   // columns: bytes of a line
  static constexpr int kAddresses = COLUMNS ? T : kSteps;
  uint32_t at[kAddresses];

  __device__ __forceinline__ explicit Fragments(int first) {
    const int lane = (int)threadIdx.x % 64, r = lane % 32, h = lane / 32;
#pragma unroll
    for (int i = 0; i < kAddresses; ++i) {
      if (!COLUMNS) {
        at[i] = (uint32_t)((first + r) * kChunkBytes + ((2 * i + h) ^ row_shift(r)) * 16);
      } else if (ItemSize<DT>::value == 2) {
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
    if (ItemSize<DT>::value == 2) {
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

template <typename DT, bool P_COLUMNS, bool Q_COLUMNS, int BP, int BQ, int WP, int WQ> struct Tile {
  static constexpr int kWaves = WP * WQ, kThreads = 64 * kWaves;
  static constexpr int TP = BP / WP / 32, TQ = BQ / WQ / 32;     // 32 x 32 tiles of a wave
  typedef Operand<DT, P_COLUMNS, BP, kWaves> OpP;
  typedef Operand<DT, Q_COLUMNS, BQ, kWaves> OpQ;
  static constexpr int kPieceReads = std::is_same<DT, BF16>::value ? 8 : 4;   // bytes that one read of columns gives a lane
  static constexpr int kRingP = 3, kRingQ = 2;                    // chunks in LDS
  static constexpr int kAtQ = kRingP * OpP::kBytes;
  static constexpr size_t kLds = kAtQ + (size_t)kRingQ * OpQ::kBytes;
  static_assert(OpP::kLoads == 4 && OpQ::kLoads == 4 && kSteps == 4 && TP % 2 == 0, "two loads of a chunk to a step");

  f32x16 acc[TP][TQ];
  f32x16 sums[TQ];          // Q summed over k, where wanted

  // K: elements of k.  SUMS: also the sums of Q over k.
  template <bool SUMS> __device__ __forceinline__ void run(OpP& P, OpQ& Q, int64_t K) {
    extern __shared__ uint4 lds[];
    lds_char* const base = (lds_char*)lds;
    const uint32_t lds_at = (uint32_t)(uintptr_t)base;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    const Fragments<DT, P_COLUMNS, BP, TP> fp(wave % WP * TP * 32);
    const Fragments<DT, Q_COLUMNS, BQ, TQ> fq(wave / WP * TQ * 32);
#pragma unroll
    for (int u = 0; u < TQ; ++u) {
#pragma unroll
      for (int t = 0; t < TP; ++t) acc[t][u] = (f32x16){};
      sums[u] = (f32x16){};
    }
    const uint32_t one = std::is_same<DT, BF16>::value ? 0x3f803f80u : 0x3f800000u;
    const u32x4 ones = {one, one, one, one};
    const int chunks = (int)((K + OpP::kChunk - 1) / OpP::kChunk);
    int64_t left_p = K * ItemSize<DT>::value, left_q = left_p;   // bytes of k whose loads are to be started
    uint32_t to_p = lds_at + wave * 1024, to_q = to_p + kAtQ;    // where they go
    int slot_p = 0;                                              // ring slot of the chunk at work
    auto next_p = [&] {
      P.next(left_p);
      left_p -= kChunkBytes;
    };
    auto next_q = [&] {
      Q.next(left_q);
      left_q -= kChunkBytes;
    };
    // Chunks 0 and 1 of Q, 0, 1 and 2 of P.  Chunks behind the last one are loaded like the others (as zeros, without a read),
    // so that the number of loads in flight is always the same.
#pragma unroll
    for (int c = 0; c < kRingP; ++c) {
      if (c < kRingQ) {
        next_q();
#pragma unroll
        for (int i = 0; i < 4; ++i) Q.load(i, to_q + c * OpQ::kBytes);
      }
      next_p();
#pragma unroll
      for (int i = 0; i < 4; ++i) P.load(i, to_p + c * OpP::kBytes);
    }
    u32x4 a[2][TP], b[2][TQ];        // fragments of a step and of the one after it
    asm volatile("s_waitcnt vmcnt(12)" : : : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
#pragma unroll
    for (int t = 0; t < TP; ++t) a[0][t] = fp.read(base, 0, t);
#pragma unroll
    for (int u = 0; u < TQ; ++u) b[0][u] = fq.read(base + kAtQ, 0, u);
    for (int c = 0; c < chunks; ++c) {
      lds_char* const now_p = base + slot_p * OpP::kBytes;
      lds_char* const now_q = base + kAtQ + (c & 1) * OpQ::kBytes;
      const int slot_next = slot_p == kRingP - 1 ? 0 : slot_p + 1;
      lds_char* const next_p_at = base + slot_next * OpP::kBytes;
      lds_char* const next_q_at = base + kAtQ + (~c & 1) * OpQ::kBytes;
      static_for<kSteps>([&](auto sc) {
        constexpr int s = decltype(sc)::value, now = s & 1, then = now ^ 1, sn = (s + 1) % kSteps;
        if (s == kSteps - 1) {
          // The last fragments of chunk c are in registers, this wave's share of chunk c + 1 has landed (P's of chunk c + 2 may be
          // under way).  Behind the barrier that is so for all waves: chunk c's slots are free, chunk c + 1 may be read.
          asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)" : : : "memory");
          __builtin_amdgcn_s_barrier();
          asm volatile("" : : : "memory");
        }
        lds_char* const from_p = s == kSteps - 1 ? next_p_at : now_p;
        lds_char* const from_q = s == kSteps - 1 ? next_q_at : now_q;
        static_for<2>([&](auto hc) {
          constexpr int half = decltype(hc)::value;
          // loads: the first two of Q's chunk c + 2 now, the other two and P's chunk c + 3 in the next chunk's steps 0 to 2
          if (s == 3 && half == 0) next_q();
          if (s == 3) Q.load(half, to_q + (c & 1) * OpQ::kBytes);
          if (s == 0 && c > 0) Q.load(2 + half, to_q + (~c & 1) * OpQ::kBytes);
          if (s == 1 && half == 0 && c > 0) next_p();
          if ((s == 1 || s == 2) && c > 0) P.load(2 * (s - 1) + half, to_p + (slot_p == 0 ? kRingP - 1 : slot_p - 1) * OpP::kBytes);
          __builtin_amdgcn_sched_barrier(0);
          // the fragments of the next step are on their way while this one's products run
#pragma unroll
          for (int t = half * TP / 2; t < (half + 1) * TP / 2; ++t) a[then][t] = fp.read(from_p, sn, t);
#pragma unroll
          for (int u = half * TQ / 2; u < (half + 1) * TQ / 2; ++u) b[then][u] = fq.read(from_q, sn, u);
#pragma unroll
          for (int t = half * TP / 2; t < (half + 1) * TP / 2; ++t)
#pragma unroll
            for (int u = 0; u < TQ; ++u) mma<DT>(a[now][t], b[now][u], acc[t][u]);
          if (SUMS)
#pragma unroll
            for (int u = half * TQ / 2; u < (half + 1) * TQ / 2; ++u) mma<DT>(ones, b[now][u], sums[u]);
          // reads and products take turns
          constexpr int kReads = TP / 2 * (P_COLUMNS ? 16 / kPieceReads : 1) + TQ / 2 * (Q_COLUMNS ? 16 / kPieceReads : 1);
          constexpr int kTurns = TP / 2 * TQ;
          constexpr int kProducts = (kTurns + (SUMS ? TQ / 2 : 0)) * (std::is_same<DT, BF16>::value ? 1 : 4);
          static_for<kTurns>([&](auto i) {
            constexpr int n = decltype(i)::value;
            __builtin_amdgcn_sched_group_barrier(0x100, kReads * (n + 1) / kTurns - kReads * n / kTurns, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, kProducts * (n + 1) / kTurns - kProducts * n / kTurns, 0);
          });
          __builtin_amdgcn_sched_barrier(0);
        });
      });
      slot_p = slot_next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory");   // nothing lands in LDS any more
  }

  // f(q, p, v): a piece's worth of results of q from p on, relative to the tile.  A wave's results go through LDS, binary32, 32 q
  // at a time, so that the 16 bytes that a lane reads and writes of the outputs are next to its neighbours': 256 bytes
  // of an output row at a time instead of 16.  Slots of 16 bytes are moved by the row against bank conflicts.
  template <typename F> __device__ __forceinline__ void finish(F&& f) const {
    constexpr int kElems = Piece<DT>::kElems, kRow = TP * 32 * 4, kLanes = TP * 32 / kElems;
    static_assert(kWaves * 32 * kRow <= (int)kLds && kRow % 256 == 0, "the waves' parts fit");
    extern __shared__ uint4 lds[];
    const int lane = (int)threadIdx.x % 64, r = lane % 32, h = lane / 32;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / 64);
    char* const part = reinterpret_cast<char*>(lds) + wave * 32 * kRow;
    __syncthreads();               // the other waves are done with the last chunk
#pragma unroll
    for (int u = 0; u < TQ; ++u) {
#pragma unroll
      for (int t = 0; t < TP; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *reinterpret_cast<float4*>(part + r * kRow + ((8 * t + 2 * j + h) ^ (r & 15)) * 16) =
              make_float4(acc[t][u][4 * j], acc[t][u][4 * j + 1], acc[t][u][4 * j + 2], acc[t][u][4 * j + 3]);
      __builtin_amdgcn_wave_barrier();
      asm volatile("" : : : "memory");
#pragma unroll
      for (int i = 0; i < 32 * kLanes / 64; ++i) {
        const int q = i * (64 / kLanes) + lane / kLanes, c = lane % kLanes;
        float v[kElems];
#pragma unroll
        for (int j = 0; j < kElems / 4; ++j) {
          const float4 w = *reinterpret_cast<const float4*>(part + q * kRow + ((c * (kElems / 4) + j) ^ (q & 15)) * 16);
          v[4 * j] = w.x; v[4 * j + 1] = w.y; v[4 * j + 2] = w.z; v[4 * j + 3] = w.w;
        }
        f((wave / WP * TQ + u) * 32 + q, wave % WP * TP * 32 + c * kElems, v);
      }
      __builtin_amdgcn_wave_barrier();
      asm volatile("" : : : "memory");
    }
  }
};

// Tile number of a workgroup out of `total`: workgroups go round the 8 XCDs, each XCD gets consecutive tiles, so that what
// neighbouring tiles share is fetched into one L2.  -1: there is none left for it.
__device__ __forceinline__ int64_t tile_of_block(uint64_t block, int64_t total) {
  const int64_t per = (total + 7) / 8, slot = (int64_t)(block / 8), n = (int64_t)(block % 8) * per + slot;
  return slot < per && n < total ? n : -1;
}
inline uint64_t blocks_for(uint64_t tiles) { return (tiles + 7) / 8 * 8; }

template <typename DT, typename TILE, int BP, int BQ>
__global__ __launch_bounds__(TILE::kThreads, 2) void forward_kernel(const char* __restrict__ x, const char* __restrict__ w,
                                                                 const char* __restrict__ bias,
                                                                 const int32_t* __restrict__ offsets, int64_t rows, int d_in,
                                                                 int d_out, int E, int act, char* __restrict__ pre,
                                                                 char* __restrict__ out) {
  constexpr int kItem = ItemSize<DT>::value, kElems = Piece<DT>::kElems;
  const RowTiles tiles(offsets, E, rows, BQ);
  const int ptiles = (d_out + BP - 1) / BP;
  const int64_t n = tile_of_block(linear_block(), tiles.total * ptiles);
  if (n < 0) return;
  const RowTile rt = tiles.find(n, ptiles);
  const int p0 = rt.column * BP, np = min(BP, d_out - p0), nq = (int)min((int64_t)BQ, rt.end - rt.first);
  typename TILE::OpP P(w + ((int64_t)rt.expert * d_out + p0) * d_in * kItem, (uint32_t)d_in * kItem, np, d_in);
  typename TILE::OpQ Q(x + rt.first * d_in * kItem, (uint32_t)d_in * kItem, nq, d_in);
  TILE tile;
  tile.template run<false>(P, Q, d_in);
  tile.finish([&](int q, int p, float (&v)[kElems]) {
    if (q >= nq || p >= np) return;
    if (bias) {
      float b[kElems];
      Piece<DT>::widen(load16(bias + ((int64_t)rt.expert * d_out + p0 + p) * kItem), b);
#pragma unroll
      for (int i = 0; i < kElems; ++i) v[i] += b[i];
    }
    const int64_t at = ((rt.first + q) * d_out + p0 + p) * kItem;
    if (pre) store16(pre + at, Piece<DT>::narrow(v));
    if (act != LSHMOE_ACT_NONE)
#pragma unroll
      for (int i = 0; i < kElems; ++i) v[i] = activate(v[i], act);
    store16(out + at, Piece<DT>::narrow(v));
  });
}

template <typename DT, typename TILE, int BP, int BQ>
__global__ __launch_bounds__(TILE::kThreads, 2) void input_grad_kernel(const char* __restrict__ grad_out,
                                                                    const char* __restrict__ w,
                                                                    const int32_t* __restrict__ offsets, int64_t rows,
                                                                    int d_in, int d_out, int E, int act,
                                                                    const char* __restrict__ pre, char* __restrict__ grad_x) {
  constexpr int kItem = ItemSize<DT>::value, kElems = Piece<DT>::kElems;
  const RowTiles tiles(offsets, E, rows, BQ);
  const int ptiles = (d_in + BP - 1) / BP;
  const int64_t n = tile_of_block(linear_block(), tiles.total * ptiles);
  if (n < 0) return;
  const RowTile rt = tiles.find(n, ptiles);
  const int p0 = rt.column * BP, np = min(BP, d_in - p0), nq = (int)min((int64_t)BQ, rt.end - rt.first);
  typename TILE::OpP P(w + ((int64_t)rt.expert * d_out * d_in + p0) * kItem, (uint32_t)d_in * kItem, np, d_out);
  typename TILE::OpQ Q(grad_out + rt.first * d_out * kItem, (uint32_t)d_out * kItem, nq, d_out);
  TILE tile;
  tile.template run<false>(P, Q, d_out);
  tile.finish([&](int q, int p, float (&v)[kElems]) {
    if (q >= nq || p >= np) return;
    const int64_t at = ((rt.first + q) * d_in + p0 + p) * kItem;
    if (act != LSHMOE_ACT_NONE) {
      float b[kElems];
      Piece<DT>::widen(load16(pre + at), b);
#pragma unroll
      for (int i = 0; i < kElems; ++i) v[i] *= activation_slope(b[i], act);
    }
    store16(grad_x + at, Piece<DT>::narrow(v));
  });
}

template <typename DT, typename TILE, int BP, int BQ>
__global__ __launch_bounds__(TILE::kThreads, 2) void weight_grad_kernel(const char* __restrict__ grad_out,
                                                                     const char* __restrict__ x,
                                                                     const int32_t* __restrict__ offsets, int64_t rows,
                                                                     int d_in, int d_out, int E, char* __restrict__ grad_w,
                                                                     char* __restrict__ grad_bias) {
  constexpr int kItem = ItemSize<DT>::value;
  const int ptiles = (d_in + BP - 1) / BP, qtiles = (d_out + BQ - 1) / BQ;
  const int64_t n = tile_of_block(linear_block(), (int64_t)E * ptiles * qtiles);
  if (n < 0) return;
  const int64_t e = n / ((int64_t)ptiles * qtiles);
  const int p0 = (int)(n % ptiles) * BP, q0 = (int)(n / ptiles % qtiles) * BQ;
  const int np = min(BP, d_in - p0), nq = min(BQ, d_out - q0);
  const RowRange range = rows_of(offsets, (int)e, rows);
  const int64_t K = range.hi - range.lo;
  typename TILE::OpP P(x + (range.lo * d_in + p0) * kItem, (uint32_t)d_in * kItem, np, K);
  typename TILE::OpQ Q(grad_out + (range.lo * d_out + q0) * kItem, (uint32_t)d_out * kItem, nq, K);
  TILE tile;
  const bool sums = grad_bias != nullptr && p0 == 0;
  if (sums)
    tile.template run<true>(P, Q, K);
  else
    tile.template run<false>(P, Q, K);
  tile.finish([&](int q, int p, float (&v)[Piece<DT>::kElems]) {
    if (q < nq && p < np) store16(grad_w + ((e * d_out + q0 + q) * d_in + p0 + p) * kItem, Piece<DT>::narrow(v));
  });
  const int lane = (int)threadIdx.x % 64, wave = (int)threadIdx.x / 64;
  if (sums && wave % (BP / 32 / TILE::TP) == 0 && lane < 32) {
#pragma unroll
    for (int u = 0; u < TILE::TQ; ++u) {
      const int q = (wave / (BP / 32 / TILE::TP) * TILE::TQ + u) * 32 + lane;
      if (q >= nq) continue;
      const float v = tile.sums[u][0];
      if (kItem == 4) reinterpret_cast<float*>(grad_bias)[e * d_out + q0 + q] = v;
      else reinterpret_cast<__bf16*>(grad_bias)[e * d_out + q0 + q] = (__bf16)v;
    }
  }
}

template <typename DT> struct Shape { static constexpr int BP = 256, BQ = 256, WP = 2, WQ = 4; };
template <> struct Shape<F32> { static constexpr int BP = 128, BQ = 128, WP = 2, WQ = 2; };

// More than 64 KB of LDS has to be asked for, once per kernel and device; asking again is harmless.
template <typename K> hipError_t allow_lds(K kernel, size_t bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename DT>
hipError_t forward(const void* x, const void* w, const void* bias, const int32_t* offsets, int64_t rows, int d_in, int d_out,
                   int E, int act, void* pre, void* out, hipStream_t stream) {
  typedef Shape<DT> S;
  typedef Tile<DT, false, false, S::BP, S::BQ, S::WP, S::WQ> TILE;
  auto kernel = forward_kernel<DT, TILE, S::BP, S::BQ>;
  if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
  const uint64_t tiles = (uint64_t)most_row_tiles(rows, E, S::BQ) * ((d_out + S::BP - 1) / S::BP);
  kernel<<<grid_of_blocks(blocks_for(tiles)), TILE::kThreads, TILE::kLds, stream>>>(
      (const char*)x, (const char*)w, (const char*)bias, offsets, rows, d_in, d_out, E, act, (char*)pre, (char*)out);
  return hipGetLastError();
}

template <typename DT>
hipError_t input_grad(const void* grad_out, const void* w, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E,
                      int act, const void* pre, void* grad_x, hipStream_t stream) {
  typedef Shape<DT> S;
  typedef Tile<DT, true, false, S::BP, S::BQ, S::WP, S::WQ> TILE;
  auto kernel = input_grad_kernel<DT, TILE, S::BP, S::BQ>;
  if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
  const uint64_t tiles = (uint64_t)most_row_tiles(rows, E, S::BQ) * ((d_in + S::BP - 1) / S::BP);
  kernel<<<grid_of_blocks(blocks_for(tiles)), TILE::kThreads, TILE::kLds, stream>>>(
      (const char*)grad_out, (const char*)w, offsets, rows, d_in, d_out, E, act, (const char*)pre, (char*)grad_x);
  return hipGetLastError();
}

template <typename DT>
hipError_t weight_grad(const void* grad_out, const void* x, const int32_t* offsets, int64_t rows, int d_in, int d_out, int E,
                       void* grad_w, void* grad_bias, hipStream_t stream) {
  typedef Shape<DT> S;
  typedef Tile<DT, true, true, S::BP, S::BQ, S::WP, S::WQ> TILE;
  auto kernel = weight_grad_kernel<DT, TILE, S::BP, S::BQ>;
  if (hipError_t e = allow_lds(kernel, TILE::kLds); e != hipSuccess) return e;
  const uint64_t tiles = (uint64_t)E * ((d_in + S::BP - 1) / S::BP) * ((d_out + S::BQ - 1) / S::BQ);
  kernel<<<grid_of_blocks(blocks_for(tiles)), TILE::kThreads, TILE::kLds, stream>>>(
      (const char*)grad_out, (const char*)x, offsets, rows, d_in, d_out, E, (char*)grad_w, (char*)grad_bias);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_expert_forward(const void* x, const void* w, const void* bias, const int32_t* offsets, int64_t rows,
                                 int d_in, int d_out, int E, bool bf16, int act, void* pre, void* out, hipStream_t stream) {
  return bf16 ? forward<BF16>(x, w, bias, offsets, rows, d_in, d_out, E, act, pre, out, stream)
              : forward<F32>(x, w, bias, offsets, rows, d_in, d_out, E, act, pre, out, stream);
}

hipError_t launch_expert_input_grad(const void* grad_out, const void* w, const int32_t* offsets, int64_t rows, int d_in,
                                    int d_out, int E, bool bf16, int act, const void* pre, void* grad_x, hipStream_t stream) {
  return bf16 ? input_grad<BF16>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x, stream)
              : input_grad<F32>(grad_out, w, offsets, rows, d_in, d_out, E, act, pre, grad_x, stream);
}

size_t expert_workspace_bytes(int64_t, int, int, int, bool) { return 0; }

hipError_t launch_expert_weight_grad(const void* grad_out, const void* x, const int32_t* offsets, int64_t rows, int d_in,
                                     int d_out, int E, bool bf16, void* grad_w, void* grad_bias, char*, hipStream_t stream) {
  return bf16 ? weight_grad<BF16>(grad_out, x, offsets, rows, d_in, d_out, E, grad_w, grad_bias, stream)
              : weight_grad<F32>(grad_out, x, offsets, rows, d_in, d_out, E, grad_w, grad_bias, stream);
}

}  // namespace lshmoe
