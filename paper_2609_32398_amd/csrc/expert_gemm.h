// The product grouped by expert.
//
// D[p][q] = sum_k P[p][k] Q[q][k], where p runs along a row of the output, so
// that a lane's accumulators are consecutive elements of one output row.  Three
// directions share the kernel; they differ in where k lies in each operand:
//
//   forward          y[r][o]  = sum_i W[e][o][i] x[r][i]    P = W[e] (k inner), Q = rows (k inner)
//   data gradient    dx[r][i] = sum_o W[e][o][i] dy[r][o]   P = W[e] (k outer), Q = rows (k inner)
//   weight gradient  dW[e][o][i] = sum_r x[r][i] dy[r][o]   P = x (k outer), Q = dy (k outer)
//
// A block takes tiles of BP x BQ outputs, one after the other: tile t of the
// list (expert by expert, its row tiles, their column tiles) belongs to one of
// eight contiguous parts of the list, one for each XCD (blocks b and b + 8 share
// an XCD and its L2), and the blocks of an XCD take its tiles in turn.  So the
// blocks that run at one time on an XCD share an expert's weights and a few row
// tiles.  The experts' row counts are read on the device.
//
// A stage is 128 bytes of k for an operand row (k inner), or that many rows of k
// (k outer), in LDS, double buffered: while a stage is multiplied the next one is
// loaded, across tiles too.  Half of the waves, one on each SIMD, issue all loads
// of a stage (both of a two-wave block's): the vector cache holds no more than 32 KiB on their way, so that
// the issue of a stage's 64 KiB takes about half of its time, in which the other
// wave of the SIMD multiplies.
// A 16-byte piece of a stage lies at a place XOR-ed with its row, so that the
// matrix operands are read from LDS without bank conflicts; the loads that go
// straight to LDS write it in lane order, so it is the global address of each
// lane that is permuted.
//
// 65,536 tokens of 8 of 128 experts (524,288 rows), bf16: 768 -> 2,048 in 1,660 to
// 1,700 us (970 to 990 TFLOP/s), its rows' gradient from 1,536 in 3,140 us (1,050), weight
// gradient of 1,536 x 2,048 in 3,460 to 3,640 us (910 to 950), 2,048 -> 2 x 768 with the
// gated activation and its checkpoint in 3,300 to 3,380 us (980 to 1,000).  The matrix
// cores are busy 55 % of the time at the clock of about 2 GHz that they leave; the rest is
// the loads' way to LDS (a stage that the L2 cache misses takes 1.4 us, one that it holds
// 0.63, its products 1.0) and the outputs at a tile's end.  fp32, 49,146 rows 1,536 ->
// 1,024 transposed: 1,260 us, 123 of the 155 TFLOP/s of a large matrix product.
#pragma once

#include <atomic>
#include <type_traits>

#include "experts.h"

namespace dol {
namespace expert {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
#define DOL_LDS __attribute__((address_space(3)))

enum { kInner = 0, kOuter = 1 };  // where the contraction lies in an operand's rows
enum { kElements = 0, kPieces = 1, kWidePieces = 2 };  // how the operands are loaded
enum { kStore = 0, kWeightGrad = 1, kSwiglu = 2, kSwigluGrad = 3 };

constexpr int kStageBytes = 128;  // of k for one operand row
constexpr size_t kLdsBytes = 160 << 10;  // of a CU
constexpr int kList = 1024;       // tokens of a list in LDS
constexpr int kPhases = 4;        // of a stage: a quarter of its k each

// Tile of BP x BQ outputs by WP x WQ waves.
template <int BP_, int BQ_, int WP_, int WQ_, int OCC_>
struct Tile {
  static constexpr int BP = BP_, BQ = BQ_, WP = WP_, WQ = WQ_;
  static constexpr int waves = WP * WQ, threads = waves * kWave;
  static constexpr int loaders = waves == 2 ? threads : threads / 2;  // threads that load
  static constexpr int MP = BP / WP / 32, MQ = BQ / WQ / 32;  // 32 x 32 matrix tiles of a wave
  static constexpr int stage = (BP + BQ) * kStageBytes;
  static constexpr int occ = OCC_;  // waves per SIMD to leave registers for
  static_assert(MP % 2 == 0, "a wave's outputs go out 64 wide: a gate and an up tile, or 128 bytes of bf16");
  static_assert(stage / waves >= 4096, "the area of a wave's outputs on their way out");
};
using Big = Tile<256, 256, 4, 2, 2>;
using Small = Tile<128, 64, 2, 2, 2>;
using Few = Tile<128, 32, 2, 1, 2>;

template <typename T>
struct Mma;
template <>
struct Mma<uint16_t> {
  static constexpr int kElems = 8;  // elements of a 16-byte piece
  using Frag = v8bf;
  static __device__ __forceinline__ v16f mul(Frag a, Frag b, v16f c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <>
struct Mma<float> {
  static constexpr int kElems = 4;
  using Frag = v4f;
  // four products of two k each: lanes 0-31 hold one 16-byte piece of k, lanes 32-63 the next
  static __device__ __forceinline__ v16f mul(Frag a, Frag b, v16f c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

// 16 bytes per lane from base (uniform) + off straight to LDS, lane after lane
// from byte address lds + place (uniform).  The statements name no memory: the
// place written is in a stage that no wave reads before a later wave_barrier,
// and volatile statements keep their order.
template <int place>
__device__ __forceinline__ void load_to_lds(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3" ::"s"(lds), "n"(place), "v"(off),
               "s"(base)
               : "scc");
}
template <int place>
__device__ __forceinline__ void load_to_lds(const void* src, uint32_t lds) {
  asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off" ::"s"(lds), "n"(place), "v"(src)
               : "scc");
}
// The same with 4 bytes per lane.
__device__ __forceinline__ void word_to_lds(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(src));
}

// All but the last `newest` of this wave's loads and stores are done (they are
// counted in order).
template <int newest>
__device__ __forceinline__ void wait_memory() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(newest) : "memory");
}
// The wave's LDS accesses are done; then all waves meet.
__device__ __forceinline__ void wave_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// XOR pattern of a k-inner row's eight pieces: any eight or sixteen neighbouring
// rows read at one piece touch different banks.
__host__ __device__ __forceinline__ int inner_swizzle(int row) { return (row ^ (row >> 3 & 1)) & 7; }

// XOR pattern of the 16-byte pieces of k-outer rows, the same for all rows of a
// thread: four neighbouring k of a transposed read (bf16) go to different banks.
// fp32 operands are read 4 bytes a lane, two lanes to a bank, which its matrix
// instructions hide.
template <typename T, int DIM>
__host__ __device__ __forceinline__ int outer_swizzle(int k) {
  return sizeof(T) == 2 ? (4 * (k & 3)) & (DIM * 2 / 16 - 1) : 0;
}

// A pointer that is the same in all lanes, in scalar registers.
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const char*>(((uint64_t)hi << 32) | lo);
}

// Token t of those up to `last`: an index out of range counts as the nearest one in it.
__host__ __device__ __forceinline__ int32_t clip_token(int32_t t, int32_t last) { return max(0, min(t, last)); }

// Stages of a contraction of `have` (rows of an expert, or elements of a row).  None where there is nothing to
// add up: an expert without rows may begin past the operands' last row, so not even its first row is there.
template <typename T>
__host__ __device__ __forceinline__ int stages(int have) {
  constexpr int KS = kStageBytes / (int)sizeof(T);
  return (have + KS - 1) / KS;
}

// The lane, as a value that is only known here: what is computed from it is not
// moved out of the loop to occupy registers throughout the kernel.
__device__ __forceinline__ int here(int lane) {
  asm volatile("" : "+v"(lane));
  return lane;
}

// f(0), f(1), .. f(N - 1) with constant arguments.
template <int N, typename F>
__device__ __forceinline__ void each(F&& f) {
  if constexpr (N > 0) {
    each<N - 1>(f);
    f(std::integral_constant<int, N - 1>{});
  }
}

// Loads one operand's stages into LDS, whole 16-byte pieces straight from global
// memory.  DIM operand rows (k inner) or columns (k outer).  A piece's address is
// a uniform base, which moves with the stage, and an offset: 32 bits of bytes, or
// of pieces where rows taken by token span 4 GiB or more (WIDE).  A thread's
// pieces lie a uniform distance apart, so that one offset does for all (and a
// limit, where a tile ends short); only rows taken by token (GATHER) have an
// offset each.  The last stage of a contraction may be short: the pieces past its
// end are loaded from a place inside it, and once they have arrived their thread
// writes zeros over them (clear).
template <typename T, int LAYOUT, int DIM, int THREADS, bool WIDE, bool GATHER>
struct PieceLoader {
  static constexpr int EL = Mma<T>::kElems;
  static constexpr int KS = kStageBytes / (int)sizeof(T);     // k of a stage
  static constexpr int N = DIM * kStageBytes / 16 / THREADS;  // pieces per thread
  static constexpr int PR = LAYOUT == kInner ? kStageBytes / 16 : DIM / EL;  // pieces of an LDS row
  static constexpr int RS = THREADS / PR;                     // LDS rows between a thread's pieces
  static constexpr uint32_t kUnit = WIDE ? EL : 1, kBytes = WIDE ? 1 : sizeof(T);  // elements / kUnit * kBytes: offsets
  // a thread's pieces share their XOR
  static_assert(LAYOUT == kInner ? RS % 16 == 0 : kWave % PR == 0 && (sizeof(T) == 4 || RS % 4 == 0));
  const char* base;  // of the stage
  int64_t step;      // bytes to the next stage
  int32_t left;      // k from the stage's first on
  uint32_t ldo;      // offset from row to row
  // k inner, by token: the pieces' offsets.  Else the first one's, and the largest (k inner) or that of
  // its column in the stage's first row (k outer).
  uint32_t off[LAYOUT == kInner && GATHER ? N : 1], lim;
  // k outer, by token: the tokens come through LDS, kList of them at a time in two lists
  const int32_t* token;
  int32_t last;        // last row of the gathered operand
  const int32_t* list;
  uint32_t list_lds;   // its LDS byte address
  int32_t pos, K;      // first k of the stage
  int32_t turn = 0;    // the list in use

  static __host__ __device__ __forceinline__ int row(int tid) { return tid / PR; }
  static __host__ __device__ __forceinline__ int piece(int tid) {
    const int slot = tid % PR;
    if constexpr (LAYOUT == kInner)
      return slot ^ inner_swizzle(row(tid));
    else
      return slot ^ outer_swizzle<T, DIM>(row(tid));
  }
  // the first k of a thread's piece in its stage
  static __host__ __device__ __forceinline__ int first_k(int tid, int j) {
    return LAYOUT == kInner ? piece(tid) * EL : row(tid) + j * RS;
  }
  // k inner, rows by token: rowi(j) is the operand row of the thread's j-th piece
  template <typename F>
  __device__ __forceinline__ void start_rows(int tid, int32_t K_, const T* b, int32_t ld, F&& rowi) {
    begin(K_, b, ld);
    step = kStageBytes;
#pragma unroll
    for (int j = 0; j < N; ++j) off[j] = (uint32_t)rowi(j) * ldo + piece(tid) * EL / kUnit * kBytes;
    shorten(tid);
  }
  // k inner: rows b + (row0 + i) * ld, not past row `end`
  __host__ __device__ __forceinline__ void start_inner(int tid, int32_t K_, const T* b, int32_t ld, int32_t row0, int32_t end) {
    begin(K_, b, ld);
    step = kStageBytes;
    off[0] = (uint32_t)(row0 + row(tid)) * ldo + piece(tid) * EL / kUnit * kBytes;
    lim = (uint32_t)end * ldo + piece(tid) * EL / kUnit * kBytes;
    shorten(tid);
  }
  // k outer: rows b + k * ld (or b + tok[k] * ld), columns col0 .. of `cols`
  __host__ __device__ __forceinline__ void start_outer(int tid, int32_t K_, const T* b, int32_t ld, int32_t col0, int32_t cols,
                                              const int32_t* tok, int64_t last_, const int32_t* lists) {
    begin(K_, b, ld);
    const int c = col0 + piece(tid) * EL;
    lim = (c < cols ? (uint32_t)c : 0u) / kUnit * kBytes;  // a column tile's end: any place inside, the result is dropped
    if constexpr (GATHER) {
      step = 0;
      token = tok;
      last = (int32_t)last_;
      pos = 0;
      list = lists;
      list_lds = (uint32_t)(uintptr_t)(const DOL_LDS char*)(lists);
      fetch(tid);
    } else {
      step = (int64_t)KS * ld * (int)sizeof(T);
      off[0] = (uint32_t)row(tid) * ldo + lim;
    }
  }
  __host__ __device__ __forceinline__ void begin(int32_t K_, const T* b, int32_t ld) {
    base = reinterpret_cast<const char*>(b);
    left = K = K_;
    ldo = (uint32_t)ld / kUnit * kBytes;
  }
  // A short stage, k inner: pieces past the end take the place of the first k.
  __host__ __device__ __forceinline__ void shorten(int tid) {
    if constexpr (LAYOUT == kInner) {
      if (left < KS && first_k(tid, 0) >= left) {
        const uint32_t back = (uint32_t)first_k(tid, 0) / kUnit * kBytes;
        lim -= back;
#pragma unroll
        for (int j = 0; j < (GATHER ? N : 1); ++j) off[j] -= back;
      }
    }
  }
  // The tokens from k = pos on to the other list, which no wave reads since the last barrier: they
  // have arrived at the next one.
  __device__ __forceinline__ void fetch(int tid) {
    turn ^= 1;
    const uint32_t dst = list_lds + turn * kList * 4 + (uint32_t)(tid & ~63) * 4;
#pragma unroll
    for (int i = 0; i < kList / THREADS; ++i)
      word_to_lds(token + max(0, min(pos + tid + i * THREADS, K - 1)),
                  __builtin_amdgcn_readfirstlane(dst + i * THREADS * 4));
  }
  // The offset of piece J of the stage.
  // far: where the rows of piece J lie from those of piece 0 (k inner).
  template <int J>
  __host__ __device__ __forceinline__ uint32_t offset(int tid, uint32_t far, uint32_t up) const {
    uint32_t o;
    if constexpr (LAYOUT == kOuter) {
      if constexpr (GATHER) {
        o = (uint32_t)clip_token(list[turn * kList + (pos & (kList - 1)) + row(tid) + J * RS], last) * ldo + lim;
      } else {
        o = off[0] + J * RS * ldo;
        if (left < KS) o = first_k(tid, J) < left ? o : lim;
      }
    } else if constexpr (GATHER) {
      o = off[J];
    } else {
      o = off[0] + far * ldo;
      o = (o < lim ? o : lim) + up;
    }
    return o;
  }
  // Piece J of the stage to LDS byte address dst (uniform: the wave's place in the operand's stage).
  template <int J>
  __device__ __forceinline__ void load(int tid, uint32_t dst, uint32_t far, uint32_t up) {
    const uint32_t o = offset<J>(tid, far, up);
    if constexpr (WIDE)
      load_to_lds<J * THREADS * 16>(base + (uint64_t)o * 16, dst);
    else
      load_to_lds<J * THREADS * 16>(uniform(base), o, dst);
  }
  __host__ __device__ __forceinline__ void next(int tid) {
    if constexpr (LAYOUT == kOuter && GATHER) {
      pos += KS;
      if ((pos & (kList - 1)) == 0) fetch(tid);
    }
    base += step;
    left -= KS;
    shorten(tid);
  }
  // Zeros over the pieces past the end of a stage with `have` k, which has arrived.
  static __device__ __forceinline__ void clear(int tid, int have, char* st) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (first_k(tid, j) >= have) *reinterpret_cast<v4u*>(st + (tid + j * THREADS) * 16) = v4u{0u, 0u, 0u, 0u};
  }
};

// The same for rows of any width and alignment, through registers.  A piece is 16
// bytes from wherever its first element lies (global memory takes any alignment),
// elements past the row's end zeroed; only a wave that would read past the
// operand's own end takes its pieces element by element.  The small tile's pieces
// of both operands are in flight together, the large one's four by four, as its
// registers allow.
template <typename T, int LAYOUT, int DIM, int THREADS>
struct ElementLoader {
  static constexpr int EL = Mma<T>::kElems;
  static constexpr int KS = kStageBytes / (int)sizeof(T);
  static constexpr int N = DIM * kStageBytes / 16 / THREADS;
  static constexpr int PR = LAYOUT == kInner ? kStageBytes / 16 : DIM / EL;
  static constexpr int RS = THREADS / PR;
  const T* ptr[LAYOUT == kInner ? N : 1];
  const T* first;  // the operand, and its end
  const T* end;
  int32_t k;       // first k of the thread's next pieces (k inner: of the piece)
  int32_t K;
  int32_t cols;    // k outer: elements of the row from the piece on
  int64_t ld;
  const int32_t* token;
  const T* base;
  int64_t last;

  static __device__ __forceinline__ int row(int tid) { return tid / PR; }
  static __device__ __forceinline__ int piece(int tid) {
    const int slot = tid % PR;
    if constexpr (LAYOUT == kInner)
      return slot ^ inner_swizzle(row(tid));
    else
      return slot ^ outer_swizzle<T, DIM>(row(tid));
  }
  __device__ __forceinline__ void bounds(const void* p, int64_t elements) {
    first = static_cast<const T*>(p);
    end = first + elements;
  }
  template <typename F>
  __device__ __forceinline__ void start_rows(int tid, int32_t K_, const T* b, int32_t ld_, F&& rowi) {
    K = K_;
    k = piece(tid) * EL;
#pragma unroll
    for (int j = 0; j < N; ++j) ptr[j] = b + (int64_t)rowi(j) * ld_ + k;
  }
  __device__ __forceinline__ void start_outer(int tid, int32_t K_, const T* b, int32_t ld_, int32_t col0,
                                              int32_t cols_, const int32_t* tok, int64_t last_, const int32_t*) {
    K = K_;
    k = row(tid);
    ld = ld_;
    token = tok;
    last = last_;
    const int c = col0 + piece(tid) * EL;
    cols = cols_ - c;
    base = b + (cols > 0 ? c : 0);
  }
  // Elements of pieces J .. J + M - 1 of the stage that exist.
  template <int J, int M>
  __device__ __forceinline__ bool count(int* n) const {
    bool part = false;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      if constexpr (LAYOUT == kInner)
        n[i] = K - k;
      else
        n[i] = k + (J + i) * RS < K ? cols : 0;
      part |= n[i] < EL;
    }
    return part;
  }
  // Loads pieces J .. J + M - 1 of the stage, what lies past a row's end with them.
  template <int J, int M>
  __device__ __forceinline__ void fetch(v4u* v) const {
    const T* src[M];
    int n[M];
    count<J, M>(n);
    bool past = first + EL > end;
#pragma unroll
    for (int i = 0; i < M; ++i) {
      if constexpr (LAYOUT == kInner) {
        src[i] = ptr[J + i];
      } else {
        const int kk = k + (J + i) * RS;
        int64_t r = kk;
        if (token != nullptr && kk < K) {
          r = clip_token(token[kk], (int32_t)last);
        }
        src[i] = base + r * ld;
      }
      past |= n[i] > 0 && src[i] + EL > end;
    }
    if (__ballot(past) == 0) {
#pragma unroll
      for (int i = 0; i < M; ++i) __builtin_memcpy(&v[i], n[i] > 0 ? src[i] : first, 16);
    } else {
#pragma unroll
      for (int i = 0; i < M; ++i) {
        v[i] = v4u{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < EL; ++e)
          if (e < n[i]) {
            if constexpr (sizeof(T) == 2)
              v[i][e >> 1] |= (uint32_t)src[i][e] << (16 * (e & 1));
            else
              v[i][e] = __float_as_uint(src[i][e]);
          }
      }
    }
  }
  // Writes them to the stage at dst, zeros past the end.
  template <int J, int M>
  __device__ __forceinline__ void put(int tid, char* dst, v4u* v) const {
    int n[M];
    if (__ballot(count<J, M>(n)) != 0) {
#pragma unroll
      for (int i = 0; i < M; ++i)
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const int bits = min(32, max(0, n[i] * (int)sizeof(T) * 8 - 32 * d));
          v[i][d] &= bits == 32 ? ~0u : (1u << bits) - 1u;
        }
    }
#pragma unroll
    for (int i = 0; i < M; ++i) *reinterpret_cast<v4u*>(dst + (tid + (J + i) * THREADS) * 16) = v[i];
  }
  __device__ __forceinline__ void next(int) {
    k += KS;
    if constexpr (LAYOUT == kInner) {
#pragma unroll
      for (int j = 0; j < N; ++j) ptr[j] += KS;
    }
  }
};

// Reads the matrix operands of a wave from a stage.  A lane's operand of step s
// is one piece of its row: lane l takes row l % 32 and piece 2 s + l / 32.
template <typename T, int LAYOUT, int DIM>
struct Reader {
  static constexpr int EL = Mma<T>::kElems;
  static constexpr int row_bytes = DIM * (int)sizeof(T);
  int off;  // k inner: byte offset of the lane's row; k outer: of the lane's k
  int sw;   // k inner: the row's XOR; k outer: the lane's XOR
  int col;  // k outer: the lane's column

  __device__ __forceinline__ void start(int lane, int base) {
    if constexpr (LAYOUT == kInner) {
      off = (base + (lane & 31)) * kStageBytes;
      sw = (lane >> 5) ^ inner_swizzle(lane & 31);
      col = 0;
    } else if constexpr (sizeof(T) == 2) {
      const int k = 8 * (lane >> 5) + ((lane & 15) >> 2);
      off = k * row_bytes;
      sw = outer_swizzle<T, DIM>(k);
      col = base + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    } else {
      const int k = 4 * (lane >> 5);
      off = k * row_bytes;
      sw = outer_swizzle<T, DIM>(k);
      col = base + (lane & 31);
    }
  }
  __device__ __forceinline__ typename Mma<T>::Frag get(const char* st, int t, int s) const {
    if constexpr (LAYOUT == kInner) {
      return *reinterpret_cast<const typename Mma<T>::Frag*>(st + off + t * 32 * kStageBytes + ((sw ^ (2 * s)) << 4));
    } else if constexpr (sizeof(T) == 2) {
      const int c = col + 32 * t;
      const char* p = st + off + 16 * s * row_bytes + (((c >> 3) ^ sw) << 4) + (c & 7) * 2;
      const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DOL_LDS v4s*)(p));
      const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((DOL_LDS v4s*)(p + 4 * row_bytes));
      typedef short v8s __attribute__((ext_vector_type(8)));
      const v8s r = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(v8bf, r);
    } else {
      const int c = col + 32 * t;
      const char* p = st + off + 8 * s * row_bytes + (((c >> 2) ^ sw) << 4) + (c & 3) * 4;
      v4f r;
#pragma unroll
      for (int j = 0; j < 4; ++j) r[j] = *reinterpret_cast<const float*>(p + j * row_bytes);
      return r;
    }
  }
};

// Between LDS writes and reads of a staging area by other lanes of the wave (in
// both orders): a wave's LDS accesses are executed in order, so only the
// compiler has to keep them so.
__device__ __forceinline__ void wave_fence() { asm volatile("" ::: "memory"); }

__device__ __forceinline__ int32_t clip_rows(int32_t v, int64_t R) {
  return v < 0 ? 0 : ((int64_t)v > R ? (int32_t)R : v);
}

// A wave's staging area in LDS holds 32 rows of 128 bytes, the 16-byte pieces
// XOR-ed with the row: written by the lanes that hold a row's outputs, read back
// as whole rows.
__device__ __forceinline__ char* staged(char* area, int row, int byte) {
  return area + row * 128 + ((((byte >> 4) ^ row) & 7) << 4) + (byte & 15);
}

// Whole pieces of the outputs are stored past the caches, which hold operands that
// other blocks still read (gradients of 65,536 tokens' weights 3,724 -> 3,665 us).
//
// Stores 32 staged rows of n elements (128 bytes of T at most): row i to
// dst + i * ld, rows `rows` and up left out, columns `cols` and up too.
template <typename T>
__device__ __forceinline__ void store_rows(char* area, int lane, T* dst, int64_t ld, int rows, int cols, bool vec) {
  constexpr int EL = 16 / (int)sizeof(T);
  wave_fence();
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i * 8 + (lane >> 3), c = (lane & 7) * EL;
    const v4u v = *reinterpret_cast<const v4u*>(staged(area, row, (lane & 7) * 16));
    if (row < rows && c < cols) {
      T* p = dst + row * ld + c;
      if (vec) {
        __builtin_nontemporal_store(v, reinterpret_cast<v4u*>(p));
      } else {
        union {
          v4u v;
          T el[EL];
        } u;
        u.v = v;
#pragma unroll
        for (int j = 0; j < EL; ++j)
          if (c + j < cols) p[j] = u.el[j];
      }
    }
  }
  wave_fence();
}

// Writes a lane's 16 outputs of one 32 x 32 tile to its staged row: outputs
// 8 b + 4 h + 0..3 (h = lane / 32) are accumulators 4 b + 0..3.
template <typename T>
__device__ __forceinline__ void stage_tile(char* area, int lane, int byte0, const v16f& a) {
  const int row = lane & 31, h = lane >> 5;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<v2u*>(staged(area, row, byte0 + 16 * b + 8 * h)) =
          v2u{bf16_pair(a[4 * b], a[4 * b + 1]), bf16_pair(a[4 * b + 2], a[4 * b + 3])};
    } else {
      *reinterpret_cast<v4f*>(staged(area, row, byte0 + 32 * b + 16 * h)) =
          v4f{a[4 * b], a[4 * b + 1], a[4 * b + 2], a[4 * b + 3]};
    }
  }
}

// A wave's 32 rows x 64 columns of the tile (two matrix tiles) to global rows.
template <typename T>
__device__ __forceinline__ void store_pair(char* area, int lane, const v16f& a0, const v16f& a1, T* dst, int64_t ld,
                                           int rows, int cols, bool vec) {
  if constexpr (sizeof(T) == 2) {
    stage_tile<T>(area, lane, 0, a0);
    stage_tile<T>(area, lane, 64, a1);
    store_rows<T>(area, lane, dst, ld, rows, cols, vec);
  } else {
    stage_tile<T>(area, lane, 0, a0);
    store_rows<T>(area, lane, dst, ld, rows, cols, vec);
    stage_tile<T>(area, lane, 0, a1);
    store_rows<T>(area, lane, dst + 32, ld, rows, cols - 32, vec);
  }
}

// 16 of the 32 rows of 64 fp32 outputs (two matrix tiles) in 4 KiB, the 16-byte
// pieces XOR-ed with the row.
__device__ __forceinline__ char* staged_wide(char* area, int row, int piece) {
  return area + row * 256 + ((piece ^ row) << 4);
}
__device__ __forceinline__ void stage_wide(char* area, int lane, int half, const v16f& a0, const v16f& a1) {
  const int row = lane & 15, h = lane >> 5;
  wave_fence();
  if (((lane >> 4) & 1) == half) {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      *reinterpret_cast<v4f*>(staged_wide(area, row, 2 * b + h)) =
          v4f{a0[4 * b], a0[4 * b + 1], a0[4 * b + 2], a0[4 * b + 3]};
      *reinterpret_cast<v4f*>(staged_wide(area, row, 8 + 2 * b + h)) =
          v4f{a1[4 * b], a1[4 * b + 1], a1[4 * b + 2], a1[4 * b + 3]};
    }
  }
  wave_fence();
}
// Eight outputs from column c (a multiple of 8) of a staged row.
__device__ __forceinline__ void read_wide(char* area, int row, int c, float* v) {
  const v4f lo = *reinterpret_cast<const v4f*>(staged_wide(area, row, c >> 2));
  const v4f hi = *reinterpret_cast<const v4f*>(staged_wide(area, row, (c >> 2) + 1));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = lo[i];
    v[4 + i] = hi[i];
  }
}

// Stores the first n of eight values to d, in 16-byte pieces when vec (then n is 8).
template <typename T>
__device__ __forceinline__ void store_eight(T* d, const float* v, int n, bool vec) {
  if constexpr (sizeof(T) == 2) {
    if (vec) {
      const v4u o{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
      __builtin_nontemporal_store(o, reinterpret_cast<v4u*>(d));
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) d[i] = bf16_bits(v[i]);
  } else {
    if (vec) {
      *reinterpret_cast<v4f*>(d) = v4f{v[0], v[1], v[2], v[3]};
      *reinterpret_cast<v4f*>(d + 4) = v4f{v[4], v[5], v[6], v[7]};
      return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n) d[i] = v[i];
  }
}

// Stores the first n of four values to d, at once when vec (then n is 4).
template <typename T>
__device__ __forceinline__ void store_four(T* d, const v4f& v, int n, bool vec) {
  if constexpr (sizeof(T) == 2) {
    if (vec) {
      const v2u o{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
      __builtin_nontemporal_store(o, reinterpret_cast<v2u*>(d));
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) d[i] = bf16_bits(v[i]);
  } else {
    if (vec) {
      *reinterpret_cast<v4f*>(d) = v;
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) d[i] = v[i];
  }
}

// 1 / (1 + e^-g), the quotient by the hardware's reciprocal (one unit in the last place off at most), the
// exponential by its power of two: about |g| units more.
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

__device__ __forceinline__ float prob_at(const ExpertGemm& g, int64_t i) {
  return g.p_bf16 ? bf16_float(static_cast<const uint16_t*>(g.prob)[i]) : static_cast<const float*>(g.prob)[i];
}

// The routing probability of row r of expert e (1 without probabilities).
__device__ __forceinline__ float row_prob(const ExpertGemm& g, int64_t r, int e) {
  if (g.prob == nullptr) return 1.0f;
  return prob_at(g, (int64_t)clip_token(g.q_token[r], (int32_t)(g.N - 1)) * g.E + e);
}

// LDS beside the stages: lists of tokens (k outer only) and probabilities of a tile's rows.
template <int EPI, bool GP, bool GQ>
constexpr int kLists = EPI == kWeightGrad ? (GP ? 2 : 0) + (GQ ? 2 : 0) : 0;
template <typename C, int EPI>
constexpr int kProbs = EPI == kSwiglu || EPI == kSwigluGrad ? C::BQ : 0;

template <typename T, typename C, int LP, int LQ, int EPI, int LOAD, bool GP, bool GQ>
__global__ __launch_bounds__(C::threads, C::occ) void k_expert_gemm(const ExpertGemm g) {
  extern __shared__ __align__(16) char sm[];  // two stages, token lists, row probabilities, the tile list
  constexpr int KS = kStageBytes / (int)sizeof(T);
  constexpr int BPo = EPI == kSwiglu ? C::BP / 2 : C::BP;  // output columns of a tile
  int32_t* first = reinterpret_cast<int32_t*>(sm + 2 * C::stage);  // [E + 1] first tile of an expert
  int32_t* lists = reinterpret_cast<int32_t*>(sm + 2 * C::stage);  // of tokens, two for each gathered operand
  first += kLists<EPI, GP, GQ> * kList;
  float* probs = reinterpret_cast<float*>(first);  // of a tile's rows
  first += kProbs<C, EPI>;
  int32_t* begin = first + g.E + 1;                                // [E + 1] first row of an expert
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wp = wave % C::WP, wq = wave / C::WP;
  const int PT = (g.Pd + BPo - 1) / BPo;
  const int QT = EPI == kWeightGrad ? (g.Qd + C::BQ - 1) / C::BQ : 0;

  if (wave == 0) {
    int carry = 0;
    for (int e0 = 0; e0 < g.E; e0 += kWave) {
      const int e = e0 + lane;
      int n = 0;
      if (e < g.E) {
        const int b = clip_rows(g.offsets[e], g.R), c = clip_rows(g.offsets[e + 1], g.R);
        begin[e] = b;
        if (e == g.E - 1) begin[g.E] = c;
        if constexpr (EPI == kWeightGrad)
          n = PT * QT;
        else
          n = c > b ? (c - b + C::BQ - 1) / C::BQ * PT : 0;
      }
#pragma unroll
      for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(n, d);
        n += lane >= d ? o : 0;
      }
      if (e < g.E) first[e + 1] = carry + n;
      carry += __builtin_amdgcn_readlane(n, 63);
    }
    if (lane == 0) first[0] = 0;
  }
  __syncthreads();
  const int total = __builtin_amdgcn_readfirstlane(first[g.E]);
  const int xcd = blockIdx.x & 7;
  int tile = (int)((int64_t)total * xcd >> 3) + (int)(blockIdx.x >> 3);
  const int tile_end = (int)((int64_t)total * (xcd + 1) >> 3);
  const int tile_step = (int)(gridDim.x >> 3);
  if (tile >= tile_end) return;

  constexpr bool VEC = LOAD != kElements, WIDE = LOAD == kWidePieces;
  using LoaderP = std::conditional_t<VEC, PieceLoader<T, LP, C::BP, C::loaders, WIDE, GP>, ElementLoader<T, LP, C::BP, C::loaders>>;
  using LoaderQ = std::conditional_t<VEC, PieceLoader<T, LQ, C::BQ, C::loaders, WIDE, GQ>, ElementLoader<T, LQ, C::BQ, C::loaders>>;
  LoaderP lp;
  LoaderQ lq;
  Reader<T, LP, C::BP> rp;
  Reader<T, LQ, C::BQ> rq;
  rp.start(lane, wp * (C::BP / C::WP));
  rq.start(lane, wq * (C::BQ / C::WQ));

  // where a tile's outputs go
  struct Where {
    int32_t e, p0, q0, r0, rows;  // q0: weight gradients; r0, rows: the tile's rows
    int32_t have, nk;             // contraction, its stages
  };
  auto locate = [&](int t) {
    Where w;
    int e = 0;
    for (int e0 = 0; e0 < g.E; e0 += kWave)
      e += __popcll(__ballot(e0 + lane < g.E && first[e0 + lane + 1] <= t));
    e = __builtin_amdgcn_readfirstlane(e);
    w.e = e;
    const int i = t - first[e];
    const int b = begin[e], n = max(0, begin[e + 1] - b);
    w.p0 = __builtin_amdgcn_readfirstlane((i % PT) * BPo);
    if constexpr (EPI == kWeightGrad) {
      w.q0 = __builtin_amdgcn_readfirstlane(i / PT * C::BQ);
      w.r0 = __builtin_amdgcn_readfirstlane(b);
      w.rows = __builtin_amdgcn_readfirstlane(n);
      w.have = w.rows;
    } else {
      w.q0 = 0;
      w.r0 = __builtin_amdgcn_readfirstlane(b + i / PT * C::BQ);
      w.rows = __builtin_amdgcn_readfirstlane(min(C::BQ, n - i / PT * C::BQ));
      w.have = g.K;
    }
    w.nk = stages<T>(w.have);
    if constexpr (EPI != kWeightGrad) w.nk = max(1, w.nk);  // K is 1 at least: a loop with its test at the end
    return w;
  };
  if constexpr (!VEC) {
    // elements of the operands
    if constexpr (EPI == kWeightGrad) {
      lp.bounds(g.P, (GP ? g.N : g.R) * g.ldp);
      lq.bounds(g.Q, (GQ ? g.N : g.R) * g.ldq);
    } else {
      lp.bounds(g.P, (int64_t)g.E * (LP == kOuter ? g.K : (EPI == kSwiglu ? 2 : 1) * g.Pd) * g.ldp);
      lq.bounds(g.Q, (GQ ? g.N : g.R) * g.ldq);
    }
  }
  // the tokens of a thread's rows of a tile, loaded ahead of start()
  struct Tokens {
    int32_t t[LoaderQ::N];
  };
  auto tokens = [&](const Where& w) {
    Tokens k;
    if constexpr (EPI != kWeightGrad && GQ) {
#pragma unroll
      for (int j = 0; j < LoaderQ::N; ++j)
        k.t[j] = g.q_token[w.r0 + min(LoaderQ::row(tid) + j * LoaderQ::RS, w.rows - 1)];
    }
    return k;
  };
  // Rows of P's pieces (k inner): piece j lies far_p(j) rows from piece 0.  The gated activation takes 32
  // gate rows and then the 32 up rows beside them (F rows on) for each wave.
  auto far_p = [](int j) {
    const int i = j * LoaderP::RS;
    return EPI == kSwiglu ? (i >> 6) * 32 + (i & 31) : i;
  };
  auto up_p = [](int j) { return EPI == kSwiglu ? (j * LoaderP::RS >> 5) & 1 : 0; };
  auto start = [&](const Where& w, const Tokens& k) {
    const T* P = static_cast<const T*>(g.P);
    const T* Q = static_cast<const T*>(g.Q);
    if constexpr (EPI == kWeightGrad) {
      const int32_t* pt = GP ? g.p_token + w.r0 : nullptr;
      const int32_t* qt = GQ ? g.q_token + w.r0 : nullptr;
      lp.start_outer(tid, w.rows, pt ? P : P + (int64_t)w.r0 * g.ldp, g.ldp, w.p0, g.Pd, pt, g.N - 1, lists);
      lq.start_outer(tid, w.rows, qt ? Q : Q + (int64_t)w.r0 * g.ldq, g.ldq, w.q0, g.Qd, qt, g.N - 1, lists + (GP ? 2 * kList : 0));
    } else {
      if constexpr (LP == kInner) {
        const T* we = P + (int64_t)w.e * (EPI == kSwiglu ? 2 * g.Pd : g.Pd) * g.ldp;
        if constexpr (VEC)
          lp.start_inner(tid, g.K, we, g.ldp, w.p0, g.Pd - 1);
        else
          lp.start_rows(tid, g.K, we, g.ldp, [&](int j) {
            return min(w.p0 + LoaderP::row(tid) + far_p(j), g.Pd - 1) + up_p(j) * g.Pd;
          });
      } else {
        lp.start_outer(tid, g.K, P + (int64_t)w.e * g.K * g.ldp, g.ldp, w.p0, g.Pd, nullptr, 0, nullptr);
      }
      if constexpr (GQ) {
        const int32_t last = (int32_t)(g.N - 1);
        lq.start_rows(tid, g.K, Q, g.ldq, [&](int j) { return clip_token(k.t[j], last); });
      } else if constexpr (VEC) {
        lq.start_inner(tid, g.K, Q + (int64_t)w.r0 * g.ldq, g.ldq, 0, w.rows - 1);
      } else {
        lq.start_rows(tid, g.K, Q + (int64_t)w.r0 * g.ldq, g.ldq,
                      [&](int j) { return min(LoaderQ::row(tid) + j * LoaderQ::RS, w.rows - 1); });
      }
    }
  };
  const uint32_t wave_lds = (uint32_t)(uintptr_t)(DOL_LDS char*)sm + (uint32_t)(tid & ~63) * 16;

  // The loaders run a stage ahead of the products, through the tiles in the same order.
  const bool loader = tid < C::loaders;
  int load_tile = tile;  // the first one to load
  Where wl;
  Tokens kn;
  // wl: the first tile from t on that has something to load, if there is one (an expert without rows has no
  // stage, though its gradient's tiles are written)
  auto look = [&](int t) {
    if constexpr (EPI == kWeightGrad) {
      while (t < tile_end && (wl = locate(t)).nk == 0) t += tile_step;
    } else if (t < tile_end) {
      wl = locate(t);
      kn = tokens(wl);
    }
    return t;
  };
  wl = locate(tile);
  if constexpr (EPI == kWeightGrad) load_tile = look(tile);
  bool loading = load_tile < tile_end;
  int load_left = wl.nk, load_slot = 0;
  int32_t load_have = wl.have, have = wl.have;  // k from the next stage's first on, and from the last loaded one's
  int next_tile = tile_end;
  if (loader && loading) {
    start(wl, tokens(wl));
    next_tile = look(load_tile + tile_step);
  }
  // piece I of a thread's pieces of the next stage, P's then Q's
  constexpr int kLoads = LoaderP::N + LoaderQ::N;
  auto load = [&](auto which) {
    constexpr int I = decltype(which)::value;
    const int at = load_slot * C::stage + (I < LoaderP::N ? 0 : C::BP * kStageBytes);
    auto one = [&](auto& l, auto piece) {
      constexpr int j = decltype(piece)::value;
      if constexpr (!VEC) {
        if constexpr (j % 4 == 0) {
          v4u v[4];
          l.template fetch<j, 4>(v);
          l.template put<j, 4>(tid, sm + at, v);
        }
      } else if constexpr (I < LoaderP::N) {
        l.template load<j>(tid, __builtin_amdgcn_readfirstlane(wave_lds + at), far_p(j), up_p(j) * g.Pd * l.ldo);
      } else {
        l.template load<j>(tid, __builtin_amdgcn_readfirstlane(wave_lds + at), j * LoaderQ::RS, 0u);
      }
    };
    if constexpr (I < LoaderP::N)
      one(lp, std::integral_constant<int, I>{});
    else
      one(lq, std::integral_constant<int, I - LoaderP::N>{});
  };
  auto load_stage = [&] {
    if (!loading) return;
    if constexpr (!VEC && kLoads <= 12) {
      v4u vp[LoaderP::N], vq[LoaderQ::N];
      char* st = sm + load_slot * C::stage;
      lp.template fetch<0, LoaderP::N>(vp);
      lq.template fetch<0, LoaderQ::N>(vq);
      lp.template put<0, LoaderP::N>(tid, st, vp);
      lq.template put<0, LoaderQ::N>(tid, st + C::BP * kStageBytes, vq);
    } else {
      each<kLoads>([&](auto i) { load(i); });
    }
    load_slot ^= 1;
    have = load_have;
    if (--load_left > 0) {
      lp.next(tid);
      lq.next(tid);
      load_have -= KS;
    } else {
      loading = next_tile < tile_end;
      if (loading) {
        start(wl, kn);
        load_left = wl.nk;
        load_have = wl.have;
        next_tile = look(next_tile + tile_step);
      }
    }
  };
  // Once the loads of the stage in a buffer have arrived: zeros past the end of a short one.
  auto clear = [&](int b) {
    if constexpr (VEC) {
      if (have < KS) {
        LoaderP::clear(tid, have, sm + b * C::stage);
        LoaderQ::clear(tid, have, sm + b * C::stage + C::BP * kStageBytes);
      }
    }
  };

  using Frag = typename Mma<T>::Frag;
  struct Frags {
    Frag p[C::MP], q[C::MQ];
  };
  // the operands of phase s of the stage in a buffer
  auto read = [&](Frags& f, int buf, int s) {
    const char* sp = sm + buf * C::stage;
    const char* sq = sp + C::BP * kStageBytes;
#pragma unroll
    for (int i = 0; i < C::MP; ++i) f.p[i] = rp.get(sp, i, s);
#pragma unroll
    for (int j = 0; j < C::MQ; ++j) f.q[j] = rq.get(sq, j, s);
  };

  if constexpr (kLists<EPI, GP, GQ> > 0) {  // the first lists
    wait_memory<0>();
    wave_barrier();
  }
  if (loader) {
    load_stage();
    __builtin_amdgcn_s_setprio(1);  // it begins to multiply later than the other wave of its SIMD
  }
  int buf = 0;
  for (; tile < tile_end; tile += tile_step) {
    const Where w = locate(tile);
    if constexpr (EPI == kWeightGrad) {
      if (w.nk == 0 && g.accumulate) continue;  // nothing to add
    }
    v16f acc[C::MP][C::MQ];
#pragma unroll
    for (int i = 0; i < C::MP; ++i)
#pragma unroll
      for (int j = 0; j < C::MQ; ++j) acc[i][j] = v16f{};
    auto multiply = [&](const Frags& f) {
#pragma unroll
      for (int j = 0; j < C::MQ; ++j)
#pragma unroll
        for (int i = 0; i < C::MP; ++i) acc[i][j] = Mma<T>::mul(f.p[i], f.q[j], acc[i][j]);
    };
    // A tile's row probabilities: loaded now, by waves that load nothing else where there are some (a wait
    // for them would include all loads before), used after the last stage.
    float prob = 0.0f;
    const int prob_row = tid - (C::threads - C::loaders);
    static_assert(kProbs<C, EPI> <= C::loaders);
    if (kProbs<C, EPI> > 0 && prob_row >= 0 && prob_row < w.rows && prob_row < C::BQ)
      prob = row_prob(g, w.r0 + prob_row, w.e);
    for (int ks = 0; ks < w.nk; ++ks) {
      if (loader) {
        wait_memory<0>();
        clear(buf);
      }
      wave_barrier();
      if (loader) load_stage();
#pragma unroll
      for (int s = 0; s < kPhases; ++s) {
        Frags f;
        read(f, buf, s);
        multiply(f);
      }
      buf ^= 1;
    }
    if (kProbs<C, EPI> > 0 && prob_row >= 0 && prob_row < C::BQ) probs[prob_row] = prob;
    // The stage just used holds the waves' areas once every wave is done with it; it is loaded again
    // only after the next barrier.
    wave_barrier();
    char* area = sm + (buf ^ 1) * C::stage + wave * (C::stage / C::waves);
    const int qw = wq * (C::BQ / C::WQ), pw = wp * (C::BP / C::WP);
    if constexpr (EPI == kStore) {
      T* y = static_cast<T*>(g.out);
#pragma unroll
      for (int ij = 0; ij < C::MP / 2 * C::MQ; ++ij) {
        const int i = ij / C::MQ * 2, j = ij % C::MQ, c = w.p0 + pw + 32 * i, r = qw + j * 32;
        store_pair<T>(area, lane, acc[i][j], acc[i + 1][j], y + (int64_t)(w.r0 + r) * g.Pd + c, g.Pd, w.rows - r,
                      g.Pd - c, g.vec_out);
      }
    } else if constexpr (EPI == kWeightGrad) {
      float* dw = static_cast<float*>(g.out) + (int64_t)w.e * g.Qd * g.Pd;
#pragma unroll
      for (int ij = 0; ij < C::MP / 2 * C::MQ; ++ij) {
        const int i = ij / C::MQ * 2, j = ij % C::MQ, c = w.p0 + pw + 32 * i, r = w.q0 + qw + j * 32;
        float* d = dw + (int64_t)r * g.Pd + c;
        if (g.accumulate) {
          const int row = r + (lane & 31), c0 = c + 4 * (lane >> 5);
          if (row < g.Qd) {
#pragma unroll
            for (int ii = 0; ii < 2; ++ii)
#pragma unroll
              for (int v = 0; v < 16; ++v) {
                const int cc = 32 * ii + 8 * (v >> 2) + (v & 3);
                if (c0 + cc < g.Pd) acc[i + ii][j][v] += dw[(int64_t)row * g.Pd + c0 + cc];
              }
          }
        }
        store_pair<float>(area, lane, acc[i][j], acc[i + 1][j], d, g.Pd, g.Qd - r, g.Pd - c, g.vec_out);
      }
    } else if constexpr (EPI == kSwiglu) {
      // 32 rows at a time: gate and up of 32 activations in fp32 to the staging area, then four
      // lanes take a row, eight activations each (a lane's group of 32 is its four lanes')
      const int F = g.Pd, G = (F + kAct8Group - 1) / kAct8Group;
#pragma unroll
      for (int ij = 0; ij < C::MP / 2 * C::MQ; ++ij) {
        const int j = ij % C::MQ, f0 = w.p0 + pw / 2 + ij / C::MQ * 32;
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
          stage_wide(area, lane, i, acc[ij / C::MQ * 2][j], acc[ij / C::MQ * 2 + 1][j]);
          const int ln = here(lane), c = (ln & 3) * 8, n = min(8, F - f0 - c);
          const int row = ln >> 2, rr = qw + j * 32 + i * 16 + row;
          float a[2][8];
          read_wide(area, row, c, a[0]);
          read_wide(area, row, 32 + c, a[1]);
          const bool live = rr < w.rows;
          const int64_t r = w.r0 + rr;
          const float p = probs[rr];
          float hv[8];
#pragma unroll
          for (int v = 0; v < 8; ++v) hv[v] = p * (a[0][v] * sigmoid(a[0][v])) * a[1][v];
          if (live && n > 0) store_eight<T>(static_cast<T*>(g.out) + r * F + f0 + c, hv, n, g.vec_out);
          if (g.q8 != nullptr) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              uint32_t m = 0;
#pragma unroll
              for (int v = 0; v < 8; ++v) m = max(m, v < n ? __float_as_uint(a[half][v]) & 0x7FFFFFFFu : 0u);
              m = max(m, (uint32_t)__shfl_xor((int)m, 1));
              m = max(m, (uint32_t)__shfl_xor((int)m, 2));
              const uint32_t byte = act8_exponent(m);
              const float inv = act8_inverse(byte);
              const v2u q = v2u{act8_round4(a[half], inv, byte), act8_round4(a[half] + 4, inv, byte)};
              if (live && n > 0) {
                int8_t* d = g.q8 + (r * 2 + half) * F + f0 + c;
                if (g.vec_q8) {
                  *reinterpret_cast<v2u*>(d) = q;
                } else {
#pragma unroll
                  for (int v = 0; v < 8; ++v)
                    if (v < n) d[v] = (int8_t)(q[v >> 2] >> (8 * (v & 3)));
                }
                if (c == 0) g.e8[(r * 2 + half) * G + f0 / 32] = (uint8_t)byte;
              }
            }
          }
        }
      }
    } else {
      // dh = W2^T dy of 64 activations and 16 rows at a time in fp32 to the staging area, with their
      // 8-bit gate and up behind (128 bytes a row, loaded 16 rows ahead); then 16 lanes take a row,
      // four activations each
      const int F = g.Pd, G = (F + kAct8Group - 1) / kAct8Group, parts = (F + 63) / 64;
      const int f0 = w.p0 + pw;
      static_assert(C::MP == 2 && C::stage / C::waves >= 4096 + 2048);
      struct Kept {
        v4u gate, up;
        uint32_t e;  // of row lane / 4: half lane / 2 % 2, group lane % 2
      };
      auto kept = [&](int block) {
        const int ln = here(lane), rr = qw + block * 16 + (ln >> 2), c = f0 + (ln & 3) * 16;
        const int64_t r = w.r0 + rr;
        Kept k{v4u{0u, 0u, 0u, 0u}, v4u{0u, 0u, 0u, 0u}, 0u};
        if (rr < w.rows) {
          const int8_t* q = g.q8 + r * 2 * F + c;
          if (g.vec_q8) {
            if (c < F) {
              k.gate = *reinterpret_cast<const v4u*>(q);
              k.up = *reinterpret_cast<const v4u*>(q + F);
            }
          } else {
#pragma unroll
            for (int v = 0; v < 16; ++v)
              if (c + v < F) {
                k.gate[v >> 2] |= (uint32_t)(uint8_t)q[v] << (8 * (v & 3));
                k.up[v >> 2] |= (uint32_t)(uint8_t)q[F + v] << (8 * (v & 3));
              }
          }
          const int grp = f0 / kAct8Group + (ln & 1);
          if (grp < G) k.e = g.e8[(r * 2 + ((ln >> 1) & 1)) * G + grp];
        }
        return k;
      };
      char* qarea = area + 4096;
      Kept next = kept(0);
#pragma unroll
      for (int j = 0; j < C::MQ; ++j) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const Kept k = next;
          if (j * 2 + half + 1 < C::MQ * 2) next = kept(j * 2 + half + 1);
          stage_wide(area, lane, half, acc[0][j], acc[1][j]);
          *reinterpret_cast<v4u*>(staged(qarea, lane >> 2, (lane & 3) * 16)) = k.gate;
          *reinterpret_cast<v4u*>(staged(qarea, lane >> 2, 64 + (lane & 3) * 16)) = k.up;
          wave_fence();
#pragma unroll 1
          for (int i = 0; i < 4; ++i) {
            const int ln = here(lane), c = (ln & 15) * 4, n = min(4, F - f0 - c);
            const int row = i * 4 + (ln >> 4), rr = qw + j * 32 + half * 16 + row;
            const int64_t r = w.r0 + rr;
            const v4f dh = *reinterpret_cast<const v4f*>(staged_wide(area, row, c >> 2));
            const uint32_t qg = *reinterpret_cast<const uint32_t*>(staged(qarea, row, c));
            const uint32_t qu = *reinterpret_cast<const uint32_t*>(staged(qarea, row, 64 + c));
            const float sg = act8_scale((uint32_t)__shfl((int)k.e, row * 4 + (c >> 5)));
            const float su = act8_scale((uint32_t)__shfl((int)k.e, row * 4 + 2 + (c >> 5)));
            const float p = probs[rr];
            float dp = 0.0f, gate[4], up[4];
            act8_values4(qg, sg, gate);
            act8_values4(qu, su, up);
            v4f dg, du, hv;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
              const float z = sigmoid(gate[v]), sl = gate[v] * z, act = sl * up[v], ds = p * dh[v];
              dp += v < n ? dh[v] * act : 0.0f;
              hv[v] = p * act;
              du[v] = ds * sl;
              dg[v] = ds * up[v] * (z + sl * (1.0f - z));
            }
            if (rr < w.rows && n > 0) {
              T* da = static_cast<T*>(g.out) + r * 2 * F + f0 + c;
              store_four<T>(da, dg, n, g.vec_out);
              store_four<T>(da + F, du, n, g.vec_out);
              store_four<T>(static_cast<T*>(g.out2) + r * F + f0 + c, hv, n, g.vec_out);
            }
            if (g.dp != nullptr && f0 < F) {
              dp += __shfl_xor(dp, 1);
              dp += __shfl_xor(dp, 2);
              dp += __shfl_xor(dp, 4);
              dp += __shfl_xor(dp, 8);
              if ((ln & 15) == 0 && rr < w.rows) g.dp[r * parts + f0 / 64] = dp;
            }
          }
          wave_fence();
        }
      }
    }
  }
}

template <typename T, typename C, int LP, int LQ, int EPI, int LOAD, bool GP = false, bool GQ = false>
hipError_t launch_gemm(const ExpertGemm& g, hipStream_t s) {
  const void* kern = reinterpret_cast<const void*>(k_expert_gemm<T, C, LP, LQ, EPI, LOAD, GP, GQ>);
  auto lds_of = [](int E) {
    return 2 * (size_t)C::stage + (kLists<EPI, GP, GQ> * kList + kProbs<C, EPI>) * 4 + (size_t)(E + 1) * 8;
  };
  // blocks per CU that the registers leave room for, and the kernel's LDS limit: set up once per device
  static std::atomic<int> by_registers[64];
  const DevInfo di = device_info();
  if (di.device < 0 || di.device >= 64) return hipErrorInvalidDevice;
  int occ = by_registers[di.device].load(std::memory_order_acquire);
  if (occ == 0) {
    hipError_t e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds_of(kMaxE));
    if (e != hipSuccess) return e;
    if ((e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&occ, kern, C::threads, 0)) != hipSuccess) return e;
    if (occ < 1) return hipErrorLaunchOutOfResources;
    by_registers[di.device].store(occ, std::memory_order_release);
  }
  const size_t lds = lds_of(g.E);
  occ = std::max(1, std::min<int>(occ, (int)(kLdsBytes / lds)));
  constexpr int BPo = EPI == kSwiglu ? C::BP / 2 : C::BP;
  const int64_t PT = (g.Pd + BPo - 1) / BPo;
  // at most this many tiles (the experts' row counts are only known on the device)
  const int64_t tiles = EPI == kWeightGrad ? (int64_t)g.E * PT * ((g.Qd + C::BQ - 1) / C::BQ)
                                           : PT * (g.R / C::BQ + std::min<int64_t>(g.E, g.R));
  if (tiles >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  const int64_t blocks = std::min<int64_t>((tiles + 7) & ~int64_t(7), (int64_t)occ * di.cu_count & ~int64_t(7));
  hipLaunchKernelGGL((k_expert_gemm<T, C, LP, LQ, EPI, LOAD, GP, GQ>), dim3((unsigned)std::max<int64_t>(8, blocks)),
                     dim3(C::threads), lds, s, g);
  return hipGetLastError();
}

// The tile by its size.  Operands that are not whole pieces go through registers; rows by token
// that span 4 GiB or more take wide offsets, on the small tile.
// GP, GQ: rows of P and Q are taken by token.
enum { kFew = 0, kSmall = 1, kBig = 2 };
template <typename T, int LP, int LQ, int EPI, bool GP = false, bool GQ = false>
hipError_t pick_gemm(const ExpertGemm& g, int size, bool vec, hipStream_t s) {
  if constexpr (GP || GQ) {
    if (vec && g.wide) return launch_gemm<T, Small, LP, LQ, EPI, kWidePieces, GP, GQ>(g, s);
  }
  if constexpr (EPI != kWeightGrad) {
    if (vec && size == kFew) return launch_gemm<T, Few, LP, LQ, EPI, kPieces, GP, GQ>(g, s);
  }
  if constexpr (EPI == kWeightGrad || sizeof(T) == 2) {
    if (size == kBig)
      return vec ? launch_gemm<T, Big, LP, LQ, EPI, kPieces, GP, GQ>(g, s)
                 : launch_gemm<T, Big, LP, LQ, EPI, kElements, GP, GQ>(g, s);
  }
  return vec ? launch_gemm<T, Small, LP, LQ, EPI, kPieces, GP, GQ>(g, s)
             : launch_gemm<T, Small, LP, LQ, EPI, kElements, GP, GQ>(g, s);
}

// Tiles of rows by the experts' rows on average.
//
// 16 or fewer: half as many rows as the small tile, all waves load.  A stage is 20
// KiB, so that a CU's blocks have more of the weights on their way, which bound
// the time (5.4 TB/s of weights).  8 of 64 experts a token, fp32, 768 -> 2,048 and
// gated 2,048 -> 2 x 768, against the small tile: 8 rows an expert 92 and 163 us
// against 125 and 227, 16 rows 114 and 226 against 128 and 232; 32 rows 121 and 286
// against 142 and 283, since half of the experts then need two tiles, 64 rows 221 and
// 428 against 171 and 357.  bf16 gains little, its products being short: 8 of 128
// experts a token, weights from memory, 1 token 13.8 and 31.8 us against 14.4 and 32.9, 16
// tokens 47.7 and 107 against 48.8 and 107.
//
// Large tiles for bf16 where an expert has rows for them, small ones else.  8 of 64
// experts a token, 768 -> 2,048, gated, and the rows' gradient 2,048 -> 768, large
// against small: 96 rows an expert 46, 146 and 51 us against 47, 134 and 55; 128 rows 64,
// 146 and 57 against 55, 129 and 54; 160 rows 66, 151 and 59 against 65, 144 and 62; 256
// rows 75, 198 and 102 against 88, 203 and 85; 512 rows 122, 281 and 138 against 159, 348
// and 178: from 96 to 256 rows neither is ahead everywhere.  fp32's
// matrix instructions take 16 times as long, so that a small tile's loads are
// hidden too, and it wastes less at the end of an expert's rows and of the tile
// list (49,146 rows 1,536 -> 1,024 of 48 experts: 1,298 us against 1,468).
template <typename T>
int tile_size(const ExpertGemm& g) {
  if (few_rows(g.R, g.E)) return kFew;
  return sizeof(T) == 2 && g.R / g.E >= 128 ? kBig : kSmall;
}

}  // namespace expert
}  // namespace dol
