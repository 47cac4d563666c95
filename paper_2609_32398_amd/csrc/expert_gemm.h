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
// (k outer), in LDS, double buffered: while a stage is multiplied the next one
// is loaded, across tiles too.  A 16-byte piece of a stage lies at a place
// XOR-ed with its row, so that the matrix operands are read from LDS without
// bank conflicts; the loads that go straight to LDS write it in lane order, so
// it is the global address of each lane that is permuted.
#pragma once

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
enum { kStore = 0, kWeightGrad = 1, kSwiglu = 2, kSwigluGrad = 3 };

constexpr int kStageBytes = 128;  // of k for one operand row

// Tile of BP x BQ outputs by WP x WQ waves, each 64 x (BQ / WQ).
template <int BP_, int BQ_, int WP_, int WQ_, int OCC_>
struct Tile {
  static constexpr int BP = BP_, BQ = BQ_, WP = WP_, WQ = WQ_;
  static constexpr int waves = WP * WQ, threads = waves * kWave;
  static constexpr int MP = BP / WP / 32, MQ = BQ / WQ / 32;  // 32 x 32 matrix tiles of a wave
  static constexpr int stage = (BP + BQ) * kStageBytes;
  static constexpr int occ = OCC_;  // waves per SIMD to leave registers for
  static_assert(MP == 2, "a wave's outputs are 64 wide: a gate and an up tile, or 128 bytes of bf16");
  static_assert(stage / waves >= 8192, "the epilogue's staging area of a wave");
};
using Big = Tile<256, 256, 4, 2, 2>;
using Small = Tile<128, 128, 2, 2, 2>;

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

// Source of the pieces that lie past an operand's end.
static __device__ const v4u zero_piece = {0u, 0u, 0u, 0u};

__device__ __forceinline__ void load_to_lds(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(src) : "memory");
}
// Every load of this wave has arrived and its LDS accesses are done; then all waves meet.
__device__ __forceinline__ void stage_barrier() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// XOR pattern of the 16-byte pieces of k-outer rows: four neighbouring k of a
// transposed read (bf16), or the two k groups of the half waves (fp32), go to
// different banks.
template <typename T, int DIM>
__device__ __forceinline__ int outer_swizzle(int k) {
  constexpr int pieces = DIM * (int)sizeof(T) / 16;
  if constexpr (sizeof(T) == 2)
    return (4 * (k & 3)) & (pieces - 1);
  else
    return (8 * ((k >> 2) & 1)) & (pieces - 1);
}

// Loads one operand's stages into LDS.  DIM operand rows (k inner) or columns
// (k outer).  VEC: whole 16-byte pieces straight to LDS; else element by
// element through registers, for rows of any width and alignment.
template <typename T, int LAYOUT, int DIM, int THREADS, bool VEC>
struct Loader {
  static constexpr int EL = Mma<T>::kElems;
  static constexpr int KS = kStageBytes / (int)sizeof(T);           // k of a stage
  static constexpr int N = DIM * kStageBytes / 16 / THREADS;        // pieces per thread
  static constexpr int PR = LAYOUT == kInner ? 8 : DIM / EL;        // pieces of an LDS row
  static constexpr int RS = THREADS / PR;                           // LDS rows between a thread's pieces
  const T* ptr[N];
  int32_t k;         // first k of the thread's next pieces (k inner: of the piece)
  int32_t K;
  int32_t left;      // k outer: elements of the row from the piece on
  int64_t step;      // elements to the next stage
  // gathered k-outer rows
  const int32_t* token;
  const T* base;
  int64_t ld;
  int64_t last;      // last row of the gathered operand
  int32_t next[N];

  static __device__ __forceinline__ int row(int tid) { return tid / PR; }
  static __device__ __forceinline__ int piece(int tid) {
    const int slot = tid % PR;
    if constexpr (LAYOUT == kInner)
      return slot ^ (row(tid) & 7);
    else
      return slot ^ outer_swizzle<T, DIM>(row(tid));
  }

  // k inner: rowp(i) is the start of operand row i of the tile
  template <typename F>
  __device__ __forceinline__ void start_inner(int tid, int32_t K_, F&& rowp) {
    K = K_;
    k = piece(tid) * EL;
    step = KS;
#pragma unroll
    for (int j = 0; j < N; ++j) ptr[j] = rowp(row(tid) + j * RS) + k;
  }
  // k outer: rows base + k * ld (or base + token[k] * ld), columns col0 .. of `cols`
  __device__ __forceinline__ void start_outer(int tid, int32_t K_, const T* base_, int64_t ld_, int32_t col0,
                                              int32_t cols, const int32_t* token_, int64_t last_) {
    K = K_;
    k = row(tid);
    ld = ld_;
    step = (int64_t)KS * ld;
    token = token_;
    last = last_;
    int c = col0 + piece(tid) * EL;
    left = cols - c;
    if (left <= 0) c = 0;  // a column tile's end: any valid address, the result is dropped
    base = base_ + c;
    if (token == nullptr) {
#pragma unroll
      for (int j = 0; j < N; ++j) ptr[j] = base + (int64_t)(k + j * RS) * ld;
    } else {
      fetch(0);
    }
  }
  __device__ __forceinline__ void fetch(int ahead) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int kk = k + j * RS + ahead;
      next[j] = kk < K ? token[kk] : 0;
    }
  }

  __device__ __forceinline__ const T* at(int j) const {
    if constexpr (LAYOUT == kOuter) {
      if (token != nullptr) {
        int64_t r = next[j];
        r = r < 0 ? 0 : (r > last ? last : r);
        return base + r * ld;
      }
    }
    return ptr[j];
  }

  // Loads the next stage to LDS byte address dst (its generic pointer: dstp).
  __device__ __forceinline__ void stage(int tid, uint32_t dst, char* dstp) {
    const uint32_t wave_dst = __builtin_amdgcn_readfirstlane(dst + (uint32_t)(tid & ~63) * 16);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int kk = LAYOUT == kInner ? k : k + j * RS;
      const T* src = at(j);
      if constexpr (VEC) {
        const void* from = kk < K ? (const void*)src : (const void*)&zero_piece;
        load_to_lds(from, wave_dst + j * THREADS * 16);
      } else {
        const int n = kk >= K ? 0 : (LAYOUT == kInner ? K - kk : left);  // elements that exist
        union {
          T el[EL];
          v4u v;
        } u;
        u.v = v4u{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < EL; ++i)
          if (i < n) u.el[i] = src[i];
        *reinterpret_cast<v4u*>(dstp + (tid + j * THREADS) * 16) = u.v;
      }
    }
    if constexpr (LAYOUT == kOuter) {
      if (token != nullptr) fetch(KS);
    }
    k += KS;
#pragma unroll
    for (int j = 0; j < N; ++j) ptr[j] += step;
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
      sw = (lane >> 5) ^ (lane & 7);
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

__device__ __forceinline__ int32_t clip_rows(int32_t v, int64_t R) {
  return v < 0 ? 0 : ((int64_t)v > R ? (int32_t)R : v);
}

// A wave's staging area in LDS holds 32 rows of 128 bytes, the 16-byte pieces
// XOR-ed with the row: written by the lanes that hold a row's outputs, read back
// as whole rows.
__device__ __forceinline__ char* staged(char* area, int row, int byte) {
  return area + row * 128 + ((((byte >> 4) ^ row) & 7) << 4) + (byte & 15);
}

// Stores 32 staged rows of n elements (128 bytes of T at most): row i to
// dst + i * ld, rows `rows` and up left out, columns `cols` and up too.
template <typename T>
__device__ __forceinline__ void store_rows(char* area, int lane, T* dst, int64_t ld, int rows, int cols, bool vec) {
  constexpr int EL = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = i * 8 + (lane >> 3), c = (lane & 7) * EL;
    const v4u v = *reinterpret_cast<const v4u*>(staged(area, row, (lane & 7) * 16));
    if (row < rows && c < cols) {
      T* p = dst + row * ld + c;
      if (vec) {
        *reinterpret_cast<v4u*>(p) = v;
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

// 32 rows of 64 fp32 outputs (two matrix tiles) in 8 KiB, the 16-byte pieces
// XOR-ed with the row.
__device__ __forceinline__ char* staged_wide(char* area, int row, int piece) {
  return area + row * 256 + ((piece ^ (row & 15)) << 4);
}
__device__ __forceinline__ void stage_wide(char* area, int lane, const v16f& a0, const v16f& a1) {
  const int row = lane & 31, h = lane >> 5;
#pragma unroll
  for (int b = 0; b < 4; ++b) {
    *reinterpret_cast<v4f*>(staged_wide(area, row, 2 * b + h)) =
        v4f{a0[4 * b], a0[4 * b + 1], a0[4 * b + 2], a0[4 * b + 3]};
    *reinterpret_cast<v4f*>(staged_wide(area, row, 8 + 2 * b + h)) =
        v4f{a1[4 * b], a1[4 * b + 1], a1[4 * b + 2], a1[4 * b + 3]};
  }
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
      *reinterpret_cast<v4u*>(d) =
          v4u{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
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

__device__ __forceinline__ float sigmoid(float g) { return 1.0f / (1.0f + __expf(-g)); }

__device__ __forceinline__ float prob_at(const ExpertGemm& g, int64_t i) {
  return g.p_bf16 ? bf16_float(static_cast<const uint16_t*>(g.prob)[i]) : static_cast<const float*>(g.prob)[i];
}

// The routing probability of row r of expert e (1 without probabilities).
__device__ __forceinline__ float row_prob(const ExpertGemm& g, int64_t r, int e) {
  if (g.prob == nullptr) return 1.0f;
  int64_t t = g.q_token != nullptr ? g.q_token[r] : r;
  t = t < 0 ? 0 : (t >= g.N ? g.N - 1 : t);
  return prob_at(g, t * g.E + e);
}

template <typename T, typename C, int LP, int LQ, int EPI, bool VEC>
__global__ __launch_bounds__(C::threads, C::occ) void k_expert_gemm(const ExpertGemm g) {
  extern __shared__ __align__(16) char sm[];  // two stages, then the tile list
  constexpr int KS = kStageBytes / (int)sizeof(T);
  constexpr int BPo = EPI == kSwiglu ? C::BP / 2 : C::BP;  // output columns of a tile
  int32_t* first = reinterpret_cast<int32_t*>(sm + 2 * C::stage);  // [E + 1] first tile of each expert
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
        if constexpr (EPI == kWeightGrad) {
          n = PT * QT;
        } else {
          n = clip_rows(g.offsets[e + 1], g.R) - clip_rows(g.offsets[e], g.R);
          n = n > 0 ? (n + C::BQ - 1) / C::BQ * PT : 0;
        }
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
  const int total = first[g.E];
  const int xcd = blockIdx.x & 7;
  int tile = (int)((int64_t)total * xcd >> 3) + (int)(blockIdx.x >> 3);
  const int tile_end = (int)((int64_t)total * (xcd + 1) >> 3);
  const int tile_step = (int)(gridDim.x >> 3);
  if (tile >= tile_end) return;

  Loader<T, LP, C::BP, C::threads, VEC> lp;
  Loader<T, LQ, C::BQ, C::threads, VEC> lq;
  Reader<T, LP, C::BP> rp;
  Reader<T, LQ, C::BQ> rq;
  rp.start(lane, wp * 64);
  rq.start(lane, wq * (C::BQ / C::WQ));

  // where a tile's outputs go
  struct Where {
    int32_t e, p0, q0, r0, rows, nk;  // q0: weight gradients; r0, rows: the tile's rows
  };
  auto locate = [&](int t) {
    Where w;
    int e = 0;
    for (int e0 = 0; e0 < g.E; e0 += kWave)
      e += __popcll(__ballot(e0 + lane < g.E && first[e0 + lane + 1] <= t));
    e = __builtin_amdgcn_readfirstlane(e);
    w.e = e;
    const int i = t - first[e];
    const int b = clip_rows(g.offsets[e], g.R), n = max(0, clip_rows(g.offsets[e + 1], g.R) - b);
    w.p0 = __builtin_amdgcn_readfirstlane((i % PT) * BPo);
    if constexpr (EPI == kWeightGrad) {
      w.q0 = __builtin_amdgcn_readfirstlane(i / PT * C::BQ);
      w.r0 = __builtin_amdgcn_readfirstlane(b);
      w.rows = __builtin_amdgcn_readfirstlane(n);
      w.nk = max(1, (w.rows + KS - 1) / KS);
    } else {
      w.q0 = 0;
      w.r0 = __builtin_amdgcn_readfirstlane(b + i / PT * C::BQ);
      w.rows = __builtin_amdgcn_readfirstlane(min(C::BQ, n - i / PT * C::BQ));
      w.nk = (g.K + KS - 1) / KS;
    }
    return w;
  };
  auto start = [&](const Where& w) {
    const T* P = static_cast<const T*>(g.P);
    const T* Q = static_cast<const T*>(g.Q);
    if constexpr (EPI == kWeightGrad) {
      const int32_t* pt = g.p_token ? g.p_token + w.r0 : nullptr;
      const int32_t* qt = g.q_token ? g.q_token + w.r0 : nullptr;
      lp.start_outer(tid, w.rows, pt ? P : P + (int64_t)w.r0 * g.ldp, g.ldp, w.p0, g.Pd, pt, g.N - 1);
      lq.start_outer(tid, w.rows, qt ? Q : Q + (int64_t)w.r0 * g.ldq, g.ldq, w.q0, g.Qd, qt, g.N - 1);
    } else {
      if constexpr (LP == kInner) {
        // the gated activation takes 32 gate rows and the 32 up rows beside them for each wave
        const T* we = P + (int64_t)w.e * (EPI == kSwiglu ? 2 * g.Pd : g.Pd) * g.ldp;
        lp.start_inner(tid, g.K, [&](int i) {
          int64_t row;
          if constexpr (EPI == kSwiglu)
            row = min(w.p0 + (i >> 6) * 32 + (i & 31), g.Pd - 1) + (int64_t)((i >> 5) & 1) * g.Pd;
          else
            row = min(w.p0 + i, g.Pd - 1);
          return we + row * g.ldp;
        });
      } else {
        lp.start_outer(tid, g.K, P + (int64_t)w.e * g.K * g.ldp, g.ldp, w.p0, g.Pd, nullptr, 0);
      }
      lq.start_inner(tid, g.K, [&](int i) {
        int64_t row = w.r0 + min(i, w.rows - 1);
        if (g.q_token != nullptr) {
          row = g.q_token[row];
          row = row < 0 ? 0 : (row >= g.N ? g.N - 1 : row);
        }
        return Q + row * g.ldq;
      });
    }
  };
  const uint32_t sm_lds = (uint32_t)(uintptr_t)(DOL_LDS char*)sm;
  auto load = [&](int buf) {
    lp.stage(tid, sm_lds + buf * C::stage, sm + buf * C::stage);
    lq.stage(tid, sm_lds + buf * C::stage + C::BP * kStageBytes, sm + buf * C::stage + C::BP * kStageBytes);
  };

  Where w = locate(tile);
  start(w);
  int buf = 0;
  load(0);
  for (;;) {
    v16f acc[C::MP][C::MQ];
#pragma unroll
    for (int i = 0; i < C::MP; ++i)
#pragma unroll
      for (int j = 0; j < C::MQ; ++j) acc[i][j] = v16f{};
    tile += tile_step;
    const bool more = tile < tile_end;
    Where wn = w;
    for (int ks = 0; ks < w.nk; ++ks) {
      stage_barrier();
      if (ks + 1 < w.nk) {
        load(buf ^ 1);
      } else if (more) {
        wn = locate(tile);
        start(wn);
        load(buf ^ 1);
      }
      const char* sp = sm + buf * C::stage;
      const char* sq = sp + C::BP * kStageBytes;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        typename Mma<T>::Frag fp[C::MP], fq[C::MQ];
#pragma unroll
        for (int i = 0; i < C::MP; ++i) fp[i] = rp.get(sp, i, s);
#pragma unroll
        for (int j = 0; j < C::MQ; ++j) fq[j] = rq.get(sq, j, s);
#pragma unroll
        for (int i = 0; i < C::MP; ++i)
#pragma unroll
          for (int j = 0; j < C::MQ; ++j) acc[i][j] = Mma<T>::mul(fp[i], fq[j], acc[i][j]);
      }
      buf ^= 1;
    }
    // The stage just used (buf ^ 1) holds the staging areas: every wave is done with it, and the
    // next tile's second stage is loaded into it only after the barrier of its first.
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    char* area = sm + (buf ^ 1) * C::stage + wave * (C::stage / C::waves);
    const int qw = wq * (C::BQ / C::WQ);
    if constexpr (EPI == kStore) {
      T* y = static_cast<T*>(g.out);
#pragma unroll
      for (int j = 0; j < C::MQ; ++j) {
        const int c = w.p0 + wp * 64, r = qw + j * 32;
        store_pair<T>(area, lane, acc[0][j], acc[1][j], y + (int64_t)(w.r0 + r) * g.Pd + c, g.Pd, w.rows - r,
                      g.Pd - c, g.vec_out);
      }
    } else if constexpr (EPI == kWeightGrad) {
      float* dw = static_cast<float*>(g.out) + (int64_t)w.e * g.Qd * g.Pd;
#pragma unroll
      for (int j = 0; j < C::MQ; ++j) {
        const int c = w.p0 + wp * 64, r = w.q0 + qw + j * 32;
        float* d = dw + (int64_t)r * g.Pd + c;
        if (g.accumulate) {
          const int row = r + (lane & 31), c0 = c + 4 * (lane >> 5);
          if (row < g.Qd) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
              for (int v = 0; v < 16; ++v) {
                const int cc = 32 * i + 8 * (v >> 2) + (v & 3);
                if (c0 + cc < g.Pd) acc[i][j][v] += dw[(int64_t)row * g.Pd + c0 + cc];
              }
          }
        }
        store_pair<float>(area, lane, acc[0][j], acc[1][j], d, g.Pd, g.Qd - r, g.Pd - c, g.vec_out);
      }
    } else if constexpr (EPI == kSwiglu) {
      // 32 rows at a time: gate and up of 32 activations in fp32 to the staging area, then four
      // lanes take a row, eight activations each (a lane's group of 32 is its four lanes')
      const int F = g.Pd, G = (F + kAct8Group - 1) / kAct8Group;
      const int f0 = w.p0 + wp * 32, c = (lane & 3) * 8, n = min(8, F - f0 - c);
#pragma unroll
      for (int j = 0; j < C::MQ; ++j) {
        stage_wide(area, lane, acc[0][j], acc[1][j]);
#pragma unroll 1
        for (int i = 0; i < 2; ++i) {
          const int row = i * 16 + (lane >> 2), rr = qw + j * 32 + row;
          float a[2][8];
          read_wide(area, row, c, a[0]);
          read_wide(area, row, 32 + c, a[1]);
          const bool live = rr < w.rows;
          const int64_t r = w.r0 + rr;
          const float p = live ? row_prob(g, r, w.e) : 0.0f;
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
              v2u q = v2u{0u, 0u};
#pragma unroll
              for (int v = 0; v < 8; ++v)
                q[v >> 2] |= ((uint32_t)act8_round(a[half][v], inv, byte) & 255u) << (8 * (v & 3));
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
      // dh = W2^T dy of 64 activations and 32 rows at a time in fp32 to the staging area; then
      // eight lanes take a row, eight activations each, with gate and up from their 8-bit values
      const int F = g.Pd, G = (F + kAct8Group - 1) / kAct8Group;
      const int f0 = w.p0 + wp * 64, c = (lane & 7) * 8, n = min(8, F - f0 - c);
#pragma unroll
      for (int j = 0; j < C::MQ; ++j) {
        stage_wide(area, lane, acc[0][j], acc[1][j]);
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
          const int row = i * 8 + (lane >> 3), rr = qw + j * 32 + row;
          const bool live = rr < w.rows && n > 0;
          const int64_t r = w.r0 + rr;
          float dh[8];
          read_wide(area, row, c, dh);
          float dp = 0.0f;
          if (live) {
            v2u qg = v2u{0u, 0u}, qu = v2u{0u, 0u};
            const int8_t* q = g.q8 + r * 2 * F + f0 + c;
            if (g.vec_q8) {
              qg = *reinterpret_cast<const v2u*>(q);
              qu = *reinterpret_cast<const v2u*>(q + F);
            } else {
#pragma unroll
              for (int v = 0; v < 8; ++v)
                if (v < n) {
                  qg[v >> 2] |= (uint32_t)(uint8_t)q[v] << (8 * (v & 3));
                  qu[v >> 2] |= (uint32_t)(uint8_t)q[F + v] << (8 * (v & 3));
                }
            }
            const uint8_t* eb = g.e8 + r * 2 * G + (f0 + c) / kAct8Group;
            const float sg = act8_scale(eb[0]), su = act8_scale(eb[G]);
            const float p = row_prob(g, r, w.e);
            float dg[8], du[8], hv[8];
#pragma unroll
            for (int v = 0; v < 8; ++v) {
              const float gt = (float)(int8_t)(qg[v >> 2] >> (8 * (v & 3))) * sg;
              const float up = (float)(int8_t)(qu[v >> 2] >> (8 * (v & 3))) * su;
              const float z = sigmoid(gt), sl = gt * z, ds = p * dh[v];
              dp += v < n ? dh[v] * (sl * up) : 0.0f;
              hv[v] = p * (sl * up);
              du[v] = ds * sl;
              dg[v] = ds * up * (z * (1.0f + gt * (1.0f - z)));
            }
            T* da = static_cast<T*>(g.out) + r * 2 * F + f0 + c;
            store_eight<T>(da, dg, n, g.vec_out);
            store_eight<T>(da + F, du, n, g.vec_out);
            store_eight<T>(static_cast<T*>(g.out2) + r * F + f0 + c, hv, n, g.vec_out);
          }
          if (g.dp != nullptr && f0 < F) {
            dp += __shfl_xor(dp, 1);
            dp += __shfl_xor(dp, 2);
            dp += __shfl_xor(dp, 4);
            if ((lane & 7) == 0 && rr < w.rows) g.dp[(int64_t)(f0 / 64) * g.R + r] = dp;
          }
        }
      }
    }
    if (!more) break;
    w = wn;
  }
}

template <typename T, typename C, int LP, int LQ, int EPI, bool VEC>
hipError_t launch_gemm(const ExpertGemm& g, hipStream_t s) {
  const void* kern = reinterpret_cast<const void*>(k_expert_gemm<T, C, LP, LQ, EPI, VEC>);
  const size_t lds = 2 * (size_t)C::stage + (size_t)(g.E + 1) * 4;
  hipError_t e = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  int occ = 0;
  if ((e = hipOccupancyMaxActiveBlocksPerMultiprocessor(&occ, kern, C::threads, lds)) != hipSuccess) return e;
  if (occ < 1) return hipErrorLaunchOutOfResources;
  constexpr int BPo = EPI == kSwiglu ? C::BP / 2 : C::BP;
  const int64_t PT = (g.Pd + BPo - 1) / BPo;
  // at most this many tiles (the experts' row counts are only known on the device)
  const int64_t tiles = EPI == kWeightGrad ? (int64_t)g.E * PT * ((g.Qd + C::BQ - 1) / C::BQ)
                                           : PT * (g.R / C::BQ + std::min<int64_t>(g.E, g.R));
  if (tiles >= (int64_t(1) << 31)) return hipErrorInvalidValue;
  const int64_t blocks = std::min<int64_t>((tiles + 7) & ~int64_t(7), (int64_t)occ * device_info().cu_count & ~int64_t(7));
  hipLaunchKernelGGL((k_expert_gemm<T, C, LP, LQ, EPI, VEC>), dim3((unsigned)std::max<int64_t>(8, blocks)),
                     dim3(C::threads), lds, s, g);
  return hipGetLastError();
}

template <typename T, int LP, int LQ, int EPI>
hipError_t pick_gemm(const ExpertGemm& g, bool big, bool vec, hipStream_t s) {
  if (big) return vec ? launch_gemm<T, Big, LP, LQ, EPI, true>(g, s) : launch_gemm<T, Big, LP, LQ, EPI, false>(g, s);
  return vec ? launch_gemm<T, Small, LP, LQ, EPI, true>(g, s) : launch_gemm<T, Small, LP, LQ, EPI, false>(g, s);
}

}  // namespace expert
}  // namespace dol
