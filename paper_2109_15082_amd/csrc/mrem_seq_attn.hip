// Softmax attention over sequences of any lengths, with its gradients: causal or not, with a window, with shared key heads.
//
// Layout as in the module's attention kernels: score tiles are formed transposed, D[key][query] = K Q^T, so that in the 32x32
// accumulator layout a lane owns one query (lane % 32) and 16 of a tile's 32 keys.  The softmax statistics of a query need one exchange
// between lane halves, and the probabilities already have the layout of the second product's operand, O^T = V^T P^T, whose
// V^T fragments come from the row-major tile by transposing LDS reads.  The kernel of the key gradients mirrors it: a lane owns a key.
//
// Rows.  The query heads of a key head read the same keys, so the queries of a key head are numbered (token, head) with the head
// fastest and tiled as one axis: a token's `group` queries are neighbours, a key tile serves all of them, and a single token
// fills `group` of a tile's rows instead of one in each of `group` tiles.
// Sequences.  Tile slots are given out without knowing the lengths on the host: a sequence whose first row is s has the slots from
// s / tile + b on, of which at least ceil(length / tile) lie before the next sequence's first; slots behind a sequence's tiles end at once.
//
// The matrix instructions and the vector-ALU work of the softmax bound the long cases, memory the single tokens.  Reached at 2 x 4096
// tokens, 32 heads on 8, 128 wide, bf16, causal, counting the products of the pairs that are seen: forward (two) 308 us, 890 TFLOP/s; query
// gradients (three) 408 us, 1010; key gradients (four) 587 us, 940; a large matrix product reaches 1195.  16 single tokens on 700 to 8192 keys: 58 us, 5.0 TB/s.
#include "mrem_common.h"
#include "mrem_kernels.h"

#include <algorithm>
#include <type_traits>

namespace mrem {

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kThreads = 256, kWaves = 4;

// Tiles in LDS.  They are read by rows (16 lanes, 16 consecutive rows, 16 bytes each) and down their columns (4 consecutive rows, 64 bytes
// each).  bf16: rows follow each other without a gap and the 16-byte pieces of a row are exchanged by an exclusive or with a number of
// the row, such that either access meets all 64 banks once: rows lie 16, 8 or 4 pieces apart, of which 16 are the banks, so the number's
// upper bits follow the row's lowest ones, which a column access counts through, and its two lowest bits the next ones.  (A gap of 16
// bytes a row instead serves the rows but lets the four rows of a column access meet.)  fp32: columns are read value by value; a gap.
template <class T, int D>
constexpr int kStride = sizeof(T) == 2 ? D : D + 16 / (int)sizeof(T);
template <class T, int D>
__device__ __forceinline__ int piece_of(int row) {
  if constexpr (sizeof(T) == 4) return 0;
  else if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
  else if constexpr (D == 64) return ((row & 2) << 1) | ((row >> 2) & 3);
  else return (row >> 2) & 3;
}
// element `col` of a row; pieces are whole: col may be advanced within its piece
template <class T, int D>
__device__ __forceinline__ int lds_at(int row, int col) {
  return row * kStride<T, D> + (col ^ (piece_of<T, D>(row) * (16 / (int)sizeof(T))));
}

// ---- fragments: 8 values a lane, contraction index 8 (lane / 32) + i ---------
template <class T>
struct Frag;
template <>
struct Frag<bf16_t> { bf16x8_t v; };
template <>
struct Frag<float> { float v[8]; };

__device__ __forceinline__ f32x16_t mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mma(const Frag<float>& a, const Frag<float>& b, f32x16_t c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[i], b.v[i], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x16_t zero16() {
  f32x16_t z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}
// row (of 32) that accumulator register r of a lane in half h holds
__device__ __forceinline__ int row_of(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

template <class T>
__device__ __forceinline__ Frag<T> zero_frag() {
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = static_cast<T>(0.f);
  return f;
}
// 8 consecutive values (16-byte aligned)
template <class T>
__device__ __forceinline__ Frag<T> load8(const T* p) {
  Frag<T> f;
  if constexpr (sizeof(T) == 2) {
    f.v = *reinterpret_cast<const bf16x8_t*>(p);
  } else {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
    f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
  }
  return f;
}
// Where a lane reads a bf16 tile (at a multiple of 256 bytes), as an address whose exclusive or with a constant is another piece of the
// same row.  Forgotten by the compiler how it came about: it would keep each of those pieces' addresses in a register of its own throughout a loop.
typedef __attribute__((address_space(3))) char lds_char_t;
__device__ __forceinline__ unsigned lane_address(const bf16_t* tile, int offset) {
  unsigned a = (unsigned)(size_t)(lds_char_t*)tile + 2 * offset;
  asm("" : "+v"(a));
  return a;
}
__device__ __forceinline__ bf16x8_t read8(unsigned a) { return *(const __attribute__((address_space(3))) bf16x8_t*)(size_t)a; }
__device__ __forceinline__ s16x4_t read_tr(unsigned a) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)(size_t)a);
}
// accumulator registers 8 s .. 8 s + 7 as an operand.  bf16: probabilities and score gradients are rounded once, to 8 bits of
// mantissa, as the values of the products around them are; what is added up stays in 32 bits
template <class T>
__device__ __forceinline__ Frag<T> from_acc(const f32x16_t& a, int s) {
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f.v[i] = static_cast<T>(a[8 * s + i]);
  return f;
}
// Fragments of a tile, in the order in which a product takes them: along its rows (32 of them, piece by piece), or down its columns
// (of 32 rows, 32 columns for each e, row r of accumulator register order: 16 s + 4 (lane / 32) + 0..3 and 8 more).
template <class T, int D>
struct AlongRows {
  static constexpr int kCount = D / 16;
  const T* p;
  unsigned a = 0;
  __device__ __forceinline__ AlongRows(const T* tile, int row0, int lane) {
    const int at = lds_at<T, D>(row0 + (lane & 31), 8 * (lane >> 5));
    p = tile + at;
    if constexpr (sizeof(T) == 2) a = lane_address(tile, at);
  }
  __device__ __forceinline__ Frag<T> operator()(int kk) const {
    if constexpr (sizeof(T) == 2) return Frag<T>{read8(a ^ (32 * kk))};
    else return load8(p + 16 * kk);
  }
};
template <class T, int D>
struct DownColumns {
  static constexpr int kCount = D / 16;  // s, e
  const T* p;
  unsigned a = 0;
  __device__ __forceinline__ DownColumns(const T* tile, int row0, int lane) {
    if constexpr (sizeof(T) == 2) {
      // the transposing read: in a group of 16 lanes, lane s names columns 4 (s % 4) .. + 3 of row s / 4 and receives column s of the four rows
      const int g = lane >> 4, s16 = lane & 15;
      a = lane_address(tile, lds_at<T, D>(row0 + 4 * (lane >> 5) + (s16 >> 2), 16 * (g & 1) + 4 * (s16 & 3)));
    } else {
      p = tile + (row0 + 4 * (lane >> 5)) * kStride<T, D> + (lane & 31);
    }
  }
  __device__ __forceinline__ Frag<T> operator()(int n) const {
    const int s = n / (D / 32), e = n % (D / 32);
    if constexpr (sizeof(T) == 2) {
      union { bf16x8_t v; s16x4_t h[2]; } u;
      u.h[0] = read_tr((a ^ (64 * e)) + 32 * s * D);
      u.h[1] = read_tr((a ^ (64 * e) ^ 32) + (32 * s + 16) * D);  // 8 rows on: piece_of differs in its bit 1
      return Frag<T>{u.v};
    } else {
      Frag<T> u;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u.v[i] = p[(16 * s + i) * kStride<T, D> + 32 * e];
        u.v[4 + i] = p[(16 * s + 8 + i) * kStride<T, D> + 32 * e];
      }
      return u;
    }
  }
};
// Fragments on their way to the matrix instructions.  An LDS read takes as long as four of these, so the fourth next fragment is read behind each
// instruction; left to itself the compiler reads one ahead, and the instructions wait for two thirds of the time.  `beside`: vector instructions
// that the product does not need, a part of which goes behind each of its N instructions (which take as long as eight of them).
struct Nothing {
  __device__ __forceinline__ void operator()(int) const {}
};
template <class T, int DEPTH>
struct Ahead {
  static constexpr int kDepth = sizeof(T) == 2 ? DEPTH : 1;
  Frag<T> f[kDepth];
  template <class L>
  __device__ __forceinline__ void start(const L& read) {
#pragma unroll
    for (int i = 0; i < kDepth; ++i) f[i] = read(i);
  }
  template <int N, class L, class M, class B>
  __device__ __forceinline__ void run(const L& read, const M& multiply, const B& beside) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      multiply(n, f[n % kDepth]);
      if (n + kDepth < N) f[n % kDepth] = read(n + kDepth);
      beside(n);
      if constexpr (sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);
    }
  }
};
// (with three wavefronts a SIMD instead of two, two fragments are enough, and all that the registers hold)
template <int D>
constexpr int kAhead = D == 128 ? 4 : 2;
// element work of an accumulator's 16 registers in D / 16 parts
template <int D, class F>
__device__ __forceinline__ void part_of_16(int n, F f) {
#pragma unroll
  for (int r = 0; r < 256 / D; ++r) f(n * (256 / D) + r);
}
// 32 x 32 tile: LDS rows [row0, row0 + 32) times the 32 rows held as fragments b(kk), 16 columns each
template <class T, int D, class B, class F = Nothing>
__device__ __forceinline__ f32x16_t rows_times(const T* tile, int row0, int lane, B b, F beside = F(), f32x16_t acc = zero16()) {
  const AlongRows<T, D> rows(tile, row0, lane);
  Ahead<T, kAhead<D>> ahead;
  ahead.start(rows);
  ahead.template run<D / 16>(rows, [&](int kk, const Frag<T>& f) { acc = mma(f, b(kk), acc); }, beside);
  return acc;
}
// acc[e][.] += sum over the tile's 32 rows of tile[row][e] w[row], w in accumulator order
template <class T, int D, class F = Nothing>
__device__ __forceinline__ void add_rows(f32x16_t (&acc)[D / 32], const T* tile, int row0, int lane, const f32x16_t& w, F beside = F()) {
  const DownColumns<T, D> columns(tile, row0, lane);
  Ahead<T, kAhead<D>> ahead;
  ahead.start(columns);
  const Frag<T> f[2] = {from_acc<T>(w, 0), from_acc<T>(w, 1)};
  ahead.template run<D / 16>(columns, [&](int n, const Frag<T>& u) { acc[n % (D / 32)] = mma(u, f[n / (D / 32)], acc[n % (D / 32)]); }, beside);
}
// LDS accesses of a wavefront are carried out in order: nothing is to be moved across, that is all
__device__ __forceinline__ void wave_fence() { asm volatile("" ::: "memory"); }
// the other half wavefront's value
__device__ __forceinline__ float other_half(float v) {
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float((threadIdx.x & 32) ? x[0] : x[1]);
}

// ---- sequences ---------------------------------------------------------------
struct Seq {
  int64_t q0, k0;  // first rows
  int qn, kn;
  int b, tile;
};
__device__ __forceinline__ int64_t uniform(int64_t v, int lane) {
  return ((int64_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32) | (unsigned)__builtin_amdgcn_readlane((int)v, lane);
}
struct Rows {
  int64_t first, end;  // of a sequence, cut to the rows that there are
  __device__ __forceinline__ Rows(const int32_t* start, const int32_t* len, int64_t rows, int64_t each, int b) {
    first = start ? min(max((int64_t)start[b], (int64_t)0), rows) : each * b;
    end = start ? max(min((int64_t)start[b + 1], rows), first) : first + each;
    if (len) end = min(end, first + max(len[b], 0));
  }
};
// The sequence and the tile of a slot of the queries' axis (or the keys'), `per` rows of it a row of the tensor, `tile` rows a tile.
// A wavefront looks at 64 sequences at a time, for the last one whose first slot is not behind this one; a lane loads all that
// there is to know about its sequence at once, so that up to 64 of them cost one trip to memory.
template <bool KEYS>
__device__ __forceinline__ Seq find_sequence(const SeqAttn& a, int per, int tile, int slot) {
  const int lane = threadIdx.x & (kWave - 1);
  const int32_t* start = KEYS ? a.k_start : a.q_start;
  int at = 0;
  if (!start) {  // first slots lie on a known line: from a guess that is never too high
    // (in 32 bits of a product and a quotient of up to 2^24: off by less than 8)
    const float guess = (float)slot * (float)tile / ((float)((KEYS ? a.k_each : a.q_each) * per) + (float)tile);
    at = min(max((int)guess - 8, 0), a.batch - 1);
  }
  Seq s{};
  for (; at < a.batch; at += kWave) {
    const int i = min(at + lane, a.batch - 1);
    const Rows q(a.q_start, a.q_len, a.q_rows, a.q_each, i), k(a.k_start, a.k_len, a.k_rows, a.k_each, i);
    const int64_t base = (KEYS ? k.first : q.first) * per / tile + i;
    const unsigned long long before = __ballot(at + lane < a.batch && base <= slot);
    if (!before) break;
    const int from = 63 - __builtin_clzll(before);
    s.q0 = uniform(q.first, from);
    s.k0 = uniform(k.first, from);
    s.qn = (int)(uniform(q.end, from) - s.q0);
    s.kn = (int)(uniform(k.end, from) - s.k0);
    s.b = at + from;
    s.tile = (int)(slot - uniform(base, from));
    if (from < 63) break;
  }
  return s;
}
int64_t slots(int64_t rows, int batch, int per, int tile) { return rows * per / tile + batch; }

// keys [lo, hi) that token i of a sequence sees
__device__ __forceinline__ int key_end(const SeqAttn& a, const Seq& s, int i) { return a.causal ? min(max(i + s.kn - s.qn + 1, 0), s.kn) : s.kn; }
__device__ __forceinline__ int key_begin(const SeqAttn& a, const Seq& s, int i) {
  return a.window ? (int)max((int64_t)i + s.kn - s.qn - a.window + 1, (int64_t)0) : 0;
}

// ---- tiles on their way to LDS -----------------------------------------------
// Tiles are read through a buffer descriptor that ends where the tile's rows do: a thread's place in it is a 32-bit offset that stays the
// same from tile to tile, what lies behind the end is read as zero by the load itself, and the address is the scalar unit's.  (With 64-bit
// addresses and tests a tile cost a lane 105 vector instructions, half as many as its softmax.)  Strides are up to 2^21 elements.
typedef __amdgpu_buffer_rsrc_t rsrc_t;
template <class T>
__device__ __forceinline__ rsrc_t window(const T* base, int64_t elements) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, (int)(elements * (int)sizeof(T)), 0x00027000);
}
// (the whole offset in the vector part, which is what the end is compared with)
__device__ __forceinline__ u32x4_t read16(rsrc_t r, unsigned offset) { return __builtin_amdgcn_raw_buffer_load_b128(r, (int)offset, 0, 0); }

// rows [j0, j0 + ROWS) of a matrix of n > j0 rows whose first element is at src; rows behind it are zero
template <class T, int D, int ROWS>
struct Stage {
  static constexpr int kPiece = 16 / sizeof(T), kRowPieces = D / kPiece, kN = ROWS * kRowPieces / kThreads, kApart = kThreads / kRowPieces;
  static_assert(ROWS * kRowPieces % kThreads == 0, "whole pieces a thread");
  u32x4_t v[kN];
  __device__ __forceinline__ void load(const T* __restrict__ src, int64_t ld, int j0, int n) {
    const rsrc_t tile = window(src + j0 * ld, (min(ROWS, n - j0) - 1) * ld + D);
    const unsigned bytes = (unsigned)ld * (unsigned)sizeof(T), offset = threadIdx.x / kRowPieces * bytes + threadIdx.x % kRowPieces * 16;
#pragma unroll
    for (int i = 0; i < kN; ++i) v[i] = read16(tile, offset + i * kApart * bytes);
  }
  __device__ __forceinline__ void store(T* dst) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) *reinterpret_cast<u32x4_t*>(dst + lds_at<T, D>(threadIdx.x / kRowPieces + i * kApart, threadIdx.x % kRowPieces * kPiece)) = v[i];
  }
};
// Rows of the packed axis, (token r / group, head r % group), tile after tile, of two tensors: a thread's rows are kThreads / pieces apart and
// move on by a tile's rows, so their places advance by a quotient and a remainder that are divided once.
template <class T, int D, int ROWS, int THREADS>
struct QueryRows {
  static constexpr int kPiece = 16 / sizeof(T), kRowPieces = D / kPiece, kN = ROWS * kRowPieces / THREADS, kApart = THREADS / kRowPieces;
  static_assert(ROWS * kRowPieces % THREADS == 0, "whole pieces a thread");
  int token[kN], head[kN], first;
  u32x4_t q[kN], c[kN];
  __device__ __forceinline__ void start(const Divisor& group, int r0) {
    first = group.of(r0);
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int row = r0 + threadIdx.x / kRowPieces + i * kApart, t = group.of(row);
      token[i] = t - first;
      head[i] = row - t * group.d;
    }
  }
  // rows r0 + ... < n (zeros behind them), `first` the token of row r0; then the next tile's places
  __device__ __forceinline__ void load(const T* __restrict__ qs, int64_t ld_q, const T* __restrict__ cs, int64_t ld_c, int r0, int n, const Divisor& group) {
    const int tokens = min(ROWS, group.of(n - 1) - first + 1);  // that the tile's rows are of, or more
    const rsrc_t qw = window(qs + first * ld_q, (tokens - 1) * ld_q + group.d * D), cw = window(cs + first * ld_c, (tokens - 1) * ld_c + group.d * D);
    const unsigned bytes_q = (unsigned)ld_q * (unsigned)sizeof(T), bytes_c = (unsigned)ld_c * (unsigned)sizeof(T);
    const int next = group.of(r0 + ROWS), quotient = group.of(ROWS), rest = ROWS - quotient * group.d;
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const unsigned col = head[i] * (D * (int)sizeof(T)) + threadIdx.x % kRowPieces * 16;
      q[i] = read16(qw, __umul24(token[i], bytes_q) + col);
      c[i] = read16(cw, __umul24(token[i], bytes_c) + col);
      token[i] += quotient - (next - first);
      head[i] += rest;
      if (head[i] >= group.d) {
        head[i] -= group.d;
        token[i] += 1;
      }
    }
    first = next;
  }
  __device__ __forceinline__ void store(T* qs, T* cs) const {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int to = lds_at<T, D>(threadIdx.x / kRowPieces + i * kApart, threadIdx.x % kRowPieces * kPiece);
      *reinterpret_cast<u32x4_t*>(qs + to) = q[i];
      *reinterpret_cast<u32x4_t*>(cs + to) = c[i];
    }
  }
};

// A wavefront's transposed tile, a row of 32 in each lane's column, times f, to the rows that `row` gives addresses of (null: not there).
// bf16 rows are put together in LDS (32 rows of a tile), so that a row leaves in pieces of 16 bytes side by side: written by the lanes
// that hold them they are pieces of 8 bytes in 32 rows at a time, a quarter of what a store can carry.
template <class T, int D, class F>
__device__ __forceinline__ void store_rows(T* scratch, const f32x16_t (&acc)[D / 32], float f, int lane, F row) {
  const int half = lane >> 5, col = lane & 31;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<bf16x4_t*>(scratch + lds_at<T, D>(col, 32 * e + 8 * i) + 4 * half) = bf16x4_t{static_cast<bf16_t>(acc[e][4 * i] * f), static_cast<bf16_t>(acc[e][4 * i + 1] * f),
                                                                    static_cast<bf16_t>(acc[e][4 * i + 2] * f), static_cast<bf16_t>(acc[e][4 * i + 3] * f)};
    wave_fence();
    constexpr int kPieces = D / 8, kRows = kWave / kPieces;
    const int at = lane % kPieces * 8;
#pragma unroll
    for (int r = lane / kPieces; r < 32; r += kRows) {
      const u32x4_t v = *reinterpret_cast<const u32x4_t*>(scratch + lds_at<T, D>(r, at));
      T* to = row(r);
      if (to) *reinterpret_cast<u32x4_t*>(to + at) = v;
    }
    wave_fence();
  } else {
    T* to = row(col);
    if (to) {
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<float4*>(to + 32 * e + 8 * i + 4 * half) = make_float4(acc[e][4 * i] * f, acc[e][4 * i + 1] * f, acc[e][4 * i + 2] * f, acc[e][4 * i + 3] * f);
    }
  }
}

// ---- values that are not finite ----------------------------------------------
// A matrix instruction multiplies what a query does not see by zero, and zero times an infinity is not a number.  So a result that is not finite
// is formed again, from what is seen only, wherever it need not be so: by a wavefront a row, value by value.  Such rows are rare (a sum
// that is not a number in all its values is given up on the way), and finite results pay for a test.
template <int D>
__device__ __forceinline__ bool not_finite(const f32x16_t (&acc)[D / 32]) {
  bool bad = false;
#pragma unroll
  for (int e = 0; e < D / 32; ++e)
#pragma unroll
    for (int r = 0; r < 16; ++r) bad |= !(fabsf(acc[e][r]) < INFINITY);
  return bad;
}
// rows of a tile, a bit each, for which either half's lane says so
__device__ __forceinline__ unsigned rows_where(bool lane_says) {
  const unsigned long long m = __ballot(lane_says);
  return (unsigned)m | (unsigned)(m >> 32);
}
// a row of D values in the lanes of a wavefront
template <class T, int D>
struct LaneRow {
  static constexpr int kN = (D + 63) / 64;
  float v[kN];
  __device__ __forceinline__ explicit LaneRow(const T* p) {
#pragma unroll
    for (int i = 0; i < kN; ++i) {
      const int d = (threadIdx.x & 63) + 64 * i;
      v[i] = d < D ? (float)p[d] : 0.f;
    }
  }
  __device__ __forceinline__ float dot(const LaneRow& o) const {
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < kN; ++i) t += v[i] * o.v[i];
    return wave_sum(t);
  }
};
template <int N>
struct LaneSum {
  float v[N] = {};
  template <class R>
  __device__ __forceinline__ void add(float f, const R& r) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += f * r.v[i];
  }
  __device__ __forceinline__ bool lost() const {  // not a number in any lane
    bool all = true;
#pragma unroll
    for (int i = 0; i < N; ++i) all &= v[i] != v[i];
    return __all(all);
  }
  template <class T>
  __device__ __forceinline__ void store(T* p, float f, int n) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int d = (threadIdx.x & 63) + 64 * i;
      if (d < n) p[d] = static_cast<T>(v[i] * f);
    }
  }
};
// the output of a (token, head) from its log-sum-exp, and with GRADIENT that of its query
template <class T, int D, bool GRADIENT>
__device__ __forceinline__ void query_again(const SeqAttn& a, const Seq& s, int head, int h, int token, float lse, float delta) {
  const T *kp = static_cast<const T*>(a.k) + s.k0 * a.ld_k + head * D, *vp = static_cast<const T*>(a.v) + s.k0 * a.ld_v + head * D;
  const LaneRow<T, D> q(static_cast<const T*>(a.q) + (s.q0 + token) * a.ld_q + h * D);
  const LaneRow<T, D> c(static_cast<const T*>(GRADIENT ? a.dout : a.q) + (s.q0 + token) * (GRADIENT ? a.ld_o : a.ld_q) + h * D);
  LaneSum<LaneRow<T, D>::kN> sum;
  const int end = key_end(a, s, token);
#pragma unroll 1
  for (int j = key_begin(a, s, token); j < end && !sum.lost(); ++j) {
    const LaneRow<T, D> k(kp + j * a.ld_k), v(vp + j * a.ld_v);
    const float p = __builtin_amdgcn_exp2f((q.dot(k) * a.scale - lse) * kLog2e);
    if constexpr (GRADIENT) sum.add(p * (c.dot(v) - delta), k);
    else sum.add(p, v);
  }
  if constexpr (GRADIENT) sum.store(static_cast<T*>(a.dq) + (s.q0 + token) * a.ld_q + h * D, a.scale, D);
  else sum.store(static_cast<T*>(a.out) + (s.q0 + token) * a.ld_o + h * D, 1.f, D);
}
// the gradients of a key and its value: rows [lo, hi) of the packed axis see it
template <class T, int D>
__device__ __forceinline__ void key_again(const SeqAttn& a, const Seq& s, int head, int key, int lo, int hi) {
  const LaneRow<T, D> k(static_cast<const T*>(a.k) + (s.k0 + key) * a.ld_k + head * D), v(static_cast<const T*>(a.v) + (s.k0 + key) * a.ld_v + head * D);
  const float2* stats = reinterpret_cast<const float2*>(a.delta) + ((int64_t)head * a.q_rows + s.q0) * a.group.d;
  LaneSum<LaneRow<T, D>::kN> dk, dv;
#pragma unroll 1
  for (int r = lo; r < hi && !(dk.lost() && dv.lost()); ++r) {
    const int t = a.group.of(r), h = head * a.group.d + r - t * a.group.d;
    const LaneRow<T, D> q(static_cast<const T*>(a.q) + (s.q0 + t) * a.ld_q + h * D), c(static_cast<const T*>(a.dout) + (s.q0 + t) * a.ld_o + h * D);
    const float2 st = stats[r];
    const float p = __builtin_amdgcn_exp2f((q.dot(k) + st.x) * a.scale * kLog2e);
    dv.add(p, c);
    dk.add(p * (c.dot(v) - st.y), q);
  }
  dk.store(static_cast<T*>(a.dk) + (s.k0 + key) * a.ld_k + head * D, a.scale, D);
  dv.store(static_cast<T*>(a.dv) + (s.k0 + key) * a.ld_v + head * D, 1.f, D);
}

// ---- forward -----------------------------------------------------------------
// rows of a block: 128, 32 a wavefront, keys in tiles of 64 (fp32: 32); or 32 that all wavefronts share, each with 32 of a tile's
// 128 keys, for sequences with few queries: what a block then does is read keys, and it reads four times as many at a time
template <class T, int RB>
constexpr int kKeyTile = RB == 32 ? 128 : sizeof(T) == 2 ? 64 : 32;

// wavefronts a SIMD, by which the registers are bounded
template <class T, int D, int RB>
constexpr int kForwardWaves = sizeof(T) == 4 ? 1 : D == 128 || RB == 32 ? 2 : 3;

template <class T, int D, int RB>
__global__ __launch_bounds__(kThreads, (kForwardWaves<T, D, RB>)) void seq_fwd_k(SeqAttn a) {
  constexpr int KT = kKeyTile<T, RB>, NS = RB == 32 ? 1 : KT / 32, S = kStride<T, D>;
  constexpr int kTileBytes = 2 * KT * S * (int)sizeof(T), kMergeBytes = RB == 32 ? 32 * D * 4 * (kWaves - 1) : 0;
  __shared__ __attribute__((aligned(256))) char lds[kTileBytes > kMergeBytes ? kTileBytes : kMergeBytes];
  __shared__ float merge_m[kWaves][32], merge_l[kWaves][32];
  T *const Ks = reinterpret_cast<T*>(lds), *const Vs = Ks + KT * S;
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = a.group.d;
  const int head = blockIdx.x % a.hk, split = blockIdx.y;
  // the last tiles see the most keys: they go first
  const int slot = (int)(gridDim.x / a.hk - 1 - blockIdx.x / a.hk);
  const Seq s = find_sequence<false>(a, group, RB, slot);
  const int rows = s.qn * group, r0 = s.tile * RB;
  if (r0 >= rows) return;

  const int wr = r0 + (RB == 32 ? 0 : 32 * wave), row = wr + col, rc = min(row, rows - 1), token = a.group.of(rc), h = head * group + rc - token * group;
  const T* q = static_cast<const T*>(a.q) + (s.q0 + token) * a.ld_q + h * D + 8 * half;
  Frag<T> qf[D / 16];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) qf[kk] = load8(q + 16 * kk);
  const int lo = key_begin(a, s, token), hi = row < rows ? key_end(a, s, token) : 0;
  // of the wavefront's and of the block's rows: keys that any of them sees; all of the wavefront's see [w_lo, w_hi)
  const int t_first = a.group.of(r0), t_last = a.group.of(min(r0 + RB, rows) - 1);
  int j_lo = key_begin(a, s, t_first), j_hi = key_end(a, s, t_last);
  const int wt0 = a.group.of(min(wr, rows - 1)), wt1 = a.group.of(min(wr + 32, rows) - 1);
  const int w_lo = key_begin(a, s, wt1), w_hi = key_end(a, s, wt0), any_lo = key_begin(a, s, wt0), any_hi = wr < rows ? key_end(a, s, wt1) : 0;
  if (a.splits > 1) {
    const int n = j_hi > j_lo ? ((j_hi - j_lo + KT - 1) / KT + a.splits - 1) / a.splits * KT : 0;
    j_lo = (int)min((int64_t)j_lo + (int64_t)split * n, (int64_t)j_hi);
    j_hi = min(j_lo + n, j_hi);
  }

  const T* kp = static_cast<const T*>(a.k) + s.k0 * a.ld_k + head * D;
  const T* vp = static_cast<const T*>(a.v) + s.k0 * a.ld_v + head * D;
  f32x16_t o[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) o[e] = zero16();
  float m = -INFINITY, l = 0.f;  // what exponentials are taken against (a score, without scale), this lane's part of their sum
  const float c = a.scale * kLog2e;
  Stage<T, D, KT> ks, vs;
  const auto load = [&](int j) {
    ks.load(kp, a.ld_k, j, s.kn);
    vs.load(vp, a.ld_v, j, s.kn);
  };
  if (j_lo < j_hi) load(j_lo);
  for (int j0 = j_lo; j0 < j_hi; j0 += KT) {
    ks.store(Ks);
    vs.store(Vs);
    __syncthreads();
    if (j0 + KT < j_hi) load(j0 + KT);
    const int base = RB == 32 ? 32 * wave : 0;
    if (j0 + base < any_hi && j0 + base + 32 * NS > any_lo) {
      f32x16_t p[NS];
#pragma unroll
      for (int t = 0; t < NS; ++t) p[t] = rows_times<T, D>(Ks, base + 32 * t, lane, [&](int kk) { return qf[kk]; });
      // keys of this tile behind the split's last one belong to the next split: it starts at a tile, so none are
      if (j0 + base < w_lo || j0 + base + 32 * NS > w_hi) {
#pragma unroll
        for (int t = 0; t < NS; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int j = j0 + base + 32 * t + row_of(r, half);
            if (j < lo || j >= hi) p[t][r] = -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int t = 0; t < NS; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, p[t][r]);
      top = fmaxf(top, other_half(top));
      // what exponentials are taken against follows the maximum only when it has risen by more than 2^8: until then they are
      // at most 256 and nothing that 32 bits hold is lost, and the 64 products a tile of following it at once are saved
      if (__any((top - m) * c > 8.f)) {
        const float to = fmaxf(top, m), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);
        m = to;
        l *= f;
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[e][r] *= f;
      }
      // fp32: the difference first, so that a single key's exponential is one and its output the value to the bit
      const float m0 = m == -INFINITY ? 0.f : m, mc = m0 * c;
      const auto exponential = [&](int t, int r) {
        p[t][r] = __builtin_amdgcn_exp2f(sizeof(T) == 4 ? (p[t][r] - m0) * c : fmaf(p[t][r], c, -mc));
        l += p[t][r];
      };
#pragma unroll
      for (int r = 0; r < 16; ++r) exponential(0, r);
#pragma unroll
      for (int t = 0; t < NS; ++t)
        add_rows<T, D>(o, Vs, base + 32 * t, lane, p[t], [&](int n) {
          if (t + 1 < NS) part_of_16<D>(n, [&](int r) { exponential(t + 1, r); });
        });
    }
    __syncthreads();
  }
  l += other_half(l);

  if constexpr (RB == 32) {  // the wavefronts' parts meet in the first one
    if (lane < 32) {
      merge_m[wave][lane] = m;
      merge_l[wave][lane] = l;
    }
    float* x = reinterpret_cast<float*>(lds);
    if (wave > 0) {
      float* to = x + (wave - 1) * 32 * D + lane;
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int r = 0; r < 16; ++r) to[(e * 16 + r) * 64] = o[e][r];
    }
    __syncthreads();
    if (wave > 0) return;
    float top = m;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) top = fmaxf(top, merge_m[w][col]);
    const float mm = top == -INFINITY ? 0.f : top;
    float f = __builtin_amdgcn_exp2f((m - mm) * c);
    l *= f;
#pragma unroll
    for (int e = 0; e < D / 32; ++e)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[e][r] *= f;
#pragma unroll 1
    for (int w = 1; w < kWaves; ++w) {
      f = __builtin_amdgcn_exp2f((merge_m[w][col] - mm) * c);
      l += merge_l[w][col] * f;
      const float* from = x + (w - 1) * 32 * D + lane;
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[e][r] += from[(e * 16 + r) * 64] * f;
    }
    m = top;
  }
  if constexpr (RB == 32) wave_fence();  // the parts have been read
  const bool whole = a.splits == 1;
  if (row < rows && half == 0) {
    const int64_t at = (int64_t)h * a.q_rows + s.q0 + token;
    if (whole) {
      a.lse[at] = l == 0.f ? -INFINITY : (m * c + log2f(l)) * kLn2;
    } else {
      float* ml = a.part + (int64_t)a.splits * a.hq * a.q_rows * D + 2 * ((int64_t)split * a.hq * a.q_rows + at);
      ml[0] = m;
      ml[1] = l;
    }
  }
  const auto place = [&](int r, int* head_of, int* token_of) {
    const int at = wr + r, t = a.group.of(at);
    *token_of = t;
    *head_of = head * group + at - t * group;
    return at < rows;
  };
  int rh, rt;
  if (!whole) {
    store_rows<float, D>(nullptr, o, 1.f, lane, [&](int r) {
      return place(r, &rh, &rt) ? a.part + (((int64_t)split * a.hq + rh) * a.q_rows + s.q0 + rt) * D : nullptr;
    });
  } else {
    const unsigned again = rows_where(row < rows && l > 0.f && l < INFINITY && not_finite<D>(o));
    store_rows<T, D>(reinterpret_cast<T*>(lds) + (RB == 32 ? 0 : wave * 32 * S), o, l == 0.f ? 0.f : 1.f / l, lane, [&](int r) {
      return place(r, &rh, &rt) && !(again >> r & 1) ? static_cast<T*>(a.out) + (s.q0 + rt) * a.ld_o + rh * D : nullptr;
    });
    const float lse = (m * c + log2f(l)) * kLn2;
#pragma unroll 1
    for (unsigned left = again; left; left &= left - 1) {
      const int r = __builtin_ctz(left);
      place(r, &rh, &rt);
      query_again<T, D, false>(a, s, head, rh, rt, __shfl(lse, r), 0.f);
    }
  }
}

// joins the parts of a row whose keys were shared out: a wavefront a (token, head)
template <class T, int D>
__global__ __launch_bounds__(kThreads) void seq_join_k(SeqAttn a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = a.group.d, head = blockIdx.x % a.hk;
  constexpr int RB = 32;
  const Seq s = find_sequence<false>(a, group, RB, (int)(blockIdx.x / a.hk));
  const int rows = s.qn * group;
  const float* ml = a.part + (int64_t)a.splits * a.hq * a.q_rows * D;
  const int64_t step = (int64_t)a.hq * a.q_rows;
  const float c = a.scale * kLog2e;
  for (int row = s.tile * RB + wave; row < min(rows, (s.tile + 1) * RB); row += kWaves) {
    const int token = a.group.of(row), h = head * group + row - token * group;
    const int64_t at = (int64_t)h * a.q_rows + s.q0 + token;
    // a lane a part, of which there are up to 32; a part without a key of its own has the sum 0 and zeros
    const float2 mine = lane < a.splits ? *reinterpret_cast<const float2*>(ml + 2 * (at + lane * step)) : make_float2(-INFINITY, 0.f);
    const float m = wave_max(mine.x), weight = mine.y == 0.f ? 0.f : __builtin_amdgcn_exp2f((mine.x - m) * c);
    const float l = wave_sum(mine.y * weight);
    float o[D / 64 > 0 ? D / 64 : 1] = {};
    for (int i0 = 0; i0 < a.splits; i0 += 4)  // four on their way together; weights of parts that there are not are 0
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), i0 + k));
        const float* part = a.part + (at + min(i0 + k, a.splits - 1) * step) * D;
#pragma unroll
        for (int e = 0; e < (D + 63) / 64; ++e)
          if (lane + 64 * e < D) o[e] += part[lane + 64 * e] * w;
      }
    const float f = l == 0.f ? 0.f : 1.f / l;
    const float lse = l == 0.f ? -INFINITY : (m * c + log2f(l)) * kLn2;
    if (lane == 0) a.lse[at] = lse;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < (D + 63) / 64; ++e) bad |= !(fabsf(o[e]) < INFINITY);
    if (__any(bad) && fabsf(lse) < INFINITY) {
      query_again<T, D, false>(a, s, head, h, token, lse, 0.f);
      continue;
    }
    T* out = static_cast<T*>(a.out) + (s.q0 + token) * a.ld_o + h * D;
#pragma unroll
    for (int e = 0; e < (D + 63) / 64; ++e)
      if (lane + 64 * e < D) out[lane + 64 * e] = static_cast<T>(o[e] * f);
  }
}

// ---- backward ----------------------------------------------------------------
// gradient of the queries: 32 rows a wavefront, keys in tiles.  Also leaves delta = out . d_out of each row, formed by the matrix
// instructions that form d_out . v, so that the two agree to the bit where a query sees one key and its gradient is zero.
template <class T, int D, int RB>
__global__ __launch_bounds__(kThreads, sizeof(T) == 4 ? 1 : D == 128 || RB == 32 ? 2 : 3) void seq_bwd_q_k(SeqAttn a) {
  constexpr int KT = kKeyTile<T, RB>, NS = RB == 32 ? 1 : KT / 32, S = kStride<T, D>;
  static_assert(2 * KT * S * (int)sizeof(T) >= (RB == 32 ? 32 * D * 4 * (kWaves - 1) : 0), "the sums meet where the tiles were");
  __shared__ __attribute__((aligned(256))) T tiles[2 * KT * S];
  T *const Ks = tiles, *const Vs = tiles + KT * S;
  __shared__ float offs[kWaves][32];
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int group = a.group.d, head = blockIdx.x % a.hk;
  const int slot = (int)(gridDim.x / a.hk - 1 - blockIdx.x / a.hk);
  const Seq s = find_sequence<false>(a, group, RB, slot);
  const int rows = s.qn * group, r0 = s.tile * RB;
  if (r0 >= rows) return;

  const int wr = r0 + (RB == 32 ? 0 : 32 * wave), row = wr + col, rc = min(row, rows - 1), token = a.group.of(rc), h = head * group + rc - token * group;
  const T* q = static_cast<const T*>(a.q) + (s.q0 + token) * a.ld_q + h * D + 8 * half;
  const int64_t o_at = (s.q0 + token) * a.ld_o + h * D + 8 * half, stat = (int64_t)h * a.q_rows + s.q0 + token;
  Frag<T> qf[D / 16], df[D / 16];
  f32x16_t oo = zero16();
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    qf[kk] = load8(q + 16 * kk);
    df[kk] = load8(static_cast<const T*>(a.dout) + o_at + 16 * kk);
    oo = mma(load8(static_cast<const T*>(a.out) + o_at + 16 * kk), df[kk], oo);  // [row of out][row of d_out]
  }
  const float c = a.scale * kLog2e;
  float delta = 0.f;  // the diagonal: row col, in the half that holds it
#pragma unroll
  for (int r = 0; r < 16; ++r) delta = row_of(r, half) == col ? oo[r] : delta;
  {
    const float other = other_half(delta);
    if (((col >> 2) & 1) != half) delta = other;
  }
  const float lse2 = a.lse[stat] * kLog2e;
  const int lo = key_begin(a, s, token), hi = row < rows ? key_end(a, s, token) : 0;
  const int t_first = a.group.of(r0), t_last = a.group.of(min(r0 + RB, rows) - 1);
  const int j_lo = key_begin(a, s, t_first), j_hi = key_end(a, s, t_last);
  const int wt0 = a.group.of(min(wr, rows - 1)), wt1 = a.group.of(min(wr + 32, rows) - 1);
  const int w_lo = key_begin(a, s, wt1), w_hi = key_end(a, s, wt0), any_lo = key_begin(a, s, wt0), any_hi = wr < rows ? key_end(a, s, wt1) : 0;

  const T* kp = static_cast<const T*>(a.k) + s.k0 * a.ld_k + head * D;
  const T* vp = static_cast<const T*>(a.v) + s.k0 * a.ld_v + head * D;
  Stage<T, D, KT> ks, vs;
  const auto load = [&](int j) {
    ks.load(kp, a.ld_k, j, s.kn);
    vs.load(vp, a.ld_v, j, s.kn);
  };
  // delta of a stored output is off by the output's rounding, which is what most of a row's gradient is made of where it sees few keys (a
  // row's gradient is a difference of its few products).  There a first pass takes the sum of the score gradients, which is zero but for
  // that error, back from delta: rows of up to 128 keys in bf16.  With more the error is below the rounding of the gradient itself, and fp32
  // rounds an output no more than the products' sums.  (Two tokens of 128 wide heads in bf16: gradients 5.6e-3 off without it, 1.7e-3 with
  // it.  In fp32 it would cost 15.8 instead of 12.4 us for four sentences of up to 77 tokens, 12 heads of 64.)
  const bool twice = sizeof(T) == 2 && (a.window ? min(a.window, j_hi) : j_hi) <= 128;
  // gradients of the scores of keys [j, j + 32), rows `at` of the tile
  const auto score_gradients = [&](int at, int j) {
    f32x16_t p = rows_times<T, D>(Ks, at, lane, [&](int kk) { return qf[kk]; });
    f32x16_t dp = rows_times<T, D>(Vs, at, lane, [&](int kk) { return df[kk]; },
                                   [&](int n) { part_of_16<D>(n, [&](int r) { p[r] = __builtin_amdgcn_exp2f(fmaf(p[r], c, -lse2)); }); });
#pragma unroll
    for (int r = 0; r < 16; ++r) dp[r] = p[r] * (dp[r] - delta);
    if (j < w_lo || j + 32 > w_hi) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = j + row_of(r, half);
        if (key < lo || key >= hi) dp[r] = 0.f;
      }
    }
    return dp;
  };
  const auto walk = [&](auto take) {
    if (j_lo < j_hi) load(j_lo);
    for (int j0 = j_lo; j0 < j_hi; j0 += KT) {
      ks.store(Ks);
      vs.store(Vs);
      __syncthreads();
      if (j0 + KT < j_hi) load(j0 + KT);
#pragma unroll
      for (int t = 0; t < NS; ++t) {
        const int at = RB == 32 ? 32 * wave : 32 * t, j = j0 + at;
        if (j < any_hi && j + 32 > any_lo) take(at, score_gradients(at, j));
      }
      __syncthreads();
    }
  };
  if (twice) {
    float off = 0.f;
    walk([&](int, const f32x16_t& ds) {
#pragma unroll
      for (int r = 0; r < 16; ++r) off += ds[r];
    });
    off += other_half(off);
    if constexpr (RB == 32) {  // each wavefront has seen a part of the keys
      offs[wave][col] = off;
      __syncthreads();
      off = offs[0][col] + offs[1][col] + offs[2][col] + offs[3][col];
    }
    delta += off;
  }
  f32x16_t dq[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) dq[e] = zero16();
  walk([&](int at, const f32x16_t& ds) { add_rows<T, D>(dq, Ks, at, lane, ds); });
  if (row < rows && half == 0 && (RB > 32 || wave == 0)) reinterpret_cast<float2*>(a.delta)[((int64_t)head * a.q_rows + s.q0) * group + row] = make_float2(lse2 == -INFINITY ? -INFINITY : -lse2 / c, delta);
  if constexpr (RB == 32) {  // the wavefronts' sums meet in the first one
    float* x = reinterpret_cast<float*>(tiles) + lane;
    if (wave > 0) {
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int r = 0; r < 16; ++r) x[(wave - 1) * 32 * D + (e * 16 + r) * 64] = dq[e][r];
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll 1
    for (int w = 1; w < kWaves; ++w)
#pragma unroll
      for (int e = 0; e < D / 32; ++e)
#pragma unroll
        for (int r = 0; r < 16; ++r) dq[e][r] += x[(w - 1) * 32 * D + (e * 16 + r) * 64];
  }
  if constexpr (RB == 32) wave_fence();  // the sums have been read
  const unsigned again = rows_where(row < rows && fabsf(lse2) < INFINITY && fabsf(delta) < INFINITY && not_finite<D>(dq));
  store_rows<T, D>(tiles + (RB == 32 ? 0 : wave * 32 * S), dq, a.scale, lane, [&](int r) -> T* {
    const int at = wr + r, t = a.group.of(at);
    return at < rows && !(again >> r & 1) ? static_cast<T*>(a.dq) + (s.q0 + t) * a.ld_q + (head * group + at - t * group) * D : nullptr;
  });
#pragma unroll 1
  for (unsigned left = again; left; left &= left - 1) {
    const int r = __builtin_ctz(left), at = wr + r, t = a.group.of(at);
    query_again<T, D, true>(a, s, head, head * group + at - t * group, t, __shfl(lse2, r) * kLn2, __shfl(delta, r));
  }
}

// Gradients of keys and values: RB keys a block, 32 a wavefront, the queries of all heads of the group in tiles of rows.  P wavefronts own
// the same keys, take every P-th tile, and meet in LDS at the end.  Both gradients, both operands and two tiles of scores are some 230
// registers a lane at head dimension 128, which allows two wavefronts a SIMD.
//   <32, 4>   fewer blocks of 128 keys than compute units.  us of a backward pass, against <128, 2>: 34 blocks (2048 tokens, 8 heads on 2, 128
//             wide) 185 against 291, 132 (2 x 4096) 455 against 618, 108 (1024 tokens, 12 heads of 64) 41 against 48; 272 (128 wide) 406
//             against 354, 324 (64 wide) 58 against 51.
//   <128, 2>  (128 wide), <128, 3> (narrower, up to two blocks a unit): the wavefronts of a SIMD share their keys.  With other keys for the second
//             one there would be half as many blocks, each twice as long, and under a causal mask the block of the first keys
//             would outlast the others by half of the kernel's time (2 x 4096 tokens, 32 heads on 8, 128 wide: 690 against 1230 us).
//   <128, 1>  (narrower, more blocks): starts and ends of some hide behind others; 432 blocks of 12 heads of 64: 64 against 66 us with
//             <128, 3>, 864: 84 against 98, 3456: 262 against 329.
// Tiles are written to LDS one step ahead, so that there is one barrier a step.
// fragments of the keys and of the values (of D / 16) that lie in LDS, a thread's own, since the registers do not hold them; read ahead like
// the tiles (the compiler's own choice, memory, is read when it is wanted: 590 -> 715 us for two fragments)
template <class T, int D>
constexpr int kKeysInLds = sizeof(T) == 2 && D == 128 ? 2 : 0;
template <class T, int D>
constexpr int kValuesInLds = sizeof(T) == 2 ? D == 128 ? 8 : D == 64 ? 4 : 0 : 0;
// rows of a wavefront's tile
template <class T, int D>
constexpr int kQueryTile = sizeof(T) == 2 && D == 32 ? 64 : 32;

template <class T, int D, int RB, int P>
__global__ __launch_bounds__(2 * RB * P, sizeof(T) == 4 || (RB == 32 && D != 64) ? 1 : D == 128 || RB == 32 ? 2 : 3) void seq_bwd_k_k(SeqAttn a) {
  constexpr int NT = 2 * RB * P, WT = kQueryTile<T, D>, QT = WT * P, S = kStride<T, D>;
  constexpr int kTileBytes = 4 * QT * S * (int)sizeof(T), kMergeBytes = (P - 1) * RB * D * 4;
  __shared__ __attribute__((aligned(256))) char tiles[kTileBytes > kMergeBytes ? kTileBytes : kMergeBytes];
  const auto Qs = [&](int buf) { return reinterpret_cast<T*>(tiles) + buf * QT * S; };
  const auto Cs = [&](int buf) { return reinterpret_cast<T*>(tiles) + (2 + buf) * QT * S; };
  constexpr int VL = RB == 32 ? 0 : kValuesInLds<T, D>, VR = D / 16 - VL;
  __shared__ Frag<T> v_lds[VL > 0 ? VL : 1][VL > 0 ? NT : 1];
  __shared__ __attribute__((aligned(16))) float stats[2][2][QT];  // -lse / scale, delta
  const int lane = threadIdx.x & 63, half = lane >> 5, col = lane & 31;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = w % (RB / 32), part = w / (RB / 32);
  const int group = a.group.d, head = blockIdx.x % a.hk;
  const int slot = (int)(blockIdx.x / a.hk);  // the first keys are seen by the most queries
  const Seq s = find_sequence<true>(a, 1, RB, slot);
  const int j0 = s.tile * RB;
  if (j0 >= s.kn) return;

  const int key = j0 + 32 * wave + col, kc = min(key, s.kn - 1);
  const T* kp = static_cast<const T*>(a.k) + (s.k0 + kc) * a.ld_k + head * D + 8 * half;
  const T* vp = static_cast<const T*>(a.v) + (s.k0 + kc) * a.ld_v + head * D + 8 * half;
  constexpr int KL = RB == 32 ? 0 : kKeysInLds<T, D>, KR = D / 16 - KL;
  __shared__ Frag<T> k_lds[KL > 0 ? KL : 1][KL > 0 ? NT : 1];
  Frag<T> kf[KR], vf[VR > 0 ? VR : 1];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    if (kk < KR) kf[kk] = load8(kp + 16 * kk);
    else k_lds[kk - KR][threadIdx.x] = load8(kp + 16 * kk);
    if (kk < VR) vf[kk] = load8(vp + 16 * kk);
    else v_lds[kk - VR][threadIdx.x] = load8(vp + 16 * kk);
  }
  const int rows = s.qn * group, off = s.kn - s.qn;
  // rows [lo, hi) whose queries see key j: token + off >= j, token + off - window < j
  const auto row_begin = [&](int j) { return a.causal ? (int)min((int64_t)max(j - off, 0) * group, (int64_t)rows) : 0; };
  const auto row_end = [&](int j) { return a.window ? (int)min(max((int64_t)j - off + a.window, (int64_t)0) * group, (int64_t)rows) : rows; };
  const int lo = row_begin(kc), hi = key < s.kn ? row_end(kc) : 0;
  const int k_last = min(j0 + RB, s.kn) - 1;
  const int r_lo = row_begin(j0), r_hi = row_end(k_last);
  const int wk0 = min(j0 + 32 * wave, s.kn - 1), wk1 = min(j0 + 32 * wave + 31, s.kn - 1);
  const bool wave_on = j0 + 32 * wave < s.kn, wave_whole = j0 + 32 * wave + 32 <= s.kn;
  const int any_lo = row_begin(wk0), any_hi = wave_on ? row_end(wk1) : 0, w_lo = row_begin(wk1), w_hi = wave_whole ? row_end(wk0) : 0;

  const T* qp = static_cast<const T*>(a.q) + s.q0 * a.ld_q + head * group * D;
  const T* cp = static_cast<const T*>(a.dout) + s.q0 * a.ld_o + head * group * D;
  const float2* sp = reinterpret_cast<const float2*>(a.delta) + ((int64_t)head * a.q_rows + s.q0) * group;
  f32x16_t dk[D / 32], dv[D / 32];
#pragma unroll
  for (int e = 0; e < D / 32; ++e) {
    dk[e] = zero16();
    dv[e] = zero16();
  }
  const float c = a.scale * kLog2e;
  QueryRows<T, D, QT, NT> qr;
  float2 stat = make_float2(0.f, 0.f);
  const auto load = [&](int r) {
    qr.load(qp, a.ld_q, cp, a.ld_o, r, rows, a.group);
    if ((int)threadIdx.x < QT) stat = sp[min(r + (int)threadIdx.x, rows - 1)];
  };
  const auto store = [&](int buf) {
    qr.store(Qs(buf), Cs(buf));
    if ((int)threadIdx.x < QT) {
      stats[buf][0][threadIdx.x] = stat.x;
      stats[buf][1][threadIdx.x] = stat.y;
    }
  };
  if (r_lo < r_hi) {
    qr.start(a.group, r_lo);
    load(r_lo);
    store(0);
    if (r_lo + QT < r_hi) load(r_lo + QT);
    __syncthreads();
  }
  for (int r = r_lo, buf = 0; r < r_hi; r += QT, buf ^= 1) {
    if (r + QT < r_hi) {
      store(buf ^ 1);
      if (r + 2 * QT < r_hi) load(r + 2 * QT);
    }
#pragma unroll
    for (int t = 0; t < WT / 32; ++t) {
      const int at_t = part * WT + 32 * t, rt = r + at_t;
      if (rt >= any_hi || rt + 32 <= any_lo) continue;
      // the wavefronts of a SIMD would fall into step, both at the matrix instructions and then both at the others: who is at them goes first
      const auto priority = [](auto on) {
        if constexpr (sizeof(T) == 2 && D == 128) __builtin_amdgcn_s_setprio(decltype(on)::value);
      };
      using First = std::integral_constant<short, 1>;
      using Last = std::integral_constant<short, 0>;
      const float* st = &stats[buf][0][at_t + 4 * half];
      // bf16: the sum starts at -lse / scale, so that nothing is left to subtract; fp32 does not, since a sum near lse / scale rounds coarser
      f32x16_t p;
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(st + 2 * i);
        p[i] = v.x;
        p[i + 1] = v.y;
        p[i + 2] = v.z;
        p[i + 3] = v.w;
      }
      Frag<T> kl[KL > 0 ? KL : 1];
      priority(First());
      p = rows_times<T, D>(
          Qs(buf), at_t, lane, [&](int kk) { return kk < KR ? kf[kk < KR ? kk : 0] : kl[kk < KR ? 0 : kk - KR]; },
          [&](int n) {
            if (n < KL) kl[n] = k_lds[n][threadIdx.x];
          },
          sizeof(T) == 2 ? p : zero16());
      if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] += st[row_of(i, 0)];
      }
      const auto exponentials = [&](int n) { part_of_16<D>(n, [&](int i) { p[i] = __builtin_amdgcn_exp2f(p[i] * c); }); };
      f32x16_t dp = zero16();
      if constexpr (VL == 0) {
        dp = rows_times<T, D>(Cs(buf), at_t, lane, [&](int kk) { return vf[kk]; }, exponentials);
      } else {  // both operands come from LDS: two of either ahead
        static_assert(VL == D / 16, "all of them");
        const AlongRows<T, D> of_c(Cs(buf), at_t, lane);
        const auto of_v = [&](int kk) { return v_lds[kk][threadIdx.x]; };
        Ahead<T, 2> c_ahead;
        Frag<T> v_ahead[2] = {of_v(0), of_v(1)};
        c_ahead.start(of_c);
        c_ahead.template run<D / 16>(
            of_c,
            [&](int kk, const Frag<T>& f) {
              dp = mma(f, v_ahead[kk % 2], dp);
              if (kk + 2 < D / 16) v_ahead[kk % 2] = of_v(kk + 2);
            },
            exponentials);
      }
      priority(Last());
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const float4 v = *reinterpret_cast<const float4*>(st + QT + 2 * i);
        dp[i] = p[i] * (dp[i] - v.x);
        dp[i + 1] = p[i + 1] * (dp[i + 1] - v.y);
        dp[i + 2] = p[i + 2] * (dp[i + 2] - v.z);
        dp[i + 3] = p[i + 3] * (dp[i + 3] - v.w);
      }
      __builtin_amdgcn_sched_barrier(0);
      if (rt < w_lo || rt + 32 > w_hi) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int at = rt + row_of(i, half);
          if (at < lo || at >= hi) {
            p[i] = 0.f;
            dp[i] = 0.f;
          }
        }
      }
      priority(First());
      add_rows<T, D>(dv, Cs(buf), at_t, lane, p);
      add_rows<T, D>(dk, Qs(buf), at_t, lane, dp);
      priority(Last());
    }
    __syncthreads();
  }
  if constexpr (P > 1) {  // the other parts' sums are added to the first's, one gradient after the other
    float* x = reinterpret_cast<float*>(tiles) + wave * 32 * D + lane;
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      f32x16_t(&acc)[D / 32] = g ? dv : dk;
      if (part > 0) {
#pragma unroll
        for (int e = 0; e < D / 32; ++e)
#pragma unroll
          for (int i = 0; i < 16; ++i) x[(part - 1) * RB * D + (e * 16 + i) * 64] = acc[e][i];
      }
      __syncthreads();
      if (part == 0) {
#pragma unroll
        for (int o = 0; o < P - 1; ++o)
#pragma unroll
          for (int e = 0; e < D / 32; ++e)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[e][i] += x[o * RB * D + (e * 16 + i) * 64];
      }
      if (g == 0) __syncthreads();
    }
    if (part > 0) return;
  }
  if constexpr (P > 1) wave_fence();  // the sums have been read; their place is this wavefront's own
  T* scratch = reinterpret_cast<T*>(tiles) + wave * (P > 1 ? 32 * D * 4 / (int)sizeof(T) : 32 * S);
  static_assert(P > 1 ? 32 * D * 4 >= 32 * S * (int)sizeof(T) || sizeof(T) == 4 : kTileBytes >= RB * S * (int)sizeof(T) || sizeof(T) == 4, "rows are put together where the tiles were");
  const unsigned again = rows_where(key < s.kn && (not_finite<D>(dk) || not_finite<D>(dv)));
  const auto rows_of = [&](void* base, int64_t ld) {
    return [=](int r) -> T* { return j0 + 32 * wave + r < s.kn && !(again >> r & 1) ? static_cast<T*>(base) + (s.k0 + j0 + 32 * wave + r) * ld + head * D : nullptr; };
  };
  store_rows<T, D>(scratch, dk, a.scale, lane, rows_of(a.dk, a.ld_k));
  store_rows<T, D>(scratch, dv, 1.f, lane, rows_of(a.dv, a.ld_v));
#pragma unroll 1
  for (unsigned left = again; left; left &= left - 1) {
    const int j = j0 + 32 * wave + __builtin_ctz(left);
    key_again<T, D>(a, s, head, j, row_begin(j), row_end(j));
  }
}

// ---- launches ----------------------------------------------------------------
constexpr int kUnits = 256;  // compute units
// Blocks of 128 rows while there is one for each compute unit.  Below that, and where a sequence has on the average fewer rows than
// half a block (the lengths are not known on the host), blocks of 32 rows, whose wavefronts share out the keys.  us, 128 rows against 32:
// 130 blocks of 128 (2048 tokens, 8 heads on 2, 128 wide) 49 against 33 forward, 216 (2 x 1024 tokens, 12 heads of 64) 20 against 16; 324 of
// those 21 and 21, query gradients equal too; 516 (2 x 4096, 8 heads on 2, 128 wide) 137 against 150.
bool few_rows(const SeqAttn& a) {
  const int64_t group = a.hq / a.hk;
  return slots(a.q_rows, a.batch, (int)group, 128) * a.hk < kUnits || a.q_rows * group <= (int64_t)64 * a.batch;
}
// With fewer blocks of 32 rows than compute units keys are shared out among blocks too, up to four blocks a unit, each keeping two tiles: the
// case of single tokens (16 of them on up to 8192 keys, 8 key heads of 128: 7 parts; one would leave 112 units idle).  With a block
// for each unit a second launch that joins the parts costs more than it gives (1024 tokens, 8 heads on 2: 30 us with three parts, 27 with none).
int splits(const SeqAttn& a) {
  if (!few_rows(a) || a.q_rows == 0) return 1;
  const int64_t blocks = slots(a.q_rows, a.batch, a.hq / a.hk, 32) * a.hk, keys = (a.k_rows + a.batch - 1) / a.batch;
  return blocks >= kUnits ? 1 : (int)std::max<int64_t>(1, std::min<int64_t>({4 * kUnits / blocks, keys / 256, 32}));
}

template <class T, int D>
void forward(const SeqAttn& a, hipStream_t st) {
  const int group = a.hq / a.hk;
  if (few_rows(a)) {
    const unsigned n = (unsigned)(slots(a.q_rows, a.batch, group, 32) * a.hk);
    seq_fwd_k<T, D, 32><<<dim3(n, (unsigned)a.splits), kThreads, 0, st>>>(a);
    if (a.splits > 1) seq_join_k<T, D><<<n, kThreads, 0, st>>>(a);
  } else {
    seq_fwd_k<T, D, 128><<<(unsigned)(slots(a.q_rows, a.batch, group, 128) * a.hk), kThreads, 0, st>>>(a);
  }
}
template <class T, int D>
void backward(const SeqAttn& a, hipStream_t st) {
  const int group = a.hq / a.hk;
  if (a.q_rows) {
    if (few_rows(a)) seq_bwd_q_k<T, D, 32><<<(unsigned)(slots(a.q_rows, a.batch, group, 32) * a.hk), kThreads, 0, st>>>(a);
    else seq_bwd_q_k<T, D, 128><<<(unsigned)(slots(a.q_rows, a.batch, group, 128) * a.hk), kThreads, 0, st>>>(a);
  }
  if (!a.k_rows) return;
  const int64_t n = slots(a.k_rows, a.batch, 1, 128) * a.hk;
  constexpr bool kSmall = sizeof(T) == 2 || D < 128;  // what LDS and registers hold
  if (kSmall && n < kUnits) {
    if constexpr (kSmall) seq_bwd_k_k<T, D, 32, 4><<<(unsigned)(slots(a.k_rows, a.batch, 1, 32) * a.hk), 256, 0, st>>>(a);
  } else if (sizeof(T) == 2 && (D == 128 || n < 2 * kUnits)) {
    constexpr int P = D == 128 ? 2 : 3;
    if constexpr (sizeof(T) == 2) seq_bwd_k_k<T, D, 128, P><<<(unsigned)n, 256 * P, 0, st>>>(a);
  } else {
    if constexpr (sizeof(T) == 4 || D < 128) seq_bwd_k_k<T, D, 128, 1><<<(unsigned)n, 256, 0, st>>>(a);
  }
}

#define MREM_SEQ_DISPATCH(f)                                    \
  do {                                                          \
    if (a.dt == DT_BF16) {                                      \
      if (a.d == 32) f<bf16_t, 32>(a, st);                      \
      else if (a.d == 64) f<bf16_t, 64>(a, st);                 \
      else f<bf16_t, 128>(a, st);                               \
    } else {                                                    \
      if (a.d == 32) f<float, 32>(a, st);                       \
      else if (a.d == 64) f<float, 64>(a, st);                  \
      else f<float, 128>(a, st);                                \
    }                                                           \
  } while (0)

}  // namespace

size_t seq_attn_fwd_bytes(const SeqAttn& a) {
  const int n = splits(a);
  return n > 1 ? (size_t)n * a.hq * a.q_rows * (a.d + 2) * 4 : 0;
}
size_t seq_attn_bwd_bytes(const SeqAttn& a) { return (size_t)a.hq * a.q_rows * 8; }

void seq_attn_fwd(SeqAttn a, void* workspace, hipStream_t st) {
  a.splits = splits(a);
  a.part = static_cast<float*>(workspace);
  MREM_SEQ_DISPATCH(forward);
}
void seq_attn_bwd(SeqAttn a, void* workspace, hipStream_t st) {
  a.delta = static_cast<float*>(workspace);
  MREM_SEQ_DISPATCH(backward);
}

}  // namespace mrem
