// Rotary positions: the first values of every head are turned in pairs by position * frequency.
//
// Each value is read and written once, so memory bounds it (8192 rows, 40 heads of 128 in bf16: 37 us, 4.5 TB/s; a copy reaches 5.2).  A block takes one to four rows: its threads first form the sine and
// cosine of every pair of those rows, which all heads share, and then walk the rows' heads in pieces of 16 bytes (two of them
// where a pair's halves lie apart).  A position times a frequency needs more than 32 bits as soon as the angle has passed some
// thousand turns, so the angle is formed in 64 bits in units of turns, and what is left of a whole turn is rounded to 32.
#include "mrem_common.h"
#include "mrem_kernels.h"

#include <algorithm>

namespace mrem {

namespace {

constexpr int kRotaryThreads = 256, kRotaryRows = 4, kRotaryPairs = 256;  // of a block; pairs a head: 512 / 2

struct RotaryArg {
  const void* x;
  void* y;
  int64_t rows, ld_x, ld_y, seq;
  const double* freq;
  const int32_t* positions;
  int heads, dim, rotary_dim, block_rows;
  float amplitude, sign;
};

template <class T>
struct Piece {  // 16 bytes
  static constexpr int kN = 16 / sizeof(T);
  T v[kN];
};

// sine and cosine, times the amplitude, of the pairs of a block's rows
__device__ __forceinline__ void form_angles(const RotaryArg& a, float2 (*cs)[kRotaryPairs], int64_t row0, int n) {
  const int pairs = a.rotary_dim / 2;
  for (int i = threadIdx.x; i < n * pairs; i += kRotaryThreads) {
    const int r = i / pairs, p = i - r * pairs;
    const int64_t t = row0 + r;
    const double at = a.positions ? (double)a.positions[t] : (double)(t % a.seq);
    const double turns = at * a.freq[p] * 0.15915494309189533577;
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    cs[r][p] = make_float2(c * a.amplitude, s * a.amplitude * a.sign);
  }
}

// LAYOUT 0: halves apart, in pieces (rotary_dim / 2 and head_dim multiples of a piece); 1: neighbouring pairs, in pieces
// (head_dim a multiple of a piece); 2, 3: the same two value by value, for all other sizes
template <class T, int LAYOUT>
__global__ __launch_bounds__(kRotaryThreads) void rotary_k(RotaryArg a) {
  constexpr int N = Piece<T>::kN;
  __shared__ float2 cs[kRotaryRows][kRotaryPairs];
  const int half = a.rotary_dim / 2;
  const bool copy = a.x != a.y;
  // what a thread takes at a time: one or two pieces, a pair, or a value behind the pairs
  const int items = LAYOUT == 0 ? (half + (copy ? a.dim - a.rotary_dim : 0)) / N : LAYOUT == 1 ? a.dim / N : half + (copy ? a.dim - a.rotary_dim : 0);
  const unsigned per_row = (unsigned)(items * a.heads);
  for (int64_t row0 = (int64_t)blockIdx.x * a.block_rows; row0 < a.rows; row0 += (int64_t)gridDim.x * a.block_rows) {
    const int n = (int)min((int64_t)a.block_rows, a.rows - row0);
    form_angles(a, cs, row0, n);
    __syncthreads();
    for (int r = 0; r < n; ++r) {
      const T* xr = static_cast<const T*>(a.x) + (row0 + r) * a.ld_x;
      T* yr = static_cast<T*>(a.y) + (row0 + r) * a.ld_y;
      for (unsigned i = threadIdx.x; i < per_row; i += kRotaryThreads) {
        const unsigned h = i / (unsigned)items;
        const int c = (int)(i - h * (unsigned)items);
        const T* x = xr + h * (unsigned)a.dim;
        T* y = yr + h * (unsigned)a.dim;
        if constexpr (LAYOUT == 0) {
          if (c * N < half) {
            Piece<T> u = *reinterpret_cast<const Piece<T>*>(__builtin_assume_aligned(x + c * N, 16));
            Piece<T> w = *reinterpret_cast<const Piece<T>*>(__builtin_assume_aligned(x + half + c * N, 16));
#pragma unroll
            for (int j = 0; j < N; ++j) {
              const float2 t = cs[r][c * N + j];
              const float p = (float)u.v[j], q = (float)w.v[j];
              u.v[j] = static_cast<T>(p * t.x - q * t.y);
              w.v[j] = static_cast<T>(q * t.x + p * t.y);
            }
            *reinterpret_cast<Piece<T>*>(__builtin_assume_aligned(y + c * N, 16)) = u;
            *reinterpret_cast<Piece<T>*>(__builtin_assume_aligned(y + half + c * N, 16)) = w;
          } else {
            const int at = half + c * N;  // rotary_dim + (c * N - half)
            *reinterpret_cast<Piece<T>*>(__builtin_assume_aligned(y + at, 16)) = *reinterpret_cast<const Piece<T>*>(__builtin_assume_aligned(x + at, 16));
          }
        } else if constexpr (LAYOUT == 1) {
          if (c * N >= a.rotary_dim && !copy) continue;
          Piece<T> u = *reinterpret_cast<const Piece<T>*>(__builtin_assume_aligned(x + c * N, 16));
#pragma unroll
          for (int j = 0; j < N; j += 2) {
            const int pair = (c * N + j) / 2;
            if (pair >= half) break;
            const float2 t = cs[r][pair];
            const float p = (float)u.v[j], q = (float)u.v[j + 1];
            u.v[j] = static_cast<T>(p * t.x - q * t.y);
            u.v[j + 1] = static_cast<T>(q * t.x + p * t.y);
          }
          *reinterpret_cast<Piece<T>*>(__builtin_assume_aligned(y + c * N, 16)) = u;
        } else {
          if (c < half) {
            const int at = LAYOUT == 3 ? 2 * c : c, to = LAYOUT == 3 ? 2 * c + 1 : c + half;
            const float2 t = cs[r][c];
            const float p = (float)x[at], q = (float)x[to];
            y[at] = static_cast<T>(p * t.x - q * t.y);
            y[to] = static_cast<T>(q * t.x + p * t.y);
          } else {
            y[half + c] = x[half + c];
          }
        }
      }
    }
    __syncthreads();
  }
}

template <class T>
void launch_rotary(const RotaryArg& a, bool interleaved, hipStream_t st) {
  constexpr int N = Piece<T>::kN;
  const unsigned blocks = (unsigned)std::min<int64_t>((a.rows + a.block_rows - 1) / a.block_rows, 1 << 20);
  const bool rows_fit = a.ld_x % N == 0 && a.ld_y % N == 0 && a.dim % N == 0;
  if (interleaved) {
    if (rows_fit) rotary_k<T, 1><<<blocks, kRotaryThreads, 0, st>>>(a);
    else rotary_k<T, 3><<<blocks, kRotaryThreads, 0, st>>>(a);
  } else {
    if (rows_fit && a.rotary_dim / 2 % N == 0) rotary_k<T, 0><<<blocks, kRotaryThreads, 0, st>>>(a);
    else rotary_k<T, 2><<<blocks, kRotaryThreads, 0, st>>>(a);
  }
}

}  // namespace

void rotary(int dt, const void* x, void* y, int64_t rows, int heads, int dim, int64_t ld_x, int64_t ld_y, int rotary_dim, bool interleaved,
            float amplitude, float sign, const double* freq, const int32_t* positions, int64_t seq, hipStream_t st) {
  RotaryArg a{x, y, rows, ld_x, ld_y, seq, freq, positions, heads, dim, rotary_dim, 1, amplitude, sign};
  // four rows a block once that still leaves a block for each of the 256 compute units: fewer waits for the angles
  a.block_rows = rows >= kRotaryRows * 256 ? kRotaryRows : 1;
  if (dt == DT_BF16) launch_rotary<bf16_t>(a, interleaved, st);
  else launch_rotary<float>(a, interleaved, st);
}

}  // namespace mrem
