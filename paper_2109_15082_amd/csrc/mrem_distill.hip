// Distillation from a teacher's top logits: the row's loss and its gradient in one pass over the student's logits.
//
// A row's 4 to 512 KB are read once and its gradient is written once; that bounds it.  One block takes a row and holds it in
// registers (up to 18 pieces of 16 bytes for each of 960 threads, as they lie in memory): the pieces are exponentiated as they
// arrive, each thread against a maximum of its own, the threads' sums meet once, and the gradient leaves from the same registers.
// A row that does not fit is read twice.  Read and written: 4096 rows of 30522 logits in bf16 in 127 us (3.9 TB/s; a copy reaches 5.2),
// of 128000 in 495 us (4.2 TB/s).
// The listed tokens' part is k terms a row: it is formed in 64 bits, since the rest r = 1 - sum p and the difference
// q_v - p_v of a student near its teacher lose what 32 bits hold.  Which tokens are listed lies in a bitmap in LDS, so the sum over all
// others is a sum of its own and not a difference of two nearly equal ones.  Sums have a fixed order.
#include "mrem_common.h"
#include "mrem_kernels.h"

#include <algorithm>

namespace mrem {

namespace {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

// 16 bytes of a row, at any address.  They stay packed: a register each for the values would be four times the registers
template <class T>
struct Logits {
  static constexpr int kN = 16 / sizeof(T);
  u32x4_t u;
  __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(&u, p, 16); }
  __device__ __forceinline__ float get(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(u[j]);
    else return __uint_as_float(j & 1 ? u[j >> 1] & 0xffff0000u : u[j >> 1] << 16);
  }
  // the same by another instruction: a value that is wanted twice would stay unpacked from one use to the other
  __device__ __forceinline__ float get_again(int j) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(u[j]);
    else return __uint_as_float(__builtin_amdgcn_perm(u[j >> 1], 0u, j & 1 ? 0x07060000u : 0x05040000u));
  }
};
template <class T>
__device__ __forceinline__ void store_piece(T* to, const float (&v)[16 / sizeof(T)]) {
  T o[16 / sizeof(T)];
#pragma unroll
  for (int j = 0; j < (int)(16 / sizeof(T)); ++j) o[j] = static_cast<T>(v[j]);
  __builtin_memcpy(to, o, 16);
}

// running maximum m and sums of 2^(c x - c m), over all tokens or over those not listed
struct Soft {
  float m = -INFINITY, others = 0.f;
  __device__ __forceinline__ void raise(float to, float c) {
    if (to > m) {
      others *= exp2f((m - to) * c);  // (-inf - finite) c: 0
      m = to;
    }
  }
};

__device__ __forceinline__ float exp_of(float x, float m, float c) { return __builtin_amdgcn_exp2f((x - m) * c); }

// the n (4 or 8) bits of piece `first` + i, `first` a multiple of 8
__device__ __forceinline__ unsigned listed_byte(const unsigned* bits, int first, int i, int n) {
  return n == 8 ? (bits[first / 4 + (i >> 2)] >> ((i & 3) * 8)) & 255u : (bits[first / 8 + (i >> 3)] >> ((i & 7) * 4)) & 15u;
}

template <class T>
__device__ __forceinline__ void take(Soft& s, const Logits<T>& p, unsigned bits, float c) {
  float top = p.get(0);
#pragma unroll
  for (int j = 1; j < Logits<T>::kN; ++j) top = fmaxf(top, p.get(j));
  s.raise(top, c);
  const float m = s.m == -INFINITY ? 0.f : s.m;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < Logits<T>::kN; ++j) sum += (bits >> j) & 1u ? 0.f : exp_of(p.get(j), m, c);
  s.others += sum;
}
__device__ __forceinline__ void take_one(Soft& s, float x, bool in_list, float c) {
  s.raise(x, c);
  if (!in_list) s.others += exp_of(x, s.m == -INFINITY ? 0.f : s.m, c);
}

__device__ __forceinline__ double wave_sum_d(double v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}
__device__ __forceinline__ double wave_max_d(double v) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, kWave));
  return v;
}

constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;

// 2^(i / 32)
__device__ const double kPowers[32] = {
    1.0, 1.0218971486541166, 1.0442737824274138, 1.0671404006768237,
    1.0905077326652577, 1.1143867425958924, 1.1387886347566916, 1.1637248587775775,
    1.189207115002721, 1.215247359980469, 1.241857812073484, 1.2690509571917332,
    1.2968395546510096, 1.3252366431597413, 1.3542555469368927, 1.383909881963832,
    1.4142135623730951, 1.4451808069770467, 1.4768261459394993, 1.5091644275934228,
    1.5422108254079407, 1.5759808451078865, 1.6104903319492543, 1.645755478153965,
    1.681792830507429, 1.718619298122478, 1.7562521603732995, 1.7947090750031072,
    1.8340080864093424, 1.8741676341103, 1.9152065613971474, 1.9571441241754002};

// exp and log in 64 bits, to about 1e-12: 2^(d log2 e) = 2^(n / 32) 2^t, |t| <= 1 / 64, with four terms of the series in t ln 2;
// log x = y - (1 - x e^-y) - ... from y = log x in 32 bits.  The library's polynomials hold their constants in some 60 registers
// throughout a loop, which are the row's here.
__device__ __forceinline__ double exp_d(double d) {
  const double e = d * kLog2e;
  if (!(e > -1000.0)) return e != e ? e : 0.0;
  if (e > 1000.0) return INFINITY;
  const double n = rint(e * 32.0), t = (e - n * 0.03125) * kLn2;
  const int i = (int)n;
  const double s = kPowers[i & 31];
  return ldexp(fma(s * t, fma(t, fma(t, fma(t, 1.0 / 24, 1.0 / 6), 0.5), 1.0), s), i >> 5);
}
__device__ __forceinline__ double log_d(double x) {
  const float y = logf((float)x);
  if (!(fabsf(y) < INFINITY)) return y;
  const double z = x * exp_d(-(double)y) - 1.0;
  return (double)y + z - 0.5 * z * z;
}

// what a row's list comes to: sums of p, p log p and p x / temperature; the student's listed tokens against their maximum
struct ListSums {
  double mass, self, cross, sum;
  float max;
  int twice;  // a token is listed twice
};
// a row's list in LDS: token (-1: not there), p, logit and later gradient
struct List {
  double* p;
  int* token;
  float* x;
};
constexpr int kListBytes = 16;  // an entry

// One wavefront reads row's list, marks its tokens and forms its sums in 64 bits.
template <class T>
__device__ void read_list(const DistillArg& a, int64_t row, const List& l, unsigned* bits, ListSums* out) {
  const int lane = threadIdx.x & (kWave - 1);
  const T* x = static_cast<const T*>(a.x) + row * a.ld;
  const double it = 1.0 / (double)a.temperature;
  double top = -INFINITY;
  float mx = -INFINITY;
  bool again = false;
#pragma unroll 1
  for (int i = lane; i < a.k; i += kWave) {
    const int t = a.index[row * a.k + i];
    const double z = (double)a.top[row * a.k + i] * it;
    const bool there = t >= 0 && t < a.vocab;
    l.token[i] = there ? t : -1;
    l.p[i] = z;
    l.x[i] = -INFINITY;
    if (there) {
      again |= (atomicOr(&bits[t >> 5], 1u << (t & 31)) >> (t & 31)) & 1u;
      l.x[i] = (float)x[t];
      mx = fmaxf(mx, l.x[i]);
      top = fmax(top, z);
    }
  }
  const bool twice = __any(again);
  mx = wave_max(mx);
  double log_total = 0;
  if (a.teacher_lse) {
    log_total = (double)a.teacher_lse[row];
  } else {
    top = wave_max_d(top);
    const double ref = top == -INFINITY ? 0.0 : top;
    double sum = 0;
#pragma unroll 1
    for (int i = lane; i < a.k; i += kWave)
      if (l.token[i] >= 0) sum += exp_d(l.p[i] - ref);
    log_total = ref + log_d(wave_sum_d(sum));
  }
  const bool none = !a.teacher_lse && log_total == -INFINITY;  // a list of -inf only has no probabilities
  const double ref = mx == -INFINITY ? 0.0 : (double)mx;
  double mass = 0, self = 0, cross = 0, sum = 0;
#pragma unroll 1
  for (int i = lane; i < a.k; i += kWave) {
    const int t = l.token[i];
    const double lg = l.p[i] - log_total, xi = (double)l.x[i], pr = t >= 0 && !none ? exp_d(lg) : 0.0;
    bool first = t >= 0;  // a token listed twice is one of the student's: its first entry counts
    if (twice && first)
      for (int j = 0; j < i; ++j) first = first && l.token[j] != t;
    if (first) sum += exp_d((xi - ref) * it);
    if (pr != 0.0) {
      mass += pr;
      self += pr * lg;
      cross += pr * xi * it;
    }
    l.p[i] = pr;
  }
  mass = wave_sum_d(mass);
  self = wave_sum_d(self);
  cross = wave_sum_d(cross);
  sum = wave_sum_d(sum);
  if (lane == 0) *out = ListSums{mass, self, cross, sum, mx, twice};
}

// wavefronts a SIMD, by which the registers of a thread are bounded: 80 of them up to 9 pieces, else 128
constexpr int kDistillWaves(int threads, int pieces) { return threads > 512 || pieces > 9 ? 4 : 6; }

// What the list's wavefront tells the others about a row.
struct Told {
  float max, scale;  // gradient of a token not listed: scale 2^(c (x - max))
};

// A block takes every gridDim.x-th row.  Its first wavefront works on the lists, the others, D threads, on the rows' pieces; the
// two are different programs that meet at three barriers a row, so that neither's registers are the other's.
// NP: pieces of a row that a thread holds; 0: as many as there are, read again for the gradient.  While a row's gradient leaves the
// registers, the next row's pieces come in behind it and the first wavefront reads the next row's list.
template <class T, int D, int NP>
__global__ __launch_bounds__(D + kWave, kDistillWaves(D, NP)) void distill_k(DistillArg a) {
  constexpr int N = Logits<T>::kN, W = D / kWave;
  extern __shared__ unsigned lds[];  // bitmap, then two lists
  __shared__ ListSums sums[2];
  __shared__ Told told;
  __shared__ float part_m[W], part_s[W];
  const int words = ((a.vocab + 127) / 128) * 4, pieces = a.vocab / N, tail = a.vocab - pieces * N;
  unsigned* bits = lds;
  const float c = (float)(kLog2e / (double)a.temperature);
  const auto weight_of = [&](int64_t r) { return r < a.rows ? a.weight ? a.weight[r] : 1.f : 0.f; };
  int64_t row = blockIdx.x;
  float weight = weight_of(row);
  for (int i = threadIdx.x; i < words; i += D + kWave) bits[i] = 0u;
  __syncthreads();

  if (threadIdx.x < kWave) {
    const int lane = threadIdx.x;
    const double it = 1.0 / (double)a.temperature;
    const auto list = [&](int b) {
      double* p = reinterpret_cast<double*>(lds + words) + b * 2 * a.k;
      int* t = reinterpret_cast<int*>(p + a.k);
      return List{p, t, reinterpret_cast<float*>(t + a.k)};
    };
    if (weight != 0.f) read_list<T>(a, row, list(0), bits, &sums[0]);
    __syncthreads();
    for (int b = 0; row < a.rows; row += gridDim.x, b ^= 1) {
      const float next_weight = weight_of(row + gridDim.x);
      const List l = list(b);
      __syncthreads();  // the wavefronts' parts are there
      if (weight != 0.f) {
        const ListSums ls = sums[b];
        const float pm = lane < W ? part_m[lane] : -INFINITY, m = fmaxf(wave_max(pm), ls.max), mm = m == -INFINITY ? 0.f : m;
        const double others = (double)wave_sum(lane < W ? part_s[lane] * exp2f((pm - mm) * c) : 0.f);
        const double total = others + ls.sum * exp_d((double)((ls.max == -INFINITY ? mm : ls.max) - mm) * it);
        const double rest = a.teacher_lse ? fmax(0.0, 1.0 - ls.mass) : 0.0;
        const double f = (double)weight * a.scale * it, each = (ls.mass + rest) / total;
        if (lane == 0) told = Told{mm, (float)(f * (each - (rest > 0.0 ? rest / others : 0.0)))};
        __syncthreads();
        if (lane == 0) {
          const double log_total = log_d(total);
          double loss = ls.self - ls.cross + (ls.mass == 0.0 ? 0.0 : ls.mass * ((double)mm * it + log_total));
          if (rest > 0.0) loss += rest * (log_d(rest) - log_d(others) + log_total);
          a.loss_rows[row] = (float)loss;
        }
        // the list's gradients, which are written when the row is; its marks are taken back
#pragma unroll 1
        for (int i = lane; i < a.k; i += kWave) {
          const int t = l.token[i];
          if (t < 0) continue;
          bits[t >> 5] = 0u;
          double pr = l.p[i];
          if (ls.twice) {  // all entries of the token form the same sum
            pr = 0;
            for (int j = 0; j < a.k; ++j) pr += l.token[j] == t ? l.p[j] : 0.0;
          }
          l.x[i] = (float)(f * (each * exp_d(((double)l.x[i] - (double)mm) * it) - pr));
        }
      } else {
        __syncthreads();
        if (lane == 0) a.loss_rows[row] = 0.f;
      }
      if (next_weight != 0.f) read_list<T>(a, row + gridDim.x, list(b ^ 1), bits, &sums[b ^ 1]);
      __syncthreads();  // the row's pieces are written
      if (a.grad && weight != 0.f) {
        T* g = static_cast<T*>(a.grad) + row * a.ld_grad;
#pragma unroll 1
        for (int i = lane; i < a.k; i += kWave)
          if (l.token[i] >= 0) g[l.token[i]] = static_cast<T>(l.x[i]);
      }
      weight = next_weight;
    }
    return;
  }

  const unsigned tid = threadIdx.x - kWave;
  const int wave = tid / kWave, lane = tid & (kWave - 1);
  Logits<T> p[NP > 0 ? NP : 1];
  float xt = -INFINITY;  // a value behind the pieces
  // Every load is taken, so that old and new pieces share their registers: with nothing to fetch, from a place that all share.
  const auto fetch = [&](int i, const T* x, bool there) {
    const T* nowhere = reinterpret_cast<const T*>(kPowers);
    p[i].load(there && (int)tid < pieces - i * D ? x + i * (D * N) + tid * N : nowhere);
  };
  const auto fetch_tail = [&](const T* x, bool there) { xt = there && (int)tid < tail ? (float)x[pieces * N + tid] : -INFINITY; };
  {
    const T* x = static_cast<const T*>(a.x) + row * a.ld;
#pragma unroll
    for (int i = 0; i < NP; ++i) fetch(i, x, weight != 0.f);
    fetch_tail(x, weight != 0.f);
  }
  __syncthreads();
  for (; row < a.rows; row += gridDim.x) {
    const int64_t next = row + gridDim.x;
    const float next_weight = weight_of(next);
    const bool more = next_weight != 0.f;
    const T* x = static_cast<const T*>(a.x) + row * a.ld;
    T* g = a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad : nullptr;
    const bool live = weight != 0.f;  // otherwise nothing of the row is read
    if (g && !live) {
      const float zero[N] = {};
      for (int i = tid; i < pieces; i += D) store_piece(g + (size_t)i * N, zero);
      if ((int)tid < tail) g[pieces * N + tid] = static_cast<T>(0.f);
      g = nullptr;
    }
    // the sum over the tokens not listed
    if (live) {
      Soft s;
      if constexpr (NP > 0) {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          if ((int)tid < pieces - i * D) take(s, p[i], listed_byte(bits, i * D, tid, N), c);
          __builtin_amdgcn_sched_barrier(0);  // piece by piece: all at once need more registers than there are
        }
      } else {
#pragma unroll 4
        for (int at = tid; at < pieces; at += D) {
          Logits<T> q;
          q.load(x + (size_t)at * N);
          take(s, q, listed_byte(bits, 0, at, N), c);
        }
      }
      if ((int)tid < tail) {
        const int t = pieces * N + tid;
        take_one(s, xt, (bits[t >> 5] >> (t & 31)) & 1u, c);
      }
      {
        const float m = wave_max(s.m), ref = m == -INFINITY ? 0.f : m;
        const float sum = wave_sum(s.others * exp2f((s.m - ref) * c));
        if (lane == 0) {
          part_m[wave] = m;
          part_s[wave] = sum;
        }
      }
    }
    __syncthreads();
    __syncthreads();
    const float mm = told.max, k = told.scale;
    if constexpr (NP > 0) {
      const T* xn = static_cast<const T*>(a.x) + next * a.ld;
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        if (g && (int)tid < pieces - i * D) {
          float v[N];
#pragma unroll
          for (int j = 0; j < N; ++j) v[j] = k * exp_of(p[i].get_again(j), mm, c);
          store_piece(g + i * (D * N) + tid * N, v);
        }
        fetch(i, xn, more);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else if (g) {
#pragma unroll 4
      for (int at = tid; at < pieces; at += D) {
        Logits<T> q;
        q.load(x + (size_t)at * N);
        float v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = k * exp_of(q.get(j), mm, c);
        store_piece(g + (size_t)at * N, v);
      }
    }
    if (g && (int)tid < tail) g[pieces * N + tid] = static_cast<T>(k * exp_of(xt, mm, c));
    fetch_tail(static_cast<const T*>(a.x) + next * a.ld, more);
    __syncthreads();
    weight = next_weight;
  }
}

__global__ __launch_bounds__(1024) void distill_total_k(const float* rows, const float* weight, int64_t n, float scale, float* out) {
  __shared__ double red[16];
  double t = 0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) {
    const float w = weight ? weight[i] : 1.f;
    if (w != 0.f) t += (double)w * rows[i];
  }
  t = wave_sum_d(t);
  if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = t;
  __syncthreads();
  if (threadIdx.x > 0) return;
  t = 0;
  for (int i = 0; i < 16; ++i) t += red[i];
  *out = (float)(t * scale);
}

template <class T, int D, int NP>
void launch(const DistillArg& a, hipStream_t st) {
  const size_t lds = (size_t)((a.vocab + 127) / 128) * 16 + (size_t)a.k * 2 * kListBytes;
  if (lds > 48 * 1024) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&distill_k<T, D, NP>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  // as many blocks as 256 compute units hold at a time
  const int64_t held = 256 * (kDistillWaves(D, NP) * 4 / (D / kWave + 1));
  distill_k<T, D, NP><<<(unsigned)std::min(a.rows, held), D + kWave, lds, st>>>(a);
}

template <class T>
void launch_rows(const DistillArg& a, hipStream_t st) {
  const int pieces = a.vocab / Logits<T>::kN;
  if (pieces <= 192 * 6) launch<T, 192, 6>(a, st);
  else if (pieces <= 448 * 9) launch<T, 448, 9>(a, st);
  else if (pieces <= 448 * 18) launch<T, 448, 18>(a, st);
  else if (pieces <= 960 * 18) launch<T, 960, 18>(a, st);
  else launch<T, 960, 0>(a, st);
}

}  // namespace

void distill_loss(int dt, const DistillArg& a, hipStream_t st) {
  if (a.rows > 0) {
    if (dt == DT_BF16) launch_rows<bf16_t>(a, st);
    else launch_rows<float>(a, st);
  }
  if (a.loss_out) distill_total_k<<<1, 1024, 0, st>>>(a.loss_rows, a.weight, a.rows, a.scale, a.loss_out);
}

}  // namespace mrem
