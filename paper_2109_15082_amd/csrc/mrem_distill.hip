// Distillation from a teacher's top logits: the row's loss and its gradient in one pass over the student's logits.
//
// A row's 4 to 512 KB are read once and its gradient is written once; that bounds it.  One block takes a row and holds it in
// registers (up to 16 pieces of 16 bytes for each of 1024 threads): the pieces are exponentiated as they arrive, each thread
// against a maximum of its own, the threads' sums meet once, and the gradient leaves from the same registers.  A row that does not
// fit is read twice.
// The listed tokens' part is k terms a row: it is formed in 64 bits, since the rest r = 1 - sum p and the difference
// q_v - p_v of a student near its teacher lose what 32 bits hold.  Which tokens are listed lies in a bitmap in LDS, so the sum over all
// others is a sum of its own and not a difference of two nearly equal ones.  Sums have a fixed order.
#include "mrem_common.h"
#include "mrem_kernels.h"

#include <algorithm>

namespace mrem {

namespace {

template <class T>
struct Logits {  // 16 bytes, at any address
  static constexpr int kN = 16 / sizeof(T);
  T v[kN];
  __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(v, p, 16); }
  __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(p, v, 16); }
};

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

template <class T, int BT>
struct Row {
  const T* x;
  T* g;
  int vocab, pieces, tail;  // tail: values behind the last piece, at most one a thread
  float c;                  // log2(e) / temperature
  const unsigned* listed;   // bitmap
};

__device__ __forceinline__ unsigned listed_byte(const unsigned* bits, int piece, int n) {
  // the n (4 or 8) bits of a piece
  return n == 8 ? (bits[piece >> 2] >> ((piece & 3) * 8)) & 255u : (bits[piece >> 3] >> ((piece & 7) * 4)) & 15u;
}

template <class T>
__device__ __forceinline__ void take(Soft& s, const Logits<T>& p, unsigned bits, float c) {
  float top = (float)p.v[0];
#pragma unroll
  for (int j = 1; j < Logits<T>::kN; ++j) top = fmaxf(top, (float)p.v[j]);
  s.raise(top, c);
  const float m = s.m == -INFINITY ? 0.f : s.m;
  float sum = 0.f;
#pragma unroll
  for (int j = 0; j < Logits<T>::kN; ++j) sum += (bits >> j) & 1u ? 0.f : exp_of((float)p.v[j], m, c);
  s.others += sum;
}
__device__ __forceinline__ void take_one(Soft& s, float x, bool in_list, float c) {
  s.raise(x, c);
  if (!in_list) s.others += exp_of(x, s.m == -INFINITY ? 0.f : s.m, c);
}

template <int BT>
__device__ __forceinline__ double block_sum_d(double v, double* scratch) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  double t = 0;
#pragma unroll 1
  for (int i = 0; i < BT / kWave; ++i) t += scratch[i];
  return t;
}
template <int BT>
__device__ __forceinline__ double block_max_d(double v, double* scratch) {
#pragma unroll
  for (int o = kWave / 2; o > 0; o >>= 1) v = fmax(v, __shfl_xor(v, o, kWave));
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) scratch[threadIdx.x / kWave] = v;
  __syncthreads();
  double t = scratch[0];
  for (int i = 1; i < BT / kWave; ++i) t = fmax(t, scratch[i]);
  return t;
}

constexpr double kLog2e = 1.4426950408889634074;

// NP: pieces of a row that a thread holds; 0: as many as there are, read again for the gradient
template <class T, int BT, int NP>
__global__ __launch_bounds__(BT) void distill_k(DistillArg a) {
  constexpr int N = Logits<T>::kN;
  extern __shared__ unsigned lds[];  // bitmap, then the list: p (64 bits), token, x
  __shared__ double red[BT / kWave];
  __shared__ float redf[17];
  __shared__ int twice;
  const int64_t row = blockIdx.x;
  const int words = ((a.vocab + 127) / 128) * 4;
  unsigned* bits = lds;
  double* lp = reinterpret_cast<double*>(lds + words);
  int* lt = reinterpret_cast<int*>(lp + a.k);
  const T* x = static_cast<const T*>(a.x) + row * a.ld;
  T* g = a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad : nullptr;
  const int pieces = a.vocab / N, tail = a.vocab - pieces * N;
  const float weight = a.weight ? a.weight[row] : 1.f;
  if (weight == 0.f) {  // nothing of the row is read
    if (threadIdx.x == 0) a.loss_rows[row] = 0.f;
    if (g) {
      Logits<T> z;
#pragma unroll
      for (int j = 0; j < N; ++j) z.v[j] = static_cast<T>(0.f);
      for (int i = threadIdx.x; i < pieces; i += BT) z.store(g + (size_t)i * N);
      if ((int)threadIdx.x < tail) g[pieces * N + threadIdx.x] = static_cast<T>(0.f);
    }
    return;
  }
  // the row's pieces are on their way while the list is worked on
  Logits<T> p[NP > 0 ? NP : 1];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int at = threadIdx.x + i * BT;
    if (at < pieces) p[i].load(x + (size_t)at * N);
  }
  const float xt = (int)threadIdx.x < tail ? (float)x[pieces * N + threadIdx.x] : -INFINITY;

  for (int i = threadIdx.x; i < words; i += BT) bits[i] = 0u;
  if (threadIdx.x == 0) twice = 0;
  __syncthreads();
  const double it = 1.0 / (double)a.temperature;
  // the teacher's probabilities; a thread takes every BT-th entry (one, up to 1024 threads)
  double top = -INFINITY;
#pragma unroll 1
  for (int i = threadIdx.x; i < a.k; i += BT) {
    const int t = a.index[row * a.k + i];
    const bool there = t >= 0 && t < a.vocab;
    lt[i] = there ? t : -1;
    lp[i] = (double)a.top[row * a.k + i] * it;
    if (there) {
      if (atomicOr(&bits[t >> 5], 1u << (t & 31)) >> (t & 31) & 1u) twice = 1;
      top = fmax(top, lp[i]);
    }
  }
  double log_total = 0;
  if (a.teacher_lse) {
    log_total = (double)a.teacher_lse[row];
  } else {
    top = block_max_d<BT>(top, red);
    double sum = 0;
  #pragma unroll 1
  for (int i = threadIdx.x; i < a.k; i += BT)
      if (lt[i] >= 0) sum += exp(lp[i] - (top == -INFINITY ? 0.0 : top));
    sum = block_sum_d<BT>(sum, red);
    log_total = (top == -INFINITY ? 0.0 : top) + log(sum);
  }
  double mass = 0, self = 0, cross = 0;  // sums of p, p log p, p x
  double own_x = 0;
#pragma unroll 1
  for (int i = threadIdx.x; i < a.k; i += BT) {
    // a list of -inf only has no probabilities
    double lg = lp[i] - log_total, pr = lt[i] >= 0 && (a.teacher_lse || log_total != -INFINITY) ? exp(lg) : 0.0;
    if (lt[i] >= 0) own_x = (double)(float)x[lt[i]];
    if (pr != 0.0) {
      mass += pr;
      self += pr * lg;
      cross += pr * own_x * it;
    }
    lp[i] = pr;
  }
  __syncthreads();  // bitmap and list are whole

  // sums over the row
  const float c = (float)(kLog2e * it);
  Soft s;
  if constexpr (NP > 0) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int at = threadIdx.x + i * BT;
      if (at < pieces) take(s, p[i], listed_byte(bits, at, N), c);
    }
  } else {
    for (int at = threadIdx.x; at < pieces; at += BT) {
      p[0].load(x + (size_t)at * N);
      take(s, p[0], listed_byte(bits, at, N), c);
    }
  }
  if ((int)threadIdx.x < tail) {
    const int t = pieces * N + threadIdx.x;
    take_one(s, xt, bits[t >> 5] >> (t & 31) & 1u, c);
  }
  const float m = block_max(s.m, redf), mm = m == -INFINITY ? 0.f : m;
  const double others = block_sum_d<BT>((double)(s.others * exp2f((s.m == -INFINITY ? -INFINITY : s.m - mm) * c)), red);
  // a token listed twice is one token of the student's: its first entry counts
  double mine = 0;
#pragma unroll 1
  for (int i = threadIdx.x; i < a.k; i += BT) {
    const int t = lt[i];
    bool first = t >= 0;
    if (first && twice)
      for (int j = 0; j < i; ++j) first = first && lt[j] != t;
    if (first) mine += exp(((double)(float)x[t] - (double)mm) * it);
  }
  const double total = others + block_sum_d<BT>(mine, red);
  mass = block_sum_d<BT>(mass, red);
  self = block_sum_d<BT>(self, red);
  cross = block_sum_d<BT>(cross, red);
  const double log_z = (double)mm * it + log(total);
  const double rest = a.teacher_lse ? fmax(0.0, 1.0 - mass) : 0.0;
  const double share = others / total;  // the student's probability of all tokens not listed
  if (threadIdx.x == 0) {
    double loss = self - cross + mass * log_z;
    if (mass == 0.0) loss = 0.0;
    if (rest > 0.0) loss += rest * (log(rest) - log(share));
    if (mass != mass) loss = mass;
    a.loss_rows[row] = (float)loss;
  }
  if (!g) return;

  const double f = (double)weight * a.scale * it;
  const float k_others = (float)(f * (mass + rest - (rest > 0.0 ? rest / share : 0.0)) / total);
  const double k_listed = f * (mass + rest) / total;
  // the list's gradients before any value of the row is overwritten (grad may be the logits)
  double mine_g[kDistillMaxK / BT > 0 ? kDistillMaxK / BT : 1];
#pragma unroll
  for (int e = 0; e < (kDistillMaxK / BT > 0 ? kDistillMaxK / BT : 1); ++e) {
    const int i = threadIdx.x + e * BT;
    mine_g[e] = 0;
    if (i < a.k && lt[i] >= 0) {
      double pr = lp[i];
      if (twice) {  // all entries of the token form the same sum
        pr = 0;
        for (int j = 0; j < a.k; ++j) pr += lt[j] == lt[i] ? lp[j] : 0.0;
      }
      mine_g[e] = k_listed * exp(((double)(float)x[lt[i]] - (double)mm) * it) - f * pr;
    }
  }
  __syncthreads();
  if constexpr (NP > 0) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int at = threadIdx.x + i * BT;
      if (at < pieces) {
#pragma unroll
        for (int j = 0; j < N; ++j) p[i].v[j] = static_cast<T>(k_others * exp_of((float)p[i].v[j], mm, c));
        p[i].store(g + (size_t)at * N);
      }
    }
  } else {
    for (int at = threadIdx.x; at < pieces; at += BT) {
      p[0].load(x + (size_t)at * N);
#pragma unroll
      for (int j = 0; j < N; ++j) p[0].v[j] = static_cast<T>(k_others * exp_of((float)p[0].v[j], mm, c));
      p[0].store(g + (size_t)at * N);
    }
  }
  if ((int)threadIdx.x < tail) g[pieces * N + threadIdx.x] = static_cast<T>(k_others * exp_of(xt, mm, c));
  __syncthreads();  // the block's own writes of the row are in order before these
#pragma unroll
  for (int e = 0; e < (kDistillMaxK / BT > 0 ? kDistillMaxK / BT : 1); ++e) {
    const int i = threadIdx.x + e * BT;
    if (i < a.k && lt[i] >= 0) g[lt[i]] = static_cast<T>((float)mine_g[e]);
  }
}

__global__ __launch_bounds__(1024) void distill_total_k(const float* rows, const float* weight, int64_t n, float scale, float* out) {
  __shared__ double red[16];
  double t = 0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) {
    const float w = weight ? weight[i] : 1.f;
    if (w != 0.f) t += (double)w * rows[i];
  }
  t = block_sum_d<1024>(t, red);
  if (threadIdx.x == 0) *out = (float)(t * scale);
}

template <class T, int BT, int NP>
void launch(const DistillArg& a, hipStream_t st) {
  const size_t lds = (size_t)((a.vocab + 127) / 128) * 16 + (size_t)a.k * 12;
  if (lds > 48 * 1024) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(&distill_k<T, BT, NP>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  distill_k<T, BT, NP><<<(unsigned)a.rows, BT, lds, st>>>(a);
}

template <class T>
void launch_rows(const DistillArg& a, hipStream_t st) {
  const int pieces = a.vocab / Logits<T>::kN;
  if (pieces <= 256 * 4) launch<T, 256, 4>(a, st);
  else if (pieces <= 1024 * 2) launch<T, 1024, 2>(a, st);
  else if (pieces <= 1024 * 4) launch<T, 1024, 4>(a, st);
  else if (pieces <= 1024 * 8) launch<T, 1024, 8>(a, st);
  else if (pieces <= 1024 * 16) launch<T, 1024, 16>(a, st);
  else launch<T, 1024, 0>(a, st);
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
