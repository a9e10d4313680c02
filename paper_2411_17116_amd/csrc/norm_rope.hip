// Queries and keys that are normed per head and then rotated, with positions on one or several axes; keys and values may go on to a cache, in the
// storage type or in four bits.  One kernel makes all of it in one pass, as rope.hip's does for the rotation alone: a workgroup owns TT tokens, whose d / 2 angles
// are evaluated once, in double precision, into LDS, and a thread keeps one (token, pair of 16-byte chunks) and walks the token's rows.
//   * The lanes that hold a row (8 or 16, neighbours) add up its squares; x r w with r = 1 / sqrt(mean x^2 + eps) takes the place of x, in fp32, and the result is
//     rounded once.  A four-bit row is made of the rounded values, so that it is what the steps one after the other would file.
//   * Bound by HBM: 32768 tokens of 32 / 8 heads, 671 MB, 115 us = 5.8 TB/s (a copy: 4.9); one token 4.5 us, a launch.
//   * One row at a time and a thread's weights and its first row requested ahead of the angles, so that nothing on a row's way waits for more than the row.
//     us for 32768 tokens, two sequences of 20011 with positions on three axes, and 9000 in fp32: 133 / 170 / 70 with three rows at once and weights loaded
//     at each, 134 / 162 / 64 with the weights ahead, 120 / 147 / 65 with two rows, 115 / 140 / 66 with one; the row behind requested early 122 / 150 / 66.
//   * Plain stores: streaming ones take 110 us for the 32768 tokens, 7.0 for 9.0 for 2000, but what reads the result next then finds less of it in the
//     caches (a reduction behind 2000 tokens: 44 us for both instead of 40, behind 8000 85 instead of 74).
#include "rotary.h"
#include "q4.h"

namespace star {

namespace {

#define INLINE __attribute__((always_inline))

constexpr int THREADS = 256;

template <bool Q4> struct Rows4 { Q4Rows q4; };      // where K and V go
template <> struct Rows4<false> {};
template <bool Q4>
struct NormArgs : Rows4<Q4> {
  const void* Q;                // [B, T, H, d] -> Yq, same layout (may be Q)
  void* Yq;
  const void* K;                // [B, T, Hkv, d] -> Yk, same layout (may be K), or (cached) rows [dst_row, dst_row + T) of Yk [B, Hkv, cap, d]
  const void* V;                // -> Vc as it is, the same rows; null: none
  void* Yk;
  void* Vc;
  const int64_t* positions;     // [B, T, n_axes] or null: token t at pos0 + t
  const void* q_norm;           // [d] or null
  const void* k_norm;
  uint64_t axis[2];             // two bits per frequency
  double log2_theta;
  int64_t cap, dst_row, pos0;
  uint32_t n_tokens, total;     // T, B T
  uint32_t first;               // first token of the launch
  int32_t H, Hkv;
  float eps;
  int16_t n_axes, cached;
  unsigned int* clear;          // eight counters to zero for the launch behind this one, or null
};

// x if `first`, else y, of two arguments: bit by bit, since the compiler makes a choice of two arguments one load from a chosen
// address, whose wait is one for every row requested before it.
template <typename P>
__device__ __forceinline__ P* pick(bool first, P* x, P* y) {
  const uint64_t m = -(uint64_t)first;
  return (P*)(((uint64_t)x & m) | ((uint64_t)y & ~m));
}

template <typename T, int half, int TT, bool Q4>
__global__ __launch_bounds__(THREADS) void norm_rope_kernel(NormArgs<Q4> a) {
  constexpr int N = Chunk<T>::N;
  typedef typename Chunk<T>::vec vec;
  __shared__ float cs_all[TT][half], sn_all[TT][half];
  const int tid = threadIdx.x;
  const uint32_t tok0 = a.first + blockIdx.x * TT;
  if (a.clear && blockIdx.x == 0 && tid < 8) a.clear[tid] = 0u;
  constexpr int cpr = half / N;                    // chunk pairs per row: 8 or 16
  const int c = (tid % cpr) * N, k = (tid / cpr) % TT, slot = tid / (cpr * TT), n_slots = THREADS / (cpr * TT);
  const uint32_t tok = tok0 + k;
  const uint32_t beta = tok / a.n_tokens, t = tok % a.n_tokens;
  constexpr size_t d = 2 * half;
  const size_t cache0 = ((size_t)beta * a.Hkv * a.cap + a.dst_row + t) * d + c;
  const int n_rows = a.H + (a.V ? 2 : 1) * a.Hkv;
  vec lo, hi;
  T* dst;
  const auto request = [&](int h) {
    const T* src;
    if (h < a.H) {
      src = (const T*)a.Q + ((size_t)tok * a.H + h) * d + c;
      dst = (T*)a.Yq + ((size_t)tok * a.H + h) * d + c;
    } else {
      const bool v = h >= a.H + a.Hkv;
      const int g = h - a.H - (v ? a.Hkv : 0);
      src = (const T*)pick(v, a.V, a.K) + ((size_t)tok * a.Hkv + g) * d + c;
      dst = (T*)pick(v, a.Vc, a.Yk) + cache0 + (size_t)g * a.cap * d;
      if constexpr (!Q4)
        if (!v && !a.cached) dst = (T*)a.Yk + ((size_t)tok * a.Hkv + g) * d + c;
    }
    lo = *(const vec*)src;
    hi = *(const vec*)(src + half);
  };
  vec q_norm[2] = {}, k_norm[2] = {};              // the weights of this thread's chunks
  if (a.q_norm) { q_norm[0] = *(const vec*)((const T*)a.q_norm + c); q_norm[1] = *(const vec*)((const T*)a.q_norm + half + c); }
  if (a.k_norm) { k_norm[0] = *(const vec*)((const T*)a.k_norm + c); k_norm[1] = *(const vec*)((const T*)a.k_norm + half + c); }
  if (tok < a.total && slot < n_rows) request(slot);
  {
    static_assert(THREADS % half == 0, "a thread's angles share their frequency");
    const int i = tid % half;
    const double inv_freq = rotary_frequency(i, 2 * half, a.log2_theta);
    const unsigned axis = (uint64_t)pick(i < 32, (void*)a.axis[0], (void*)a.axis[1]) >> (2 * (i & 31)) & 3;
#pragma unroll
    for (int k0 = 0; k0 < TT; k0 += THREADS / half) {
      const int k = k0 + tid / half;
      if (k < TT) {                                // tokens past the last: angles nobody reads
        int64_t pos = a.pos0 + (tok0 + k) % a.n_tokens;
        if (a.positions && tok0 + k < a.total)
          pos = a.positions[(int64_t)(tok0 + k) * a.n_axes + axis];
        rotary_angle(pos, inv_freq, &cs_all[k][i], &sn_all[k][i]);
      }
    }
  }
  __syncthreads();

  if (tok >= a.total) return;
  float cs[N], sn[N];
#pragma unroll
  for (int e = 0; e < N; ++e) { cs[e] = cs_all[k][c + e]; sn[e] = sn_all[k][c + e]; }
  for (int h = slot; h < n_rows; h += n_slots) {
    if (h != slot) request(h);
    if (h < a.H + a.Hkv) {
      float x[N], y[N], xr[N], yr[N];
#pragma unroll
      for (int e = 0; e < N; ++e) { x[e] = (float)lo[e]; y[e] = (float)hi[e]; }
      if (h < a.H ? a.q_norm != nullptr : a.k_norm != nullptr) {
        const vec wlo = h < a.H ? q_norm[0] : k_norm[0], whi = h < a.H ? q_norm[1] : k_norm[1];
        const auto mean_square = [&](float eps) INLINE {
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < N; ++e) sum = fmaf(x[e], x[e], fmaf(y[e], y[e], sum));
#pragma unroll
          for (int l = 1; l < cpr; l <<= 1) sum += __shfl_xor(sum, l);
          return sum * (1.f / d) + eps;
        };
        float ms = mean_square(a.eps);
        if (__builtin_expect(!(ms >= 0x1p-100f && ms < INFINITY), 0)) {
          // (elements whose squares 32 bits do not hold: of 2^60 in size or, with an eps as small, of 2^-50)
          const float f = ms < 1.f ? 0x1p100f : 0x1p-70f;
#pragma unroll
          for (int e = 0; e < N; ++e) { x[e] *= f; y[e] *= f; }
          ms = mean_square(a.eps * f * f);
        }
        const float r = 1.f / sqrtf(ms);
#pragma unroll
        for (int e = 0; e < N; ++e) { x[e] = x[e] * r * (float)wlo[e]; y[e] = y[e] * r * (float)whi[e]; }
      }
#pragma unroll
      for (int e = 0; e < N; ++e) { xr[e] = rotary_lo(x[e], y[e], cs[e], sn[e]); yr[e] = rotary_hi(x[e], y[e], cs[e], sn[e]); }
      lo = Chunk<T>::pack(xr);
      hi = Chunk<T>::pack(yr);
    }
    if constexpr (Q4) {
      if (h >= a.H) {
        const bool v = h >= a.H + a.Hkv;
        const size_t row = ((size_t)beta * a.Hkv + h - a.H - (v ? a.Hkv : 0)) * a.cap + a.dst_row + t;
        q4_file<N, d>(v ? a.q4.v_codes : a.q4.k_codes, v ? a.q4.v_scales : a.q4.k_scales, row, c, lo);
        q4_file<N, d>(v ? a.q4.v_codes : a.q4.k_codes, v ? a.q4.v_scales : a.q4.k_scales, row, c + half, hi);
        continue;
      }
    }
    *(vec*)dst = lo;
    *(vec*)(dst + half) = hi;
  }
}

template <typename T, int half, int TT, bool Q4>
hipError_t launch_tokens(NormArgs<Q4> a, hipStream_t st) {
  return launch_in_pieces(((int64_t)a.total + TT - 1) / TT, THREADS, [&](unsigned first, unsigned n_wgs) {
    a.first = first * TT;
    norm_rope_kernel<T, half, TT, Q4><<<dim3(n_wgs), THREADS, 0, st>>>(a);
    a.clear = nullptr;
  });
}

// Tokens per workgroup.  One where a token's rows keep most of 256 threads busy, or where there are too few tokens to fill the GPU otherwise; sixteen where
// the angles outweigh the rows; else four.  us with 1 / 4 / 16 tokens, bf16: 40 rows, 32768 tokens 115 / 121 / 142; 24 rows, 30000 71 / 66 / 78; 16 rows,
// 8000 13.4 / 11.8 / 13.8; 10 rows, 20000 26 / 18.4 / 19.8; 5 rows, 4500 7.2 / 5.3 / 6.7 and 80000 73 / 43 / 35; 2 rows, 100000 89 / 38 / 28.  fp32: 10 rows
// of 128, 20000 29.9 / 31.4 / 38.7; 20 rows of 64 30.4 / 31.3 / 36.6; 5 rows of 128 22.2 / 16.6 / 18.0; 2 rows of 128 18.5 / 11.1 / 10.2, 5000 6.7 / 4.7 / 5.3.
template <typename T, int half, bool Q4>
hipError_t launch_rows(const NormArgs<Q4>& a, hipStream_t st) {
  const int64_t busy = ((int64_t)a.H + (a.V ? 2 : 1) * a.Hkv) * (half / Chunk<T>::N);       // threads that one token's rows would fill
  if (busy >= (sizeof(T) == 2 ? 256 : 160) || a.total < 1024) return launch_tokens<T, half, 1, Q4>(a, st);
  if (busy > 40 || a.total < 8192) return launch_tokens<T, half, 4, Q4>(a, st);
  return launch_tokens<T, half, 16, Q4>(a, st);
}
template <bool Q4>
hipError_t launch(int dtype, int d, const NormArgs<Q4>& a, hipStream_t st) {
  if (dtype != 0) return launch_rows<__bf16, 64, Q4>(a, st);
  return d == 64 ? launch_rows<float, 32, Q4>(a, st) : launch_rows<float, 64, Q4>(a, st);
}

}  // namespace

hipError_t launch_qk(int dtype, const Geom& g, const QkArgs& q, hipStream_t st) {
  const int64_t total = (int64_t)g.B * q.n_tokens;
  if (total == 0) return hipSuccess;
  if (total > 0x7fffffff) return hipErrorInvalidValue;
  const auto fill = [&](auto& a) {
    a.Q = q.Q; a.Yq = q.Yq; a.K = q.K; a.V = q.V; a.Yk = q.Yk; a.Vc = q.Vc;
    a.H = q.Q ? g.Hq : 0; a.Hkv = q.K ? g.Hkv : 0;
    a.n_tokens = (uint32_t)q.n_tokens; a.total = (uint32_t)total; a.first = 0;
    a.cap = g.cap; a.dst_row = q.dst_row; a.pos0 = q.pos0; a.log2_theta = log2(q.theta);
    a.positions = q.positions; a.q_norm = q.q_norm; a.k_norm = q.k_norm; a.eps = q.eps; a.n_axes = (int16_t)q.n_axes;
    a.axis[0] = q.axis[0]; a.axis[1] = q.axis[1]; a.cached = (int16_t)q.cached;
    a.clear = q.clear;
  };
  if (q.q4.k_codes) {
    NormArgs<true> a;
    fill(a);
    a.q4 = q.q4;
    return launch(dtype, g.d, a, st);
  }
  NormArgs<false> a;
  fill(a);
  return launch(dtype, g.d, a, st);
}

}  // namespace star
