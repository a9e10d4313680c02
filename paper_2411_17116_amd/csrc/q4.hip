// A cache held in four bits: rows filed into it and read from it, and phase 2 over it (Eq. 1-2 per split of the cache; the
// merge kernels fold the splits, Eq. 3-4).  q4.h says what a row is.
#include "q4.h"

namespace star {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;

#define LDS_AS __attribute__((address_space(3)))

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// ------------------------------------------------------------------ rows filed and read
// Bound by HBM: a lane has eight elements of K and then of V, four lanes a group.
struct CopyArgs {
  Q4Copy c;
  int64_t cap;
  Div Hkv, rows;          // rows: of a (batch, head)
  uint32_t total;         // (batch, head, row)
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 v = *(const bf16x8*)p;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  } else {
    const f32x4 v = *(const f32x4*)p, w = *(const f32x4*)(p + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = v[e]; x[4 + e] = w[e]; }
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (__bf16)x[e];
    *(bf16x8*)p = v;
  } else {
    *(f32x4*)p = f32x4{x[0], x[1], x[2], x[3]};
    *(f32x4*)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
  }
}
// Eight codes times their unit (255: NaN).
__device__ __forceinline__ void values8(uint32_t c, uint32_t e, float (&x)[8]) {
  const float u = q4_unit_value(e);
#define PAIR(k) { const q4_f32x2 y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, u, k); x[2 * k] = y[0]; x[2 * k + 1] = y[1]; }
  PAIR(0) PAIR(1) PAIR(2) PAIR(3)
#undef PAIR
  if (e == 255u)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(0x7fc00000u);
}

template <typename T, int d, bool LOAD>
__global__ __launch_bounds__(256) void q4_rows_kernel(CopyArgs a, unsigned first_wg) {
  constexpr int LANES = d / 8;                  // of a row
  const uint32_t r = (first_wg + blockIdx.x) * (256 / LANES) + threadIdx.x / LANES;
  if (r >= a.total) return;
  const int c = (threadIdx.x % LANES) * 8;
  const uint32_t pair = quotient(r, a.rows), n = r - pair * a.rows.d, beta = quotient(pair, a.Hkv), h = pair - beta * a.Hkv.d;
  const size_t plain = beta * a.c.batch + h * a.c.head + n * a.c.row_stride + c;
  const size_t row = (size_t)pair * a.cap + a.c.row + n;
  unsigned char* codes[2] = {(unsigned char*)a.c.q4.k_codes, (unsigned char*)a.c.q4.v_codes};
  unsigned char* scales[2] = {(unsigned char*)a.c.q4.k_scales, (unsigned char*)a.c.q4.v_scales};
  T* from[2] = {(T*)a.c.K, (T*)a.c.V};
  if constexpr (LOAD) {
    uint32_t code[2], e[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      code[i] = *(const uint32_t*)(codes[i] + row * (d / 2) + c / 2);
      e[i] = scales[i][row * (d / 32) + c / 32];
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      float x[8];
      values8(code[i], e[i], x);
      store8(from[i] + plain, x);
    }
  } else {
    float x[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) load8(from[i] + plain, x[i]);
#pragma unroll
    for (int i = 0; i < 2; ++i) q4_file<8, d>(codes[i], scales[i], row, c, x[i]);
  }
}

template <typename T, int d, bool LOAD>
hipError_t launch_rows(const CopyArgs& a, hipStream_t st) {
  constexpr int PER = 256 / (d / 8);
  return launch_in_pieces(((int64_t)a.total + PER - 1) / PER, 256, [&](unsigned first, unsigned n_wgs) {
    q4_rows_kernel<T, d, LOAD><<<dim3(n_wgs), 256, 0, st>>>(a, first);
  });
}
template <bool LOAD>
hipError_t launch_rows(int dtype, const Geom& g, const Q4Copy& c, hipStream_t st) {
  const int64_t total = (int64_t)g.B * g.Hkv * c.n;
  if (total > 0x7fffffff) return hipErrorInvalidValue;
  const CopyArgs a = {c, g.cap, make_div(g.Hkv), make_div((uint32_t)c.n), (uint32_t)total};
  if (dtype != 0) return launch_rows<__bf16, 128, LOAD>(a, st);
  return g.d == 64 ? launch_rows<float, 64, LOAD>(a, st) : launch_rows<float, 128, LOAD>(a, st);
}

// ------------------------------------------------------------------ attention
// chunk c (16 bytes) of key row r of V sits in slot c ^ swz(r): what rows of 16 chunks (8) are spread by
template <int D>
__device__ __forceinline__ int swz(int r) { return D == 128 ? ((r << 1) & 15) | ((r >> 3) & 1) : r & 7; }

__device__ __forceinline__ float xor16(float x) { return __int_as_float(__builtin_amdgcn_ds_swizzle(__float_as_int(x), 0x401F)); }
__device__ __forceinline__ float xor32_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xor32_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What a lane holds of 16 keys of K or of V: D / 4 elements of key lane % 16, from D / 4 * (lane / 16) on, and their unit.
template <int D>
struct Rows16 {
  uint32_t c[D / 32];
  uint32_t e;
};
template <int D>
__device__ __forceinline__ Rows16<D> load_rows(const unsigned char* codes, const unsigned char* scales, size_t row, int j4) {
  Rows16<D> x;
  const unsigned char* p = codes + row * (D / 2) + j4 * (D / 8);
#pragma unroll
  for (int i = 0; i < D / 32; ++i) x.c[i] = ((const uint32_t*)p)[i];
  x.e = scales[row * (D / 32) + (D == 128 ? j4 : j4 >> 1)];
  return x;
}
__device__ __forceinline__ bf16x8 values(uint32_t c, float unit) {
  const q4_bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 1);
  const q4_bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 2), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 3);
  return bf16x8{a[0], a[1], b[0], b[1], x[0], x[1], y[0], y[1]};
}

// x = p[0] + p[1] + .. in bf16 parts.  Three hold 24 bits and are cut off, so that none overflows; an infinity or NaN is the
// first's alone.
template <int P>
__device__ __forceinline__ void split(float x, __bf16 (&p)[P]) {
  if constexpr (P == 3) {
    const bool finite = magnitude_bits(x) < 0x7f800000u;
    float r = x;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const float y = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
      p[i] = i == 0 && !finite ? (__bf16)x : (__bf16)y;
      r = finite ? r - y : 0.f;
    }
  } else {
    p[0] = (__bf16)x;
    if constexpr (P == 2) p[1] = (__bf16)(x - (float)p[0]);
  }
}

constexpr int WAVES = 4;
constexpr int UNIT = 32;              // keys a wavefront takes at once

struct TileDiv {
  Div Hkv, tiles, splits, G;
};

// A workgroup of four wavefronts has 16 rows (token x head of a KV group) and a split of the cache, whose units of 32 keys they take
// in turn; their results meet in LDS.  S^T = K Q^T in bf16 products, which are exact: a four-bit value is a bf16 number, fp32 queries are
// three of them.  The exponentiated tile is the B operand of O^T += V^T P^T, weights in PP bf16 parts; V goes through LDS to
// be read back transposed.
template <typename T, int D, int PP>
__global__ __launch_bounds__(64 * WAVES) void q4_attend_kernel(Q4Args a, TileDiv by, unsigned first_wg) {
  constexpr int QP = sizeof(T) == 2 ? 1 : 3, NT = D / 32, DT = D / 16, ROWB = 2 * D;
  __shared__ __attribute__((aligned(1024))) char lds_v[WAVES][UNIT * ROWB];
  __shared__ float lds_m[WAVES][16], lds_l[WAVES][16];
  const Geom& g = a.g;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, qc = lane & 15, j4 = lane >> 4;
  uint32_t w = first_wg + blockIdx.x;
  uint32_t x = quotient(w, by.Hkv);
  const uint32_t kvh = w - x * by.Hkv.d;
  w = quotient(x, by.tiles);
  const uint32_t tile = x - w * by.tiles.d;
  x = quotient(w, by.splits);
  const uint32_t sp = w - x * by.splits.d, beta = x;

  const int row = tile * 16 + qc, R = g.G * a.q_len;
  const bool live = row < R;
  const int j = live ? (int)quotient(row, by.G) : 0, head = kvh * g.G + (live ? row - j * g.G : 0);
  const int total = (int)(a.cache_len + (a.causal ? a.q_len : 0));
  int64_t lo64, hi64;
  split_range(a.plan, g.L, g.b, total, sp, &lo64, &hi64);
  const int lo = (int)lo64, hi = (int)hi64;
  const int lim0 = a.causal ? (int)a.cache_len + j + 1 : (int)a.cache_len, lim = lim0 < hi ? lim0 : hi;

  bf16x8 q[QP][NT];
  {
    const T* p = (const T*)a.Qq + (((size_t)beta * a.q_len + j) * g.Hq + head) * D + j4 * (D / 4);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float y[8];
      load8(p + 8 * t, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        __bf16 part[QP];
        split<QP>(live ? y[e] : 0.f, part);
#pragma unroll
        for (int i = 0; i < QP; ++i) q[i][t][e] = part[i];
      }
    }
  }
  f32x4 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  const float c = g.scale * LOG2E;

  const size_t base = ((size_t)beta * g.Hkv + kvh) * (size_t)g.cap;
  const unsigned char *kc = (const unsigned char*)a.q4.k_codes, *ks = (const unsigned char*)a.q4.k_scales;
  const unsigned char *vc = (const unsigned char*)a.q4.v_codes, *vs = (const unsigned char*)a.q4.v_scales;
  char* vl = lds_v[wave];
  const unsigned lds0 = (unsigned)(size_t)(LDS_AS char*)vl;

  for (int key0 = lo + UNIT * wave; key0 < hi; key0 += UNIT * WAVES) {
    // keys past the last are that one again, masked below
    Rows16<D> k[2], v[2];
    f32x4 s[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const int key = key0 + 16 * kt + qc;
      const size_t r = base + (key < hi ? key : hi - 1);
      k[kt] = load_rows<D>(kc, ks, r, j4);
      v[kt] = load_rows<D>(vc, vs, r, j4);
    }
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const float unit = q4_unit_value(k[kt].e);
      s[kt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const bf16x8 y = values(k[kt].c[t], unit);
#pragma unroll
        for (int i = QP - 1; i >= 0; --i) s[kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, q[i][t], s[kt], 0, 0, 0);
      }
    }
    // A value that is NaN counts where its key is seen and nowhere else, and its weight may be zero where it is not: it goes
    // to the outputs of the rows that see it, and zeros to the products.
    uint64_t bad[2];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      bad[kt] = __builtin_amdgcn_ballot_w64(v[kt].e == 255u);
      if (v[kt].e == 255u) {
        v[kt].e = 127;
#pragma unroll
        for (int t = 0; t < NT; ++t) v[kt].c[t] = 0;
      }
      const float unit = q4_unit_value(v[kt].e);
      const int r = 16 * kt + qc;
#pragma unroll
      for (int t = 0; t < NT; ++t) *(bf16x8*)(vl + r * ROWB + (((j4 * NT + t) ^ swz<D>(r)) << 4)) = values(v[kt].c[t], unit);
    }
    const int n = lim - key0 - 4 * j4;              // element (kt, e) is key key0 + 16 kt + 4 j4 + e
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[kt][e] = 16 * kt + e < n ? s[kt][e] : -INFINITY;
    const float tmax = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    const float mn = fmaxf(m, xor32_max(fmaxf(tmax, xor16(tmax)))), mm = mn == -INFINITY ? 0.f : mn;
    const float alpha = __builtin_amdgcn_exp2f((m - mm) * c), neg = mm * -c;
    m = mn;
    l *= alpha;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
    bf16x8 p[PP];
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][e], c, neg));
        l += y;
        __bf16 part[PP];
        split<PP>(y, part);
#pragma unroll
        for (int i = 0; i < PP; ++i) p[i][4 * kt + e] = part[i];
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int rr = 4 * j4 + (qc >> 2);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const unsigned at = lds0 + rr * ROWB + (((2 * dt + ((lane & 3) >> 1)) ^ swz<D>(rr)) << 4) + 8 * (lane & 1);
      const s16x4 y0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(size_t)at);
      const unsigned at1 = lds0 + (rr + 16) * ROWB + (((2 * dt + ((lane & 3) >> 1)) ^ swz<D>(rr + 16)) << 4) + 8 * (lane & 1);
      const s16x4 y1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(size_t)at1);
      const bf16x8 y = __builtin_shufflevector(__builtin_bit_cast(bf16x4, y0), __builtin_bit_cast(bf16x4, y1), 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
      for (int i = PP - 1; i >= 0; --i) o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, p[i], o[dt], 0, 0, 0);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int kt = 0; kt < 2; ++kt)
      for (uint64_t b = bad[kt]; b; b &= b - 1) {
        const int at = __builtin_ctzll(b), key = key0 + 16 * kt + (at & 15);
        if (key >= lim) continue;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)                  // lane at / 16 had columns D / 4 (at / 16) ..
          if (dt / (DT / 4) == at >> 4) o[dt] = f32x4{NAN, NAN, NAN, NAN};
      }
  }

  // the wavefronts meet, in a fixed order
  l = xor32_sum(l + xor16(l));
  if (j4 == 0) { lds_m[wave][qc] = m; lds_l[wave][qc] = l; }
  __syncthreads();
  float mt = -INFINITY, lt = 0.f;
#pragma unroll
  for (int k = 0; k < WAVES; ++k) mt = fmaxf(mt, lds_m[k][qc]);
  const float mm = mt == -INFINITY ? 0.f : mt;
#pragma unroll
  for (int k = 0; k < WAVES; ++k) lt += lds_l[k][qc] * __builtin_amdgcn_exp2f((lds_m[k][qc] - mm) * c);
  const float scale = lt == 0.f ? 0.f : __builtin_amdgcn_exp2f((m - mm) * c) * (1.f / lt);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] *= scale;
  const size_t out0 = ((size_t)beta * a.plan.s_total + sp) * g.Hq * a.q_len;
  if (threadIdx.x < 16 && live) a.LSE_sub[out0 + (size_t)head * a.q_len + j] = lt == 0.f ? -INFINITY : (mm * c + __builtin_amdgcn_logf(lt)) * LN2;
  float* meet = (float*)lds_v[0];                     // [wave][16][D]: what V took, 16 rows of D floats a wavefront
  static_assert(sizeof(lds_v[0]) == 16 * D * sizeof(float), "");
  float* mine = meet + wave * 16 * D + qc * D;
  __syncthreads();
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) *(f32x4*)(mine + (((4 * dt + j4) ^ qc) & (D / 4 - 1)) * 4) = o[dt];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * (D / 4); i += 64 * WAVES) {
    const int r = i / (D / 4), chunk = i % (D / 4), rw = tile * 16 + r;
    if (rw >= R) break;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < WAVES; ++k) acc += *(const f32x4*)(meet + k * 16 * D + r * D + ((chunk ^ r) & (D / 4 - 1)) * 4);
    const int tj = (int)quotient(rw, by.G);
    *(f32x4*)(a.O_sub + (out0 + (size_t)(kvh * g.G + rw - tj * g.G) * a.q_len + tj) * D + 4 * chunk) = acc;
  }
}

template <typename T, int D, int PP>
hipError_t launch_attend(const Q4Args& a, hipStream_t st) {
  const Geom& g = a.g;
  const uint32_t tiles = (uint32_t)(((int64_t)g.G * a.q_len + 15) / 16);
  const TileDiv by = {make_div(g.Hkv), make_div(tiles), make_div(a.plan.s_total), make_div(g.G)};
  const int64_t wgs = (int64_t)g.B * g.Hkv * tiles * a.plan.s_total;
  if (wgs > 0x7fffffff) return hipErrorInvalidValue;
  return launch_in_pieces(wgs, 64 * WAVES, [&](unsigned first, unsigned n) {
    q4_attend_kernel<T, D, PP><<<dim3(n), 64 * WAVES, 0, st>>>(a, by, first);
  });
}

}  // namespace

hipError_t launch_q4_store(int dtype, const Geom& g, const Q4Copy& c, hipStream_t st) { return launch_rows<false>(dtype, g, c, st); }
hipError_t launch_q4_load(int dtype, const Geom& g, const Q4Copy& c, hipStream_t st) { return launch_rows<true>(dtype, g, c, st); }

hipError_t launch_phase2_q4(int dtype, const Q4Args& a, hipStream_t st) {
  if (dtype != 0) return a.parts == 2 ? launch_attend<__bf16, 128, 2>(a, st) : launch_attend<__bf16, 128, 1>(a, st);
  return a.g.d == 64 ? launch_attend<float, 64, 3>(a, st) : launch_attend<float, 128, 3>(a, st);
}

}  // namespace star
