// A cache held in four bits: rows filed into it and read from it, and phase 2 over it (Eq. 1-2 per split of the cache; the
// merge kernels fold the splits, Eq. 3-4).  q4.h says what a row is.
#include "q4_attend.h"

#include <type_traits>

namespace star {

namespace {

// ------------------------------------------------------------------ rows filed and read
// Bound by HBM: a lane has eight elements of K and of V, four lanes a group.  32768 rows of eight heads in bf16, 170 MB: filed in 29 to 33 us (5.2 to 5.9 TB/s), read in
// 25 (6.7); a copy reaches 4.9 TB/s, a pure read 7.15.
struct CopyArgs {
  Q4Copy c;
  int64_t cap;
  Div Hkv, rows;          // rows: of a (batch, head)
  uint32_t total;         // (batch, head, row)
};

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

// ------------------------------------------------------------------ attention, few rows
// A call of up to 32 rows (token x head of a KV group) reads every code once and does 16 to 128 flops per byte: a stream, bound by HBM.
//   * A workgroup is four wavefronts that share a split and meet in LDS behind the key loop; without per-part outputs the wavefronts of a
//     KV head take the comb of 32-key units w, w + N, w + 2N, .., so that together they read one contiguous window of its cache.
//   * A lane has D / 4 elements of a key (with 128 of them a group: 16 bytes of codes and a byte of exponent), straight from the cache in the layout that the MFMA wants of
//     K; two units are in registers, and a unit's are requested again as soon as its K is multiplied and its V in LDS.
//   * S^T = K Q^T in bf16 products, which lose nothing: a four-bit value is a bf16 number, an fp32 query three of them.  (The instruction that
//     multiplies four-bit codes as they are, by queries in two 8-bit parts, adds up a group's products in fewer bits: 2^-11 of sum |q k| off with
//     queries of different sizes.)  The exponentiated unit is the B operand of O^T += V^T P^T, weights in PP parts (q4_attend.h), V by way of LDS to be read back transposed.
//   * The call's own keys are put into four bits by the wavefront whose unit has them, which files them and attends to them from its registers.
// One token, 32 / 8 heads: 131072 keys (143 MB) 24 to 25 us, 5.8 TB/s; 1048576 (1.14 GB) 169 to 178 us, 6.4 to 6.7 TB/s; 2000 keys 5.6 us, the chain of one unit per
// wavefront.  Two workgroups on a CU: with three or four wavefronts on a SIMD 131072 keys take 28 to 58 us instead of 25 (registers spill, or each waits longer).

constexpr int WAVES = 4;
constexpr int UNIT = 32;              // keys a wavefront takes at once

typedef const __attribute__((address_space(1))) unsigned char* GlobalBytes;

// What a lane holds of 16 keys of K or of V: D / 4 elements of key lane % 16, from D / 4 * (lane / 16) on, and their unit.
template <int D>
struct Rows16 {
  uint32_t c[D / 32];
  uint32_t e;
};
template <int D>
struct UnitRegs {
  Rows16<D> k[2], v[2];
};
template <typename V, bool NT>
__device__ __forceinline__ V fetch(GlobalBytes p) {
  const __attribute__((address_space(1))) V* q = (const __attribute__((address_space(1))) V*)p;
  return NT ? __builtin_nontemporal_load(q) : *q;
}
// (codes and exponents of the lane's key; codes' rows are D / 2 bytes, exponents' D / 32)
template <int D, bool NT>
__device__ __forceinline__ void load_rows(Rows16<D>& x, GlobalBytes codes, GlobalBytes scales) {
  if constexpr (D == 128) {
    const i32x4 c = fetch<i32x4, NT>(codes);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.c[i] = (uint32_t)c[i];
  } else {
    const i32x2 c = fetch<i32x2, NT>(codes);
    x.c[0] = (uint32_t)c[0];
    x.c[1] = (uint32_t)c[1];
  }
  x.e = fetch<unsigned char, NT>(scales);
}
template <int QP, int NT, int DT, int RB>
struct StreamState {
  bf16x8 q[RB][QP][NT];   // Q^T fragments: D / 4 (lane / 16) + 8 t ..+7 of row lane % 16
  f32x4 o[RB][DT];        // O^T: element 16 dt + 4 (lane / 16) + v of that row
  float m[RB], l[RB], neg[RB], above[RB];      // reference (a logit whose weight is 2^(TOP - 3)), this lane's share of the sum, TOP - 3 - m c (0 while nothing was
                          // visible), and the exponent that moves the reference
};

struct StreamDiv {
  Div Hkv, splits, G, steps;      // steps between two of a wavefront's (flat plans): splits times wavefronts
};
// What a launch is handed: packed under a flat plan (but for a pair that is stored as it is), else as it is.
struct StreamCall {
  Q4Args a;
  StreamDiv by;
  unsigned first_wg;
};
struct FlatStream {
  const void *Qq, *Kn, *Vn;
  Q4Rows q4;
  void* out;                    // O, or O_sub with LSE_sub behind it
  int32_t cache_len, cap;
  uint32_t heads, rows;         // G << 16 | Hkv, q_len << 16 | splits
  float scale;
  int32_t batch_kind;           // B << 2 | whether `out` is O << 1 | causal
  uint32_t m[4];                // the divisors'
  uint32_t first_wg;
};
static_assert(sizeof(FlatStream) <= 112, "");
template <int D>
__device__ __forceinline__ StreamCall unpacked(const StreamCall& c) { return c; }
template <int D>
__device__ __forceinline__ StreamCall unpacked(const FlatStream& c) {
  StreamCall x;
  Geom& g = x.a.g;
  g.B = c.batch_kind >> 2; g.G = c.heads >> 16; g.Hkv = c.heads & 0xffff; g.Hq = g.G * g.Hkv; g.d = D;
  g.L = g.b = g.a = 0; g.cap = c.cap; g.scale = c.scale;
  const int splits = c.rows & 0xffff;
  x.a.plan = SplitPlan{0, 0, 0, 0, splits, 1, 1, 0, 0};
  x.a.cache_len = c.cache_len; x.a.q_len = c.rows >> 16; x.a.causal = c.batch_kind & 1;
  x.a.Qq = c.Qq; x.a.Kn = c.Kn; x.a.Vn = c.Vn; x.a.q4 = c.q4;
  x.a.O = c.batch_kind & 2 ? c.out : nullptr;
  x.a.O_sub = (float*)c.out;
  x.a.LSE_sub = (float*)c.out + (size_t)g.B * splits * g.Hq * x.a.q_len * D;
  x.by = StreamDiv{div_of(g.Hkv, c.m[0]), div_of(splits, c.m[1]), div_of(g.G, c.m[2]), div_of(splits * WAVES, c.m[3])};
  x.first_wg = c.first_wg;
  return x;
}

template <typename T, int D, int PP, int RB, bool NT, typename C>
__global__ __launch_bounds__(64 * WAVES, 2) void q4_stream_kernel(C call) {
  const StreamCall from = unpacked<D>(call);
  const Q4Args& a = from.a;
  const StreamDiv& by = from.by;
  constexpr int QP = sizeof(T) == 2 ? 1 : 3, NS = D / 32, DT = D / 16, ROWB = 2 * D;
  __shared__ __attribute__((aligned(1024))) char lds_v[WAVES][UNIT * ROWB];      // 16 rows of D floats of a wavefront, too
  __shared__ float lds_m[WAVES][16 * RB], lds_l[WAVES][16 * RB];
  __shared__ int lds_wide[WAVES];
  const Geom& g = a.g;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, qc = lane & 15, j4 = lane >> 4;
  const uint32_t w = from.first_wg + blockIdx.x, x = quotient(w, by.Hkv), kvh = w - x * by.Hkv.d;
  const uint32_t beta = quotient(x, by.splits), sp = x - beta * by.splits.d;

  const int R = g.G * a.q_len;
  int j[RB], head[RB];
  bool live[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int row = 16 * b + qc;
    live[b] = row < R;
    j[b] = live[b] ? (int)quotient(row, by.G) : 0;
    head[b] = kvh * g.G + (live[b] ? row - j[b] * g.G : 0);
  }
  const int cache_len = (int)a.cache_len, total = cache_len + (a.causal ? a.q_len : 0);
  const int cached = a.Kn ? cache_len : total;
  // unit `s` of this wavefront is keys [base + s stride, + 32) below hi; the first n_whole are cached and seen by every row as a whole
  const int free_hi = a.causal && cache_len + 1 < cached ? cache_len + 1 : cached;
  int base, stride, n_units, n_whole, hi;
  if (std::is_same<C, FlatStream>::value || a.plan.flat) {
    const int all = a.plan.s_total * WAVES, first = sp * WAVES + wave, T_ = (total + UNIT - 1) / UNIT, whole = free_hi / UNIT;
    base = first * UNIT;
    stride = all * UNIT;
    n_units = first < T_ ? (int)quotient(T_ - first + all - 1, by.steps) : 0;
    n_whole = first < whole ? (int)quotient(whole - first + all - 1, by.steps) : 0;
    hi = total;
  } else {
    int64_t lo64, hi64;
    split_range(a.plan, g.L, g.b, total, sp, &lo64, &hi64);
    hi = (int)hi64;
    base = (int)lo64 + UNIT * wave;
    stride = UNIT * WAVES;
    n_units = hi > base ? (hi - base + stride - 1) / stride : 0;
    const int room = (free_hi < hi ? free_hi : hi) - UNIT - base;
    n_whole = room >= 0 ? room / stride + 1 : 0;
  }

  const size_t pair = (size_t)beta * g.Hkv + kvh, rows0 = pair * (size_t)g.cap;
  GlobalBytes kc = (GlobalBytes)a.q4.k_codes + rows0 * (D / 2), ks = (GlobalBytes)a.q4.k_scales + rows0 * (D / 32);
  GlobalBytes vc = (GlobalBytes)a.q4.v_codes + rows0 * (D / 2), vs = (GlobalBytes)a.q4.v_scales + rows0 * (D / 32);
  const int group = D == 128 ? j4 : j4 >> 1;
  const unsigned c_off = qc * (D / 2) + j4 * (D / 8), s_off = qc * (D / 32) + group;
  const auto load_whole = [&](UnitRegs<D>& u, int s) INLINE {
    const int key0 = base + s * stride;
    GlobalBytes a0 = kc + (size_t)key0 * (D / 2), a1 = ks + (size_t)key0 * (D / 32), a2 = vc + (size_t)key0 * (D / 2), a3 = vs + (size_t)key0 * (D / 32);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) load_rows<D, NT>(u.k[kt], a0 + kt * 16 * (D / 2) + c_off, a1 + kt * 16 * (D / 32) + s_off);
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) load_rows<D, NT>(u.v[kt], a2 + kt * 16 * (D / 2) + c_off, a3 + kt * 16 * (D / 32) + s_off);
  };

  StreamState<QP, NS, DT, RB> st;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const T* p = (const T*)a.Qq + (((size_t)beta * a.q_len + j[b]) * g.Hq + head[b]) * D + j4 * (D / 4);
#pragma unroll
    for (int t = 0; t < NS; ++t) {
      float y[8];
      load8(p + 8 * t, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        __bf16 part[QP];
        split(live[b] ? y[e] : 0.f, part);
#pragma unroll
        for (int i = 0; i < QP; ++i) st.q[b][i][t][e] = part[i];
      }
    }
  }
  const float c = g.scale * LOG2E;
  char* vl = lds_v[wave];
  const unsigned lds0 = (unsigned)(size_t)(LDS_AS char*)vl;
  unsigned vw[NS];                      // (row qc of the first 16; the others' are 16 rows further)
#pragma unroll
  for (int t = 0; t < NS; ++t) vw[t] = lds0 + qc * ROWB + (((j4 * NS + t) ^ swz<D>(qc)) << 4);
  const int rr = 4 * j4 + (qc >> 2);
  unsigned vr[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) vr[dt] = lds0 + rr * ROWB + (((2 * dt + ((lane & 3) >> 1)) ^ swz<D>(rr)) << 4) + 8 * (lane & 1);

  Wide wide = {0, 0};
  int down = 0;
  const auto walk = [&](auto WIDE) INLINE {
    typedef Product<WIDE.value> P;
    typedef typename P::Vec Vec;
    constexpr int PARTS = WIDE.value && PP > 1 ? 3 : PP;
    UnitRegs<D> u0, u1;
    if (0 < n_whole) load_whole(u0, 0);
    if (1 < n_whole) load_whole(u1, 1);
#pragma unroll
    for (int b = 0; b < RB; ++b) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) st.o[b][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
      st.m[b] = st.above[b] = -INFINITY;
      st.l[b] = st.neg[b] = 0.f;
    }
    // A unit's scores, and V into LDS: its registers are then free.
    f32x4 s[RB][2];
    const auto score = [&](const UnitRegs<D>& u) INLINE {
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const float unit = q4_unit_value(u.k[kt].e);
#pragma unroll
        for (int t = 0; t < NS; ++t) {
          const bf16x8 y = values(u.k[kt].c[t], unit);
#pragma unroll
          for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int i = QP - 1; i >= 0; --i) {
              const f32x4 acc = t == 0 && i == QP - 1 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[b][kt];
              s[b][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, st.q[b][i][t], acc, 0, 0, 0);
            }
        }
      }
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        const float unit = WIDE.value ? unit_down(u.v[kt].e, down) : q4_unit_value(u.v[kt].e);
        if (!WIDE.value) wide.note(u.v[kt].e);
#pragma unroll
        for (int t = 0; t < NS; ++t) *(LDS_AS Vec*)(size_t)(vw[t] + kt * 16 * ROWB) = P::values(u.v[kt].c[t], unit);
      }
    };
    // Then softmax and products.
    const auto attend = [&]() INLINE {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      Vec v[DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const s16x4 y0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(size_t)vr[dt]);
        const s16x4 y1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(size_t)(vr[dt] + 16 * ROWB));
        v[dt] = __builtin_bit_cast(Vec, __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7));
      }
      Vec p[RB][PARTS];
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        Exponents t = exponents(s[b], c, st.neg[b]);
        // lanes exchange their maxima, and references move, only where a weight would pass 2^(TOP + 1)
        // (with each new maximum: 32 rows on 131072 keys 37.6 us instead of 34.0)
        if (__builtin_amdgcn_ballot_w64(largest(t) > st.above[b]) != 0) {
          const float m = fmaxf(st.m[b], quad_max(largest(exponents(s[b], 1.f, 0.f)))), mm = m == -INFINITY ? 0.f : m;
          const float alpha = __builtin_amdgcn_exp2f((st.m[b] - mm) * c);
          st.l[b] *= alpha;
#pragma unroll
          for (int dt = 0; dt < DT; ++dt) st.o[b][dt] *= alpha;
          st.m[b] = m;
          st.neg[b] = __builtin_fmaf(mm, -c, TOP - 3);
          st.above[b] = m == -INFINITY ? -INFINITY : TOP + 1;
          t = exponents(s[b], c, st.neg[b]);
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          const float y = __builtin_amdgcn_exp2f(t.x[i]), z = __builtin_amdgcn_exp2f(t.x[i + 1]);
          sum += y;
          sum += z;
          P::template split<PARTS>(y, z, p[b], i);
        }
        st.l[b] += sum;
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
          for (int i = PARTS - 1; i >= 0; --i) st.o[b][dt] = P::multiply(v[dt], p[b][i], st.o[b][dt]);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    };
    int n = 0;
    for (; n + 1 < n_whole; n += 2) {
      score(u0);
      if (n + 2 < n_whole) load_whole(u0, n + 2);
      attend();
      score(u1);
      if (n + 3 < n_whole) load_whole(u1, n + 3);
      attend();
    }
    if (n < n_whole) {
      score(u0);
      attend();
    }
    // The units that end past `hi` or among the call's tokens, or that not every row sees.
    int lim[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const int end = a.causal ? cache_len + j[b] + 1 : total;
      lim[b] = !live[b] ? 0 : end < hi ? end : hi;
    }
    for (n = n_whole; n < n_units; ++n) {
      const int key0 = base + n * stride;
      UnitRegs<D> u;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        int key = key0 + 16 * kt + qc;
        const bool there = key < hi;                 // keys past the last are that one again, masked below
        key = there ? key : hi - 1;
        if (key < cached) {
          load_rows<D, false>(u.k[kt], kc + (size_t)key * (D / 2) + j4 * (D / 8), ks + (size_t)key * (D / 32) + group);
          load_rows<D, false>(u.v[kt], vc + (size_t)key * (D / 2) + j4 * (D / 8), vs + (size_t)key * (D / 32) + group);
        }
        if (__builtin_amdgcn_ballot_w64(key >= cached) != 0) {
          // (all lanes, so that the lanes of a group meet; those of cached keys keep what they have)
          const size_t from = (((size_t)beta * a.q_len + (key < cached ? 0 : key - cached)) * g.Hkv + kvh) * D + j4 * (D / 4);
          const T* src[2] = {(const T*)a.Kn + from, (const T*)a.Vn + from};
          Rows16<D>* to[2] = {&u.k[kt], &u.v[kt]};
          unsigned char* codes[2] = {(unsigned char*)a.q4.k_codes, (unsigned char*)a.q4.v_codes};
          unsigned char* scales[2] = {(unsigned char*)a.q4.k_scales, (unsigned char*)a.q4.v_scales};
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            float y[NS][8];
            uint32_t most = 0;
#pragma unroll
            for (int t = 0; t < NS; ++t) {
              load8(src[i] + 8 * t, y[t]);
#pragma unroll
              for (int e = 0; e < 8; ++e) most = magnitude_bits(y[t][e]) > most ? magnitude_bits(y[t][e]) : most;
            }
            if (D == 64) {
              const uint32_t other = (uint32_t)__shfl_xor((int)most, 16);
              most = other > most ? other : most;
            }
            Rows16<D> r;
            r.e = q4_unit(most);
#pragma unroll
            for (int t = 0; t < NS; ++t) r.c[t] = r.e == 255u ? 0u : q4_codes(y[t], q4_unit_value(r.e));
            if (key < cached) continue;
            *to[i] = r;
            if (there) {
              unsigned char* at = codes[i] + (rows0 + key) * (D / 2) + j4 * (D / 8);
              if constexpr (D == 128) *(i32x4*)at = i32x4{(int)r.c[0], (int)r.c[1], (int)r.c[2], (int)r.c[3]};
              else *(i32x2*)at = i32x2{(int)r.c[0], (int)r.c[1]};
              if (D == 128 || (j4 & 1) == 0) scales[i][(rows0 + key) * (D / 32) + group] = (unsigned char)r.e;
            }
          }
        }
      }
      // A value that is NaN counts where its key is seen and nowhere else, and its weight may be zero where it is not: it goes
      // to the outputs of the rows that see it, and zeros to the products.
      uint64_t bad[2];
#pragma unroll
      for (int kt = 0; kt < 2; ++kt) {
        bad[kt] = __builtin_amdgcn_ballot_w64(u.v[kt].e == 255u);
        if (u.v[kt].e == 255u) {
          u.v[kt].e = 127;
#pragma unroll
          for (int t = 0; t < NS; ++t) u.v[kt].c[t] = 0;
        }
      }
      score(u);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int room = lim[b] - key0 - 4 * j4;      // element (kt, e) is key key0 + 16 kt + 4 j4 + e
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[b][kt][e] = 16 * kt + e < room ? s[b][kt][e] : -INFINITY;
      }
      attend();
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
        for (uint64_t left = bad[kt]; left; left &= left - 1) {
          const int at = __builtin_ctzll(left), key = key0 + 16 * kt + (at & 15);
#pragma unroll
          for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)                  // lane at / 16 had columns D / 4 (at / 16) ..
              if (key < lim[b] && dt / (DT / 4) == at >> 4) st.o[b][dt] = f32x4{NAN, NAN, NAN, NAN};
        }
    }

  };
  // the wavefronts meet, in a fixed order
  const auto tell = [&]() INLINE {
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const float l = quad_sum(st.l[b]);
      if (j4 == 0) { lds_m[wave][16 * b + qc] = st.m[b]; lds_l[wave][16 * b + qc] = l; }
    }
  };
  walk(std::integral_constant<bool, false>());
  tell();
  if (lane == 0) lds_wide[wave] = wide.flags();
  __syncthreads();
  int any_wide = 0;
#pragma unroll
  for (int k = 0; k < WAVES; ++k) any_wide |= lds_wide[k];
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(any_wide) != 0, 0)) {
    down = any_wide & 2 ? DOWN : 0;
    walk(std::integral_constant<bool, true>());
    __syncthreads();
    tell();
    __syncthreads();
  }
  const float up = down ? __builtin_ldexpf(1.f, DOWN) : 1.f;
  const size_t out0 = ((size_t)beta * a.plan.s_total + sp) * g.Hq * a.q_len;
  float* meet = (float*)lds_v;                        // [wave][16][D]
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    float mt = -INFINITY, lt = 0.f;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) mt = fmaxf(mt, lds_m[k][16 * b + qc]);
    const float mm = mt == -INFINITY ? 0.f : mt;
#pragma unroll
    for (int k = 0; k < WAVES; ++k) lt += lds_l[k][16 * b + qc] * __builtin_amdgcn_exp2f((lds_m[k][16 * b + qc] - mm) * c);
    const float scale = lt == 0.f ? 0.f : __builtin_amdgcn_exp2f((st.m[b] - mm) * c) * (1.f / lt);
    if (threadIdx.x < 16 && live[b] && !a.O)
      a.LSE_sub[out0 + (size_t)head[b] * a.q_len + j[b]] = lt == 0.f ? -INFINITY : (mm * c - (TOP - 3) + __builtin_amdgcn_logf(lt)) * LN2;
    float* mine = meet + wave * 16 * D + qc * D;
    if (b > 0) __syncthreads();
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *(f32x4*)(mine + ((4 * dt + j4) ^ qc) * 4) = st.o[b][dt] * scale * up;
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * (D / 4); i += 64 * WAVES) {
      const int r = i / (D / 4), chunk = i % (D / 4), row = 16 * b + r;
      if (row >= R) break;
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < WAVES; ++k) acc += *(const f32x4*)(meet + k * 16 * D + r * D + (chunk ^ r) * 4);
      const int tj = (int)quotient(row, by.G);
      const int h = kvh * g.G + row - tj * g.G;
      if (a.O) store4((T*)a.O + (((size_t)beta * a.q_len + tj) * g.Hq + h) * D + 4 * chunk, acc);
      else *(f32x4*)(a.O_sub + (out0 + (size_t)h * a.q_len + tj) * D + 4 * chunk) = acc;
    }
  }
}

template <typename T, int D, int PP, int RB, bool NT>
hipError_t launch_stream(const Q4Args& a, hipStream_t st) {
  const Geom& g = a.g;
  const StreamDiv by = {make_div(g.Hkv), make_div(a.plan.s_total), make_div(g.G), make_div((uint32_t)a.plan.s_total * WAVES)};
  const int64_t wgs = (int64_t)g.B * g.Hkv * a.plan.s_total;
  if (wgs > 0x7fffffff) return hipErrorInvalidValue;
  // (a pair that is stored as it is need not have its two parts one behind the other)
  if (a.plan.flat && (a.O || a.LSE_sub == a.O_sub + (size_t)g.B * a.plan.s_total * g.Hq * a.q_len * D)) {
    if (a.plan.s_total > 0xffff) return hipErrorInvalidValue;
    FlatStream c = {a.Qq, a.Kn, a.Vn, a.q4, a.O ? a.O : a.O_sub, (int32_t)a.cache_len, (int32_t)g.cap, (uint32_t)g.G << 16 | (uint32_t)g.Hkv,
                    (uint32_t)a.q_len << 16 | (uint32_t)a.plan.s_total, g.scale, g.B << 2 | (a.O ? 2 : 0) | a.causal, {by.Hkv.m, by.splits.m, by.G.m, by.steps.m}, 0};
    return launch_in_pieces(wgs, 64 * WAVES, [&](unsigned first, unsigned n) {
      c.first_wg = first;
      q4_stream_kernel<T, D, PP, RB, NT, FlatStream><<<dim3(n), 64 * WAVES, 0, st>>>(c);
    });
  }
  StreamCall c = {a, by, 0};
  return launch_in_pieces(wgs, 64 * WAVES, [&](unsigned first, unsigned n) {
    c.first_wg = first;
    q4_stream_kernel<T, D, PP, RB, NT, StreamCall><<<dim3(n), 64 * WAVES, 0, st>>>(c);
  });
}
template <typename T, int D, int PP, int RB>
hipError_t launch_stream(const Q4Args& a, hipStream_t st) {
  return q4_cache_resident(a.g, a.cache_len) ? launch_stream<T, D, PP, RB, false>(a, st) : launch_stream<T, D, PP, RB, true>(a, st);
}

}  // namespace

hipError_t launch_q4_store(int dtype, const Geom& g, const Q4Copy& c, hipStream_t st) { return launch_rows<false>(dtype, g, c, st); }
hipError_t launch_q4_load(int dtype, const Geom& g, const Q4Copy& c, hipStream_t st) { return launch_rows<true>(dtype, g, c, st); }

hipError_t launch_phase2_q4_stream(int dtype, const Q4Args& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.g.G * a.q_len;
  if (rows > a.plan.tile_rows || a.plan.tile_rows != (rows <= 16 ? 16 : 32)) return hipErrorInvalidValue;
  if (dtype == 0) {
    if (rows > 16) return hipErrorInvalidValue;
    return a.g.d == 64 ? launch_stream<float, 64, 2, 1>(a, st) : launch_stream<float, 128, 2, 1>(a, st);
  }
  if (rows <= 16) return a.parts == 2 ? launch_stream<__bf16, 128, 2, 1>(a, st) : launch_stream<__bf16, 128, 1, 1>(a, st);
  return a.parts == 2 ? launch_stream<__bf16, 128, 2, 2>(a, st) : launch_stream<__bf16, 128, 1, 2>(a, st);
}

}  // namespace star
