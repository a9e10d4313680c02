// Phase 2 over a cache held in four bits for calls of many rows (query encoding): bound by the matrix instructions.
//   * A workgroup is eight wavefronts of 16 RB rows each (token x head of a KV group) and a run of the cache.  All eight walk the same tiles of
//     64 keys, or (H = 2) four the even and four the odd ones, and meet behind the key loop.
//   * The wavefronts of a ring put a tile's codes into LDS as the bf16 numbers they stand for, once for all of its rows: K and V in two buffers each, written
//     while the ones before are read, a barrier per tile.  Codes are requested a tile ahead of that.
//   * S^T = K Q^T, the exponentiated scores are the B operand of O^T += V^T P^T, as in the stream (q4.hip).  A stage of 32 keys has the scores of unit
//     u + 1, the exponentials of unit u and the products of unit u - 1, which do not wait for each other.
//   * The reference of a row's exponentials is a whole power of two that moves where a weight would pass 2^15: what has been summed up so far, and the weights
//     of the unit on its way, are then multiplied by a power of two, which loses nothing, in a branch of its own.
// 256 tokens of 32 / 8 heads on 131072 keys, 5.5e11 flops: 452 to 475 us, 1.2 PFLOP/s, with weights in one part; 615 to 715 in two (8.2e11 flops with the part more, 1.15 to
// 1.3 PFLOP/s), where the matrix instructions are busy for 62 % of the cycles at 1.9 GHz.  A large library product reaches 1.34 to 1.38.
#include "q4_attend.h"

#include <type_traits>

namespace star {

namespace {

typedef const __attribute__((address_space(1))) unsigned char* GlobalBytes;

constexpr int KEYS = 64;              // of a tile
constexpr int THREADS = 512;
constexpr float HEADROOM = 4.f;       // a reference is set where the largest weight is 2^(TOP - 3) or down to half that, and moves where one passes 2^(TOP + 1)

struct TileDiv {
  Div Hkv, tiles, splits, G;
};

template <int D, int W>
struct Raw {                          // a thread's codes of a tile: E elements of one key, and their unit
  static constexpr int E = KEYS * D / (64 * W);
  uint32_t c[E / 8];
  uint32_t e;
};

template <int QP, int NS, int DT, int RB>
struct Rows {
  bf16x8 q[RB][QP][NS];
  f32x4 o[RB][DT];
  float ref[RB], above[RB];    // exponent of the reference (0 while nothing was seen), and what moves it
  f32x4 l[RB];                 // sums of the weights (see sum_up)
};
template <int RB>
struct Scores {
  f32x4 s[RB][2];
};

template <typename T, int D, int PP, int RB, int H>
__global__ __launch_bounds__(THREADS, 2) void q4_tiles_kernel(Q4Args a, TileDiv by, unsigned first_wg) {
  constexpr int QP = sizeof(T) == 2 ? 1 : 3, NS = D / 32, DT = D / 16, ROWB = 2 * D, W = 8 / H, ROWS = 16 * RB * W;
  constexpr int TILEB = KEYS * ROWB, UNITB = 32 * ROWB;
  typedef Raw<D, W> RawT;
  constexpr int E = RawT::E;
  __shared__ __attribute__((aligned(1024))) char lds[H][4][TILEB];            // K, K, V, V
  __shared__ uint32_t lds_e[H][2][KEYS];                                      // exponents of V, of tiles that not every row sees as a whole
  const Geom& g = a.g;
  const int ring = H == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 8), tid = threadIdx.x & (64 * W - 1);
  // Wavefronts w and w + 4 share a SIMD: the halves number their rows' from different ones, so that those of few rows keep all four busy.
  const int wave = (__builtin_amdgcn_readfirstlane(tid >> 6) + (ring ? 2 : 0)) & (W - 1), lane = tid & 63, qc = lane & 15, j4 = lane >> 4;
  uint32_t w = first_wg + blockIdx.x;
  uint32_t n = quotient(w, by.Hkv);
  const uint32_t kvh = w - n * by.Hkv.d;
  w = quotient(n, by.tiles);
  const uint32_t tile = by.tiles.d - 1 - (n - w * by.tiles.d);      // those that see most first
  n = quotient(w, by.splits);
  const uint32_t sp = w - n * by.splits.d, beta = n;

  const int R = g.G * a.q_len;
  const int cache_len = (int)a.cache_len, total = cache_len + (a.causal ? a.q_len : 0);
  const int cached = a.Kn ? cache_len : total;
  int64_t lo64, hi64;
  split_range(a.plan, g.L, g.b, total, sp, &lo64, &hi64);
  // Keys up to what the tile's last row sees; the last tile of the rows sees all, and files the call's tokens.
  // (us, 32 / 8 heads, 4096 tokens on 4000 keys: 634 with all keys for every tile, 535 so, 453 with the tiles that see most first; 300 of 20 sequences on 100 119 / 97 / 89)
  const uint32_t last_row = (tile + 1) * ROWS < (uint32_t)R ? (tile + 1) * ROWS - 1 : R - 1;
  const int seen = a.causal ? cache_len + (int)quotient(last_row, by.G) + 1 : total;
  const int lo = (int)lo64, hi = hi64 < seen ? (int)hi64 : seen;
  const int all_tiles = hi > lo ? (hi - lo + KEYS - 1) / KEYS : 0;
  const int n_tiles = H == 1 ? all_tiles : (all_tiles - ring + 1) / 2, most_tiles = H == 1 ? all_tiles : (all_tiles + 1) / 2;
  const auto key_of = [&](int t) INLINE { return lo + KEYS * (H == 1 ? t : 2 * t + ring); };

  Rows<QP, NS, DT, RB> r;
  int lim[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int row = tile * ROWS + wave * 16 * RB + 16 * b + qc;
    const bool live = row < R;
    const int j = live ? (int)quotient(row, by.G) : 0, head = kvh * g.G + (live ? row - j * g.G : 0);
    const int end = a.causal ? cache_len + j + 1 : total;
    lim[b] = !live ? 0 : end < hi ? end : hi;
    const T* p = (const T*)a.Qq + (((size_t)beta * a.q_len + j) * g.Hq + head) * D + j4 * (D / 4);
#pragma unroll
    for (int t = 0; t < NS; ++t) {
      float y[8];
      load8(p + 8 * t, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        __bf16 part[QP];
        split(live ? y[e] : 0.f, part);
#pragma unroll
        for (int i = 0; i < QP; ++i) r.q[b][i][t][e] = part[i];
      }
    }
  }
  // Keys from which on some row does not see all: of the workgroup, and of the wavefront
  const auto seen_by_all = [&](int row) INLINE {
    const int end = a.causal && row < R ? cache_len + (int)quotient(row, by.G) + 1 : total;
    return end < hi ? end : hi;
  };
  const int wg_free = seen_by_all(tile * ROWS), wave_free = seen_by_all(tile * ROWS + wave * 16 * RB);

  const bool busy = tile * ROWS + wave * 16 * RB < R;      // (the others put codes into LDS, no more)
  const float c = g.scale * LOG2E;
  const size_t rows0 = ((size_t)beta * g.Hkv + kvh) * (size_t)g.cap;

  // ---- codes to LDS
  constexpr int PER = D / E;                             // threads of a key
  const int my_key = tid / PER, my_col = tid % PER * E;
  const unsigned c_off = my_key * (D / 2) + my_col / 2, s_off = my_key * (D / 32) + my_col / 32;
  const int whole_hi = hi < cached ? hi : cached;
  const auto take = [&](RawT& raw, GlobalBytes codes, GlobalBytes scales) INLINE {
    if constexpr (E == 32) {
      const i32x4 y = *(const __attribute__((address_space(1))) i32x4*)codes;
#pragma unroll
      for (int i = 0; i < 4; ++i) raw.c[i] = (uint32_t)y[i];
    } else if constexpr (E == 16) {
      const i32x2 y = *(const __attribute__((address_space(1))) i32x2*)codes;
      raw.c[0] = (uint32_t)y[0];
      raw.c[1] = (uint32_t)y[1];
    } else {
      raw.c[0] = *(const __attribute__((address_space(1))) uint32_t*)codes;
    }
    raw.e = *scales;
  };
  const auto request = [&](RawT& raw, bool v, int t) INLINE {
    const unsigned char* codes = (const unsigned char*)(v ? a.q4.v_codes : a.q4.k_codes);
    const unsigned char* scales = (const unsigned char*)(v ? a.q4.v_scales : a.q4.k_scales);
    if (__builtin_expect(key_of(t) + KEYS <= whole_hi, 1)) {
      const size_t row = rows0 + key_of(t);
      take(raw, (GlobalBytes)codes + row * (D / 2) + c_off, (GlobalBytes)scales + row * (D / 32) + s_off);
      return;
    }
    const int key0 = key_of(t);
    int key = key0 + my_key;
    const bool there = key < hi;                         // keys past the last are that one again, masked below
    key = there ? key : hi - 1;
    if (key < cached) {
      take(raw, (GlobalBytes)codes + (rows0 + key) * (D / 2) + my_col / 2, (GlobalBytes)scales + (rows0 + key) * (D / 32) + my_col / 32);
    }
    if (key0 + KEYS > cached && cached < hi) {           // the call's own tokens among them (workgroup-uniform)
      const T* p = (const T*)(v ? a.Vn : a.Kn) + (((size_t)beta * a.q_len + (key < cached ? 0 : key - cached)) * g.Hkv + kvh) * D + my_col;
      float y[E / 8][8];
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < E / 8; ++i) {
        load8(p + 8 * i, y[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e) most = magnitude_bits(y[i][e]) > most ? magnitude_bits(y[i][e]) : most;
      }
#pragma unroll
      for (int s = 1; s < 32 / E; s <<= 1) {
        const uint32_t other = (uint32_t)__shfl_xor((int)most, s);
        most = other > most ? other : most;
      }
      if (key >= cached) {
        raw.e = q4_unit(most);
#pragma unroll
        for (int i = 0; i < E / 8; ++i) raw.c[i] = raw.e == 255u ? 0u : q4_codes(y[i], q4_unit_value(raw.e));
        if (there && tile + 1 == by.tiles.d) {
          uint32_t* at = (uint32_t*)((unsigned char*)codes + (rows0 + key) * (D / 2) + my_col / 2);
#pragma unroll
          for (int i = 0; i < E / 8; ++i) at[i] = raw.c[i];
          if (my_col % 32 == 0) ((unsigned char*)scales)[(rows0 + key) * (D / 32) + my_col / 32] = (unsigned char)raw.e;
        }
      }
    }
  };
  const unsigned lds0 = (unsigned)(size_t)(LDS_AS char*)lds[ring][0];
  unsigned put[E / 8];
#pragma unroll
  for (int i = 0; i < E / 8; ++i) put[i] = lds0 + my_key * ROWB + (((my_col / 8 + (E == 16 ? i ^ (my_key & 1) : i)) ^ swz<D>(my_key & 15)) << 4);
  const uint32_t swapped = E == 16 && (my_key & 1) ? 0xffffffffu : 0u;
  const auto file = [&](auto AS, const RawT& raw, unsigned buffer, int below = 0) INLINE {
    const float unit = below ? unit_down(raw.e, below) : q4_unit_value(raw.e);
#pragma unroll
    for (int i = 0; i < E / 8; ++i) {
      // (two chunks a thread: the first of every second key's threads is the odd one, so that they spread over all slots)
      const uint32_t code = E == 16 ? (swapped & raw.c[(i ^ 1) % (E / 8)]) | (~swapped & raw.c[i]) : raw.c[i];
      *(LDS_AS typename decltype(AS)::Vec*)(size_t)(put[i] + buffer) = decltype(AS)::values(code, unit);
    }
  };
  // ---- operands from LDS
  unsigned ka[NS], va[DT];
#pragma unroll
  for (int t = 0; t < NS; ++t) ka[t] = lds0 + qc * ROWB + (((j4 * NS + t) ^ swz<D>(qc)) << 4);
  const int rr = 4 * j4 + (qc >> 2);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) va[dt] = lds0 + 2 * TILEB + rr * ROWB + (((2 * dt + ((lane & 3) >> 1)) ^ swz<D>(rr)) << 4) + 8 * (lane & 1);

  Wide wide = {0, 0};
  int down = 0;
  const auto walk = [&](auto WIDE) INLINE {
    typedef Product<WIDE.value> P;
    typedef typename P::Vec Vec;
    typedef std::remove_reference_t<decltype(Vec()[0])> Elem;
    constexpr int PARTS = WIDE.value && PP > 1 ? 3 : PP;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) r.o[b][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
      r.ref[b] = 0.f;
      r.above[b] = -INFINITY;
      r.l[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // V of a tile that not every row sees: its NaN go to the rows that see them, behind the products (see below).
    const auto file_v = [&](RawT& raw, int t, unsigned buffer) INLINE {
      if (key_of(t) + KEYS > wg_free) {
        if (my_col % 32 == 0) {
          unsigned char* at = (unsigned char*)&lds_e[ring][t & 1][my_key];
          at[my_col / 32] = (unsigned char)raw.e;
          if (D == 64 && my_col == 0) at[2] = at[3] = 0;
        }
        if (raw.e == 255u) {
          raw.e = 127;
#pragma unroll
          for (int i = 0; i < E / 8; ++i) raw.c[i] = 0;
        }
      }
      wide.note(raw.e);
      file(P(), raw, buffer, WIDE.value ? down : 0);
    };

    typedef Scores<RB> S;
    typedef Vec Weights[RB][PARTS];
    static_assert(2 * NS == DT, "as many operands of K as of V in 32 keys");
    // K operand f of a unit: keys 16 (f % 2) .. +15, step f / 2 of the products.  V operand f: columns 16 f .. +15; slot e is key 4 j4 + e or 16 + 4 j4 + e - 4, as in
    // the weights.
    const auto read_k = [&](int f, unsigned at) INLINE { return *(LDS_AS bf16x8*)(size_t)(ka[f >> 1] + at + (f & 1) * 16 * ROWB); };
    const auto read_v = [&](int f, unsigned at) INLINE {
      const s16x4 y0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(size_t)(va[f] + at));
      const s16x4 y1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(size_t)(va[f] + at + 16 * ROWB));
      return __builtin_bit_cast(Vec, __builtin_shufflevector(y0, y1, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    const auto score_by = [&](S& s, const bf16x8& y, int f) INLINE {
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int i = QP - 1; i >= 0; --i) {
          const f32x4 acc = f < 2 && i == QP - 1 ? f32x4{0.f, 0.f, 0.f, 0.f} : s.s[b][f & 1];
          s.s[b][f & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y, r.q[b][i][f >> 1], acc, 0, 0, 0);
        }
    };
    const auto multiply_by = [&](const Weights& p, const Vec& y, int f) INLINE {
#pragma unroll
      for (int n = 0; n < RB; ++n) {
        const int b = f & 1 ? RB - 1 - n : n;       // (the same operand twice in a row where rows change)
#pragma unroll
        for (int i = PARTS - 1; i >= 0; --i) r.o[b][f] = P::multiply(y, p[b][i], r.o[b][f]);
      }
    };
    const auto mask = [&](S& s, int key0) INLINE {
      asm volatile("");                             // (a branch of its own: few tiles want it)
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int room = lim[b] - key0 - 4 * j4;      // element (kt, e) is key key0 + 16 kt + 4 j4 + e
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s.s[b][kt][e] = 16 * kt + e < room ? s.s[b][kt][e] : -INFINITY;
      }
    };
    // Exponents of a unit's weights; the references of its rows are raised first, where it asks for it.  `p`: weights against the ones before.
    typedef Exponents Powers[RB];
    const auto raise = [&](const S& s, Powers& x, Weights& p) INLINE {
      bool far = false;
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        x[b] = exponents(s.s[b], c, -r.ref[b]);
        far |= largest(x[b]) > r.above[b];
      }
      if (__builtin_expect(__builtin_amdgcn_ballot_w64(far) == 0, 1)) return;
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const float top = __builtin_ceilf(quad_max(largest(exponents(s.s[b], c, 0.f)))) - (TOP + 1 - HEADROOM);
        const bool none = r.above[b] == -INFINITY;                       // nothing was seen
        const float ref = none ? (top == -INFINITY ? 0.f : top) : fmaxf(r.ref[b], top);
        const float alpha = none ? 0.f : __builtin_amdgcn_exp2f(r.ref[b] - ref);
        r.ref[b] = ref;
        r.above[b] = none && top == -INFINITY ? -INFINITY : TOP + 1;
        r.l[b] *= alpha;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) r.o[b][dt] *= alpha;
#pragma unroll
        for (int i = 0; i < PARTS; ++i)
#pragma unroll
          for (int e = 0; e < 8; ++e) p[b][i][e] = (Elem)((float)p[b][i][e] * alpha);
        x[b] = exponents(s.s[b], c, -ref);
      }
    };
    const auto weigh = [&](const Powers& x, Weights& p) INLINE {
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int i = 0; i < 8; i += 2) P::template split<PARTS>(__builtin_amdgcn_exp2f(x[b].x[i]), __builtin_amdgcn_exp2f(x[b].x[i + 1]), p[b], i);
    };
    // The sums of the weights, as they are multiplied: products with ones in row 0, whose element 0 is the lanes' with j4 = 0.
    const Elem one = qc == 0 ? (Elem)1.f : (Elem)0.f;
    const Vec ones = {one, one, one, one, one, one, one, one};
    const auto sum_up = [&](const Weights& p) INLINE {
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int i = PARTS - 1; i >= 0; --i) r.l[b] = P::multiply(ones, p[b][i], r.l[b]);
    };

    RawT rk, rv;
    // A stage: scores of a unit (K at `k`), weights of the one before, products of the one before that (V at `v`).  The order of instructions is pinned:
    // a few of the vector unit's between two products, operands read ahead.
    // FILE: codes are put into LDS on the way (K at `to_k`, V at `to_v`).
    constexpr std::integral_constant<bool, true> FILED;
    constexpr std::integral_constant<bool, false> NOT_FILED;
    const auto stage = [&](auto FILE, S& next, unsigned k, Powers& now, Weights& p, const Weights& before, unsigned v, unsigned to_k, unsigned to_v) INLINE {
#pragma unroll
      for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(now[b].x[i]));      // (weights stay in their stage)
      bf16x8 kf[DT];
      Vec vf[DT];
#pragma unroll
      for (int f = 0; f < DT; ++f) { kf[f] = read_k(f, k); vf[f] = read_v(f, v); }
      weigh(now, p);
      if constexpr (FILE.value) {
        file(Product<true>(), rk, to_k);
        wide.note(rv.e);
        file(P(), rv, to_v, WIDE.value ? down : 0);
      }
#pragma unroll
      for (int f = 0; f < DT; f += 2) {
        score_by(next, kf[f], f);
        score_by(next, kf[f + 1], f + 1);
        multiply_by(before, vf[f], f);
        multiply_by(before, vf[f + 1], f + 1);
      }
      sum_up(before);
      constexpr int PRODUCTS = RB * (DT * (QP + PARTS) + PARTS), OPS = RB * (PARTS == 1 ? 12 : PARTS == 2 ? 24 : 52) + (FILE.value ? E + 8 : 0), READS = 3 * DT;
      constexpr int PER = (OPS + PRODUCTS - 1) / PRODUCTS, EVERY = RB * (QP + PARTS);
      __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
      for (int i = 0; i < PRODUCTS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (i % EVERY == EVERY - 1 && 6 + i / EVERY * 3 < READS) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, PER, 0);
        if (FILE.value && i % EVERY == EVERY - 1 && i / EVERY >= DT - E / 4 && i / EVERY < DT) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b) {
#pragma unroll
        for (int i = 0; i < PARTS; ++i) asm volatile("" : "+v"(p[b][i]));
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    const auto score = [&](S& s, unsigned k) INLINE {
#pragma unroll
      for (int f = 0; f < DT; ++f) score_by(s, read_k(f, k), f);
    };
    const auto multiply = [&](const Weights& p, unsigned v) INLINE {
#pragma unroll
      for (int f = 0; f < DT; ++f) multiply_by(p, read_v(f, v), f);
      sum_up(p);
    };

    const auto barrier = []() INLINE {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
      __builtin_amdgcn_s_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    };
    S sA, sB;
    Weights pA, pB;
    Powers x;
    if (n_tiles > 0) {
      request(rk, false, 0);
      request(rv, true, 0);
      file(Product<true>(), rk, 0);
      file_v(rv, 0, 2 * TILEB);
      if (n_tiles > 1) {
        request(rk, false, 1);
        request(rv, true, 1);
        file(Product<true>(), rk, TILEB);
        if (n_tiles > 2) request(rk, false, 2);
      }
    }
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
      for (int i = 0; i < PARTS; ++i) pA[b][i] = Vec{0, 0, 0, 0, 0, 0, 0, 0};
    barrier();
    if (!busy) {
      for (int t = 0; t < most_tiles; ++t) {
        barrier();
        const unsigned odd = t & 1 ? TILEB : 0;
        if (t + 2 < n_tiles) file(Product<true>(), rk, odd);
        if (t + 1 < n_tiles) file_v(rv, t + 1, 2 * TILEB + TILEB - odd);
        if (t + 3 < n_tiles) request(rk, false, t + 3);
        if (t + 2 < n_tiles) request(rv, true, t + 2);
      }
      return;
    }
    if (n_tiles > 0) {
      score(sA, 0);
      score(sB, UNITB);
      const int key0 = key_of(0);
      if (key0 + KEYS > wave_free) { mask(sA, key0); mask(sB, key0 + 32); }
      raise(sA, x, pA);
      weigh(x, pA);
    }
    // A value that is NaN counts where its key is seen and nowhere else, and its weight may be zero where it is not.
    const auto not_numbers = [&](int t) INLINE {
      const int key0 = key_of(t);
      if (key0 + KEYS <= wg_free) return;
      const uint32_t e = lds_e[ring][t & 1][lane];
      bool nan = false;
#pragma unroll
      for (int k = 0; k < D / 32; ++k) nan |= (e >> (8 * k) & 255u) == 255u;
      for (uint64_t left = __builtin_amdgcn_ballot_w64(nan); left; left &= left - 1) {
        const int key = __builtin_ctzll(left);
        const uint32_t which = lds_e[ring][t & 1][key];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
          for (int dt = 0; dt < DT; ++dt)
            if (key0 + key < lim[b] && (which >> (8 * (dt / 2)) & 255u) == 255u) r.o[b][dt] = f32x4{NAN, NAN, NAN, NAN};
      }
    };
    // Tile t: its V is multiplied while K of tile t + 1 makes the next scores, K of tile t + 2 and V of tile t + 1 are filed.
    const auto step = [&](int t, unsigned odd) INLINE {      // odd: TILEB for odd t
      const unsigned even = TILEB - odd;
      barrier();
      if (t + 2 < n_tiles) file(Product<true>(), rk, odd);
      file_v(rv, t + 1, 2 * TILEB + even);
      if (t + 3 < n_tiles) request(rk, false, t + 3);
      if (t + 2 < n_tiles) request(rv, true, t + 2);
      const int key1 = key_of(t + 1);
      const bool partly = key1 + KEYS > wave_free;
      raise(sB, x, pA);
      stage(NOT_FILED, sA, even, x, pB, pA, odd, 0, 0);
      if (__builtin_expect(partly, 0)) mask(sA, key1);
      raise(sA, x, pB);
      stage(NOT_FILED, sB, even + UNITB, x, pA, pB, odd + UNITB, 0, 0);
      if (__builtin_expect(partly, 0)) mask(sB, key1 + 32);
      not_numbers(t);
    };
    const auto last = [&](int t, unsigned odd) INLINE {
      barrier();
      raise(sB, x, pA);
      weigh(x, pB);
      multiply(pA, odd);
      multiply(pB, odd + UNITB);
      not_numbers(t);
    };
    // The same where tiles up to t + 3 are cached and seen by all rows as a whole: nothing to ask for.
    const int plain_hi = whole_hi < wg_free ? whole_hi : wg_free;
    const int n_plain = plain_hi > key_of(0) ? (plain_hi - key_of(0) + KEYS * (H - 1)) / (KEYS * H) : 0;
    GlobalBytes next_kc = (GlobalBytes)a.q4.k_codes + (rows0 + key_of(3)) * (D / 2), next_ks = (GlobalBytes)a.q4.k_scales + (rows0 + key_of(3)) * (D / 32);
    GlobalBytes next_vc = (GlobalBytes)a.q4.v_codes + (rows0 + key_of(2)) * (D / 2), next_vs = (GlobalBytes)a.q4.v_scales + (rows0 + key_of(2)) * (D / 32);
    const auto plain_step = [&](unsigned odd) INLINE {
      const unsigned even = TILEB - odd;
      barrier();
      raise(sB, x, pA);
      stage(FILED, sA, even, x, pB, pA, odd, odd, 2 * TILEB + even);
      take(rk, next_kc + c_off, next_ks + s_off);
      take(rv, next_vc + c_off, next_vs + s_off);
      next_kc += KEYS * H * (D / 2);
      next_ks += KEYS * H * (D / 32);
      next_vc += KEYS * H * (D / 2);
      next_vs += KEYS * H * (D / 32);
      raise(sA, x, pB);
      stage(NOT_FILED, sB, even + UNITB, x, pA, pB, odd + UNITB, 0, 0);
    };
    int t = 0;
    for (; t + 4 < n_plain; t += 2) {
      plain_step(0);
      plain_step(TILEB);
    }
    for (; t + 2 < n_tiles; t += 2) {
      step(t, 0);
      step(t + 1, TILEB);
    }
    if (t + 2 == n_tiles) {
      step(t, 0);
      last(t + 1, TILEB);
    } else if (t < n_tiles) {
      last(t, 0);
    }
    if (H == 2 && n_tiles < most_tiles) barrier();      // (the other half has a tile more)

  };
  walk(std::integral_constant<bool, false>());
  __shared__ int lds_wide[8];
  if (lane == 0) lds_wide[threadIdx.x >> 6] = wide.flags();
  __syncthreads();
  int any_wide = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) any_wide |= lds_wide[k];
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(any_wide) != 0, 0)) {
    down = any_wide & 2 ? DOWN : 0;
    walk(std::integral_constant<bool, true>());
  }

  // ---- results.  The halves meet: the second hands over (O, m, l), register by register.
  float l[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) l[b] = quad_sum(j4 == 0 ? r.l[b][0] : 0.f);
  if constexpr (H == 2) {
    static_assert(4 * RB * (DT + 1) * 1024 <= (int)sizeof(lds), "");
    __syncthreads();
    LDS_AS char* box = (LDS_AS char*)(size_t)(unsigned)(size_t)(LDS_AS char*)lds[0][0] + wave * (RB * (DT + 1) * 1024) + lane * 16;
    if (ring == 1) {
#pragma unroll
      for (int b = 0; b < RB; ++b) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(LDS_AS f32x4*)(box + (b * (DT + 1) + dt) * 1024) = r.o[b][dt];
        *(LDS_AS f32x4*)(box + (b * (DT + 1) + DT) * 1024) = f32x4{r.above[b] == -INFINITY ? -INFINITY : r.ref[b], l[b], 0.f, 0.f};
      }
    }
    __syncthreads();
    if (ring == 1) return;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const f32x4 ml = *(LDS_AS f32x4*)(box + (b * (DT + 1) + DT) * 1024);
      const float mine = r.above[b] == -INFINITY ? -INFINITY : r.ref[b], most = fmaxf(mine, ml[0]), ref = most == -INFINITY ? 0.f : most;
      const float s0 = __builtin_amdgcn_exp2f(mine - ref), s1 = __builtin_amdgcn_exp2f(ml[0] - ref);
      l[b] = l[b] * s0 + ml[1] * s1;
      r.ref[b] = ref;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) r.o[b][dt] = r.o[b][dt] * s0 + *(LDS_AS f32x4*)(box + (b * (DT + 1) + dt) * 1024) * s1;
    }
  }
  const size_t out0 = ((size_t)beta * a.plan.s_total + sp) * g.Hq * a.q_len;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int row = tile * ROWS + wave * 16 * RB + 16 * b + qc;
    if (row >= R) continue;
    const int j = (int)quotient(row, by.G);
    const int h = kvh * g.G + row - j * g.G;
    const size_t out = out0 + (size_t)h * a.q_len + j;
    const float inv = l[b] == 0.f ? 0.f : 1.f / l[b], up = down ? __builtin_ldexpf(1.f, DOWN) : 1.f;
    if (a.O) {
      T* o = (T*)a.O + (((size_t)beta * a.q_len + j) * g.Hq + h) * D + 4 * j4;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) store4(o + 16 * dt, r.o[b][dt] * inv * up);
      continue;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) *(f32x4*)(a.O_sub + out * D + 16 * dt + 4 * j4) = r.o[b][dt] * inv * up;
    if (j4 == 0) a.LSE_sub[out] = l[b] == 0.f ? -INFINITY : (r.ref[b] + __builtin_amdgcn_logf(l[b])) * LN2;
  }
}

template <typename T, int D, int PP, int RB, int H>
hipError_t launch_tiles(const Q4Args& a, hipStream_t st) {
  const Geom& g = a.g;
  constexpr int ROWS = 16 * RB * (8 / H);
  const uint32_t tiles = (uint32_t)(((int64_t)g.G * a.q_len + ROWS - 1) / ROWS);
  const TileDiv by = {make_div(g.Hkv), make_div(tiles), make_div(a.plan.s_total), make_div(g.G)};
  const int64_t wgs = (int64_t)g.B * g.Hkv * tiles * a.plan.s_total;
  if (wgs > 0x7fffffff) return hipErrorInvalidValue;
  return launch_in_pieces(wgs, THREADS, [&](unsigned first, unsigned n) {
    q4_tiles_kernel<T, D, PP, RB, H><<<dim3(n), THREADS, 0, st>>>(a, by, first);
  });
}

}  // namespace

hipError_t launch_phase2_q4_tiles(int dtype, const Q4Args& a, hipStream_t st) {
  const int rows = a.plan.tile_rows;
  if (dtype != 0) {
    if (rows == 256) return a.parts == 2 ? launch_tiles<__bf16, 128, 2, 2, 1>(a, st) : launch_tiles<__bf16, 128, 1, 2, 1>(a, st);
    return a.parts == 2 ? launch_tiles<__bf16, 128, 2, 2, 2>(a, st) : launch_tiles<__bf16, 128, 1, 2, 2>(a, st);
  }
  if (a.g.d == 64) return rows == 128 ? launch_tiles<float, 64, 2, 1, 1>(a, st) : launch_tiles<float, 64, 2, 1, 2>(a, st);
  return rows == 128 ? launch_tiles<float, 128, 2, 1, 1>(a, st) : launch_tiles<float, 128, 2, 1, 2>(a, st);
}

}  // namespace star
