// arbor_append: norm of each query and key head, rotation by position, and the K/V
// rows of new tokens into the paged pool, in one pass over the projections.
//
// A workgroup takes one token.  Its angles are formed once, in 64 bits (a far
// position times a frequency does not fit 24 bits of mantissa: at position 10^5 an
// fp32 angle is off by up to 4e-3), and their sines and cosines, rounded once, shared
// through LDS; then every group of D / 8 lanes takes one head, eight elements a lane.
// The sum of squares crosses the lanes by DPP; nothing but the angles goes through LDS,
// and each element is read and written once: HBM-bound.  The norm's factor comes last: a
// bf16 element times its weight is exact in fp32.
//
// Where a pair of the rotation lies in one lane's 16 bytes (neighbours) or in those of the
// lane half a head further on (halves of a whole head), a lane takes eight elements in a
// row and its partner's come by DPP.  Otherwise (part of a head rotated by halves) it
// takes two pieces of four whose elements are pairs: 4 q and rotary_dim / 2 + 4 q.
#include "arbor_internal.h"
#include "mfma_ops.h"

namespace arbor {

namespace {

struct AppendArgs {
  Pool pl;
  arbor_append_t a;
  int64_t num_tokens;     // rows of the record
  int layer, n_tokens;
  int32_t *status;
};

template <class T>
struct Piece;                                   // four elements
template <>
struct Piece<__bf16> {
  typedef __bf16 reg __attribute__((ext_vector_type(4)));
};
template <>
struct Piece<float> {
  typedef f32x4 reg;
};

// sum over the LPR lanes of a row's group, in each of them
template <int LPR, class F>
__device__ __forceinline__ F row_sum(F v) {
  v += dpp_move<dpp::kQuadXor1>(v);
  v += dpp_move<dpp::kQuadXor2>(v);
  v += dpp_move<dpp::kRowHalfMirror>(v);
  if constexpr (LPR == 16) v += dpp_move<dpp::kRowMirror>(v);
  return v;
}

// value of the lane half a row's group further on
template <int LPR>
__device__ __forceinline__ uint32_t other_half(uint32_t v) {
  if constexpr (LPR == 16) return dpp_move<dpp::kRowMirror>(dpp_move<dpp::kRowHalfMirror>(v));
  return dpp_move<dpp::kQuadMirror>(dpp_move<dpp::kRowHalfMirror>(v));
}

// sin and cos of 2 pi x by their Taylor series, after x is brought to an eighth of a turn
// on either side of a quarter: the first terms left out are 5e-17 and 2e-18.
template <class F>
__device__ __forceinline__ void sin_cos_turns(double x, F *s, F *c) {
  x -= rint(x);                                 // (exact)
  const double k = rint(4.0 * x);
  const double r = (x - 0.25 * k) * 6.283185307179586476925, z = r * r;
  double ps = -1.0 / 1307674368000.0, pc = 1.0 / 20922789888000.0;
  ps = fma(ps, z, 1.0 / 6227020800.0), pc = fma(pc, z, -1.0 / 87178291200.0);
  ps = fma(ps, z, -1.0 / 39916800.0), pc = fma(pc, z, 1.0 / 479001600.0);
  ps = fma(ps, z, 1.0 / 362880.0), pc = fma(pc, z, -1.0 / 3628800.0);
  ps = fma(ps, z, -1.0 / 5040.0), pc = fma(pc, z, 1.0 / 40320.0);
  ps = fma(ps, z, 1.0 / 120.0), pc = fma(pc, z, -1.0 / 720.0);
  ps = fma(ps, z, -1.0 / 6.0), pc = fma(pc, z, 1.0 / 24.0);
  pc = fma(pc, z, -0.5);
  const F sr = (F)fma(r * z, ps, r), cr = (F)fma(pc, z, 1.0);
  const int quarter = (int)k & 3;
  const F u = quarter & 1 ? cr : sr, v = quarter & 1 ? sr : cr;
  *s = quarter & 2 ? -u : u;
  *c = (quarter + 1) & 2 ? -v : v;
}

// A bf16 result is formed again in 64 bits where fp32 does not decide it: where the value
// and kOff of its terms' magnitudes more, and as much less, round to different bf16.  In
// units of 2^-24 of r (|y_a cos| + |y_b sin|), r the norm's factor: r is off by at most 6
// (seven additions of exact squares and one of eps, halved by the root, which adds 2), sine
// and cosine by 1, one product and the sum by 1 each, the product with r by 1, the two ends
// by 1; 12 covers their products too.  Where the terms cancel, that is many last places of
// the result.
constexpr float kOff = 12.0f * 0x1p-24f;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// The values f, which may be off by d, rounded; the bits in which the rounded ends of
// [f - d, f + d] differ are added to `open`.
__device__ __forceinline__ bf16x2 rounded(f32x2 f, f32x2 d, uint32_t *open) {
  const bf16x2 lo = __builtin_convertvector(f - d, bf16x2);
  const bf16x2 hi = __builtin_convertvector(f + d, bf16x2);
  *open |= __builtin_bit_cast(uint32_t, lo) ^ __builtin_bit_cast(uint32_t, hi);
  return lo;
}
// Sum of the squares of eight elements, exact for bf16 but for the additions, in pairs.
__device__ __forceinline__ float squares(const float (&v)[8]) {
  float s[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    s[e] = __builtin_fmaf(v[2 * e], v[2 * e], v[2 * e + 1] * v[2 * e + 1]);
  return (s[0] + s[1]) + (s[2] + s[3]);
}
__device__ __forceinline__ double squares_64(const float (&v)[8]) {
  double s = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fma((double)v[e], (double)v[e], s);
  return s;
}
// rounded to fp32 and to T, as fp32 arithmetic without an error would be
template <class T>
__device__ __forceinline__ T by_fp32(double v) {
  float f = (float)v;
  asm volatile("" : "+v"(f));
  return (T)f;
}

// 1 / sqrt(x), within 2^-23: for bf16 rows by the instruction, which takes an x below the
// normal range for 0
template <class T>
__device__ __forceinline__ float norm_factor(float x) {
  if constexpr (sizeof(T) == 4) return 1.0f / sqrtf(x);
  const bool tiny = x < 0x1p-100f;
  return __builtin_amdgcn_rsqf(tiny ? x * 0x1p100f : x) * (tiny ? 0x1p50f : 1.0f);
}

// 1 / sqrt(x) by the instruction, good to 2^-23 or so, and two steps of Newton's method
__device__ __forceinline__ double inverse_root(double x) {
  const double r = __builtin_amdgcn_rsq(x);
  const double n = fma(0.5 * r, fma(-x * r, r, 1.0), r), m = fma(0.5 * n, fma(-x * n, n, 1.0), n);
  return r > 0.0 && r < 1.0e300 ? m : r;        // (0 of an infinity, infinity of 0)
}

// What a token has, loaded in one round trip beside its first rows.
struct Token {
  int64_t slot, rec;
  int32_t pos;
  float freq;                                   // of pair tid
  int32_t status;
};
__device__ __forceinline__ Token load_token(const AppendArgs &args, int64_t t, int tid) {
  const arbor_append_t &a = args.a;
  const int half = a.rotary_dim / 2;
  // (no branches: what is not needed is read from where something else lies)
  const float *freq = half > 0 ? a.inv_freq + min(tid, half - 1)
                               : reinterpret_cast<const float *>(a.positions);
  Token k;
  k.status = status_word(args.status);
  k.freq = *freq;
  k.slot = a.slots[t];
  k.rec = (a.record_k ? a.tokens : a.slots)[t];
  k.pos = a.positions[t];
  return k;
}
// Whether the token has a place; it is left out if not, and refused unless it is padding.
__device__ __forceinline__ bool has_place(const AppendArgs &args, Token &k, int tid) {
  const bool record = args.a.record_k != nullptr;
  asm volatile("" : "+s"(k.slot), "+s"(k.rec), "+s"(k.pos));   // (no load moves below)
  if (k.slot == -1) return false;
  if (k.slot < 0 || k.slot >= args.pl.num_pages * args.pl.P ||
      (record && (k.rec < 0 || k.rec >= args.num_tokens))) {
    if (tid == 0) status_error(args.status, ARBOR_EINVAL);
    return false;
  }
  return true;
}

// Token t's rows of q, k and v as heads 0, 1, .. of one row: where the next tensor begins,
// its distance is added.  (Of a choice between the arguments the compiler makes loads of
// what each lane needs from the arguments in memory.)
template <class T, int D>
struct Heads {
  const char *q;
  int64_t to_k, to_v;
  int hq, hkv;
  __device__ __forceinline__ Heads(const arbor_append_t &a, const Pool &pl, int64_t t)
      : hq(pl.Hkv * pl.G), hkv(pl.Hkv) {
    q = reinterpret_cast<const char *>(static_cast<const T *>(a.q) + t * a.q_stride);
    const char *k = reinterpret_cast<const char *>(static_cast<const T *>(a.k) + t * a.k_stride);
    const char *v = reinterpret_cast<const char *>(static_cast<const T *>(a.v) + t * a.v_stride);
    to_k = (k - q) - (int64_t)hq * (D * sizeof(T));
    to_v = (v - k) - (int64_t)hkv * (D * sizeof(T));
  }
  __device__ __forceinline__ const T *operator[](int h) const {
    return reinterpret_cast<const T *>(q + (int64_t)h * (D * sizeof(T)) + (h >= hq ? to_k : 0) +
                                       (h >= hq + hkv ? to_v : 0));
  }
};

// Part of a head rotated by halves; see above.  8,192 tokens of the 70B shape, half of each
// head rotated: 73 us.
template <class T, int D>
__global__ __launch_bounds__(256) void append_rows(AppendArgs args) {
  constexpr int LPR = D / 8;                    // lanes of a head
  constexpr int RPS = 256 / LPR;                // heads a step
  constexpr int UNROLL = 4;                     // steps whose loads are in flight together
  typedef typename Piece<T>::reg reg;
  __shared__ double sh_cos[D / 2], sh_sin[D / 2];
  __shared__ int32_t sh_status;
  const arbor_append_t &a = args.a;
  const Pool &pl = args.pl;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, q8 = tid % LPR;
  const int rd = a.rotary_dim, half = rd / 2;
  const bool turns = q8 < rd / 8;               // this lane's pieces lie half apart
  const int ca = turns ? 4 * q8 : 8 * q8, cb = turns ? half + 4 * q8 : 8 * q8 + 4;
  const int Hq = pl.Hkv * pl.G, heads = Hq + 2 * pl.Hkv;
  const Heads<T, D> rows(a, pl, t);
  // the first heads' loads are on their way while the angles are formed (without a branch,
  // behind which the compiler would wait for all of them)
  reg xa[UNROLL], xb[UNROLL];
  auto load = [&](int h0, int last) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int h = min(h0 + u * RPS, last);
      if (h < heads) {
        const T *p = rows[h];
        xa[u] = *reinterpret_cast<const reg *>(p + ca);
        xb[u] = *reinterpret_cast<const reg *>(p + cb);
      }
    }
  };
  int h0 = tid / LPR;
  Token k = load_token(args, t, tid);
  load(h0, heads - 1);
  if (!has_place(args, k, tid)) return;
  // in turns: x = pos f / (2 pi) in fp64 is off by 2^-53 relative, 1e-10 turns at position
  // 10^6
  if (tid < half)
    sin_cos_turns((double)k.pos * (double)k.freq * 0.15915494309189535, &sh_sin[tid],
                  &sh_cos[tid]);
  if (tid == 0) sh_status = k.status;
  __syncthreads();
  if (sh_status < 0) return;
  float co[4], si[4];                           // of the pairs (xa[e], xb[e])
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    co[e] = turns ? (float)sh_cos[4 * q8 + e] : 1.0f;
    si[e] = turns ? (float)sh_sin[4 * q8 + e] : 0.0f;
  }
  const int64_t page = k.slot / pl.P, row = k.slot % pl.P;
  for (; h0 < heads; h0 += UNROLL * RPS) {
    if (h0 >= UNROLL * RPS) load(h0, INT32_MAX);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int h = h0 + u * RPS;
      if (h >= heads) break;
      const bool is_q = h < Hq, is_v = h >= Hq + pl.Hkv;
      reg ya = xa[u], yb = xb[u];
      if (!is_v) {
        float va[4], vb[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          va[e] = (float)ya[e];
          vb[e] = (float)yb[e];
        }
        const void *w = is_q ? a.q_norm : a.k_norm;
        float r = 1.0f;
        if (w) {
          const float all[8] = {va[0], va[1], va[2], va[3], vb[0], vb[1], vb[2], vb[3]};
          r = norm_factor<T>(row_sum<LPR>(squares(all)) * (1.0f / D) + a.eps);
          const reg wa = *reinterpret_cast<const reg *>(static_cast<const T *>(w) + ca);
          const reg wb = *reinterpret_cast<const reg *>(static_cast<const T *>(w) + cb);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            va[e] *= (float)wa[e];               // (exact for bf16)
            vb[e] *= (float)wb[e];
          }
        }
        uint32_t open = 0;
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          f32x2 f, g, df, dg;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float x = va[e + i], y = vb[e + i], c = co[e + i], s = si[e + i];
            const float ys = y * s, xs = x * s;
            f[i] = r * (turns ? __builtin_fmaf(x, c, -ys) : x);
            g[i] = r * (turns ? __builtin_fmaf(y, c, xs) : y);
            df[i] = kOff * r * (turns ? __builtin_fmaf(fabsf(x), fabsf(c), fabsf(ys)) : fabsf(x));
            dg[i] = kOff * r * (turns ? __builtin_fmaf(fabsf(y), fabsf(c), fabsf(xs)) : fabsf(y));
          }
          if constexpr (sizeof(T) == 2) {
            const bf16x2 wa = rounded(f, df, &open), wb = rounded(g, dg, &open);
            ya[e] = wa[0], ya[e + 1] = wa[1], yb[e] = wb[0], yb[e + 1] = wb[1];
          } else {
            ya[e] = f[0], ya[e + 1] = f[1], yb[e] = g[0], yb[e + 1] = g[1];
          }
        }
        if (sizeof(T) == 2 && __builtin_expect(ballot(open != 0) != 0, 0)) {
          double x = 1.0;
          if (w) {
            float all[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) all[e] = (float)xa[u][e], all[4 + e] = (float)xb[u][e];
            x = inverse_root(row_sum<LPR>(squares_64(all)) * (1.0 / D) + a.eps);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const double c = turns ? sh_cos[4 * q8 + e] : 1.0, s = sh_sin[turns ? 4 * q8 + e : 0];
            const double p = va[e], q = vb[e];       // (exact)
            ya[e] = by_fp32<T>(x * (turns ? fma(-q, s, p * c) : p));
            yb[e] = by_fp32<T>(x * (turns ? fma(p, s, q * c) : q));
          }
        }
      }
      T *out;
      if (is_q) {
        out = static_cast<T *>(a.q_out) + (t * Hq + h) * D;
      } else {
        const int g = is_v ? h - Hq - pl.Hkv : h - Hq;
        out = reinterpret_cast<T *>(static_cast<char *>(is_v ? pl.v : pl.k) +
                                    row_byte_offset(pl, args.layer, page, g, (int)row));
        if (a.record_k) {
          T *r = static_cast<T *>(is_v ? a.record_v : a.record_k) +
                 ((k.rec * pl.L + args.layer) * pl.Hkv + g) * D;
          *reinterpret_cast<reg *>(r + ca) = ya;
          *reinterpret_cast<reg *>(r + cb) = yb;
        }
      }
      *reinterpret_cast<reg *>(out + ca) = ya;
      *reinterpret_cast<reg *>(out + cb) = yb;
    }
  }
}

// The same with eight elements in a row a lane; see above.  A workgroup of four waves, or of
// one, takes a token.  A step's registers take the next load as soon as they are read, two
// steps ahead (four: as fast in the 70B shape, 5 to 15 % slower in fp32 and for fewer
// heads).  Each line is read once and written once, past the caches (with ordinary stores
// 8,192 tokens of the 8B shape 48 us against 45, of the 70B shape 82 against 74).
// 8,192 tokens of 64 + 8 + 8 heads of 128 bf16, 336 MB: 70 us, 4.8 TB/s of the 5.1 of a
// large copy.
//
// A bf16 that fp32 rounds to the other side moves its key's logits by up to 2^-8 of a
// product, so the few pairs of elements that fp32 does not decide are formed again in 64 bits
// (2 to 5 us; where one of a lane's eight brought on all of them, 10 to 12; all
// elements of all rows, 18 and more).
template <class T, int D, bool HALVES, int BLOCK>
__global__ __launch_bounds__(BLOCK, BLOCK == 64 && sizeof(T) == 2 ? 8 : 4) void append_whole(
    AppendArgs args) {
  constexpr int LPR = D / 8;                    // lanes of a head
  constexpr int RPS = BLOCK / LPR;              // heads a step
  constexpr int UNROLL = 2;                     // steps whose loads are in flight together
  constexpr int W = sizeof(T) * 2;              // words of eight elements
  struct Eight {
    T e[8];
  };
  typedef uint32_t words __attribute__((ext_vector_type(W), aligned(16)));
  __shared__ __attribute__((aligned(16))) double sh_cos[D / 2], sh_sin[D / 2];
  __shared__ __attribute__((aligned(16))) float near_cos[D / 2], near_sin[D / 2];
  __shared__ int32_t sh_status;
  const arbor_append_t &a = args.a;
  const Pool &pl = args.pl;
  const int64_t t = blockIdx.x;
  const int tid = threadIdx.x, q8 = tid % LPR;
  const int rd = a.rotary_dim, half = rd / 2;
  const int Hq = pl.Hkv * pl.G, heads = Hq + 2 * pl.Hkv;
  const Heads<T, D> rows(a, pl, t);
  // the first heads' loads are on their way while the angles are formed (without a branch,
  // behind which the compiler would wait for all of them)
  words x[UNROLL];
  auto fetch = [&](int u, int h) {
    if (h < heads)
      x[u] = __builtin_nontemporal_load(reinterpret_cast<const words *>(rows[h] + 8 * q8));
  };
  int h0 = tid / LPR;
  Token k = load_token(args, t, tid);
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) fetch(u, min(h0 + u * RPS, heads - 1));
  if (!has_place(args, k, tid)) return;
  // in turns: pos f / (2 pi) in fp64 is off by 2^-53 relative, 1e-10 turns at position
  // 10^6
  if (tid < half) {
    double s, c;
    sin_cos_turns((double)k.pos * (double)k.freq * 0.15915494309189535, &s, &c);
    sh_sin[tid] = s, sh_cos[tid] = c;
    near_sin[tid] = (float)s, near_cos[tid] = (float)c;
  }
  if (tid == 0) sh_status = k.status;
  __syncthreads();
  if (sh_status < 0) return;
  // element e becomes own co + partner si
  const bool turns = 8 * q8 < rd;
  auto pair = [&](int e) { return HALVES ? (8 * q8 + e) & (D / 2 - 1) : 4 * q8 + e / 2; };
  auto first = [&](int e) { return HALVES ? 8 * q8 < half : e % 2 == 0; };
  const int64_t page = k.slot / pl.P, row = k.slot % pl.P;
  for (; h0 < heads; h0 += UNROLL * RPS) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int h = h0 + u * RPS;
      if (h >= heads) break;
      const bool is_q = h < Hq, is_v = h >= Hq + pl.Hkv;
      words y = x[u];
      fetch(u, h + UNROLL * RPS);
      if (!is_v) {
        words z = y;
        if constexpr (HALVES)
#pragma unroll
          for (int i = 0; i < W; ++i) z[i] = other_half<LPR>(y[i]);
        const Eight own = __builtin_bit_cast(Eight, y), far = __builtin_bit_cast(Eight, z);
        float v[8], p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          v[e] = (float)own.e[e];
          p[e] = (float)far.e[HALVES ? e : e ^ 1];
        }
        const T *w = static_cast<const T *>(is_q ? a.q_norm : a.k_norm);
        float r = 1.0f;
        if (w) {
          r = norm_factor<T>(row_sum<LPR>(squares(v)) * (1.0f / D) + a.eps);
          const int c = 8 * q8;
          const Eight wo = __builtin_bit_cast(Eight, *reinterpret_cast<const words *>(w + c));
          const Eight wf = __builtin_bit_cast(
              Eight, *reinterpret_cast<const words *>(w + (HALVES ? c ^ (D / 2) : c)));
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] *= (float)wo.e[e];              // (exact for bf16)
            p[e] *= (float)wf.e[HALVES ? e : e ^ 1];
          }
        }
        Eight out;
        uint32_t open[4] = {0, 0, 0, 0};
        asm volatile("" ::: "memory");   // (the sines are read here, not kept in registers)
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          f32x2 f, d;
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float c = near_cos[pair(e + i)], s = near_sin[pair(e + i)], y = v[e + i];
            const float t = p[e + i] * (first(e + i) ? -s : s);
            f[i] = r * (turns ? __builtin_fmaf(y, c, t) : y);
            d[i] = kOff * r * (turns ? __builtin_fmaf(fabsf(y), fabsf(c), fabsf(t)) : fabsf(y));
          }
          if constexpr (sizeof(T) == 2) {
            const bf16x2 w2 = rounded(f, d, &open[e / 2]);
            out.e[e] = w2[0], out.e[e + 1] = w2[1];
            if (e == 2) __builtin_amdgcn_sched_barrier(0);   // (half the sines at a time)
          } else {
            out.e[e] = f[0], out.e[e + 1] = f[1];
          }
        }
        if (sizeof(T) == 2 &&
            __builtin_expect(ballot((open[0] | open[1] | open[2] | open[3]) != 0) != 0, 0)) {
          // (v and p are exact)
          asm volatile("" ::: "memory");
          double x = 1.0;
          if (w) {
            float all[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) all[e] = (float)own.e[e];
            x = inverse_root(row_sum<LPR>(squares_64(all)) * (1.0 / D) + a.eps);
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            if (ballot(open[e / 2] != 0)) {
              double y = v[e];
              if (turns) {
                const double s = sh_sin[pair(e)];
                y = fma((double)p[e], first(e) ? -s : s, y * sh_cos[pair(e)]);
              }
              out.e[e] = by_fp32<T>(y * x);
            }
            __builtin_amdgcn_sched_barrier(0);       // (one at a time, in few registers)
          }
        }
        y = __builtin_bit_cast(words, out);
      }
      T *out;
      if (is_q) {
        out = static_cast<T *>(a.q_out) + (t * Hq + h) * D;
      } else {
        const int g = is_v ? h - Hq - pl.Hkv : h - Hq;
        out = reinterpret_cast<T *>(static_cast<char *>(is_v ? pl.v : pl.k) +
                                    row_byte_offset(pl, args.layer, page, g, (int)row));
        if (a.record_k) {
          T *r = static_cast<T *>(is_v ? a.record_v : a.record_k) +
                 ((k.rec * pl.L + args.layer) * pl.Hkv + g) * D;
          *reinterpret_cast<words *>(r + 8 * q8) = y;
        }
      }
      __builtin_nontemporal_store(y, reinterpret_cast<words *>(out + 8 * q8));
    }
  }
}

// Whether a wave takes a token by itself.  Four waves have a token's heads in flight at
// once, one wave takes them a few at a time but wastes no lanes, and forms the sines once in
// as many waves: it wins where tokens are many and their heads few.  In lanes of a token's
// heads (16 a head of 128, 8 a head of 64), one wave and four, us: 48 lanes, 1,000 tokens 3.8
// and 4.2, 16,384 12.9 and 20.4; 128 lanes, 1,000 4.9 and 4.5, 2,000 5.9 and 6.0, 16,384 19
// and 27; 256 lanes, 2,000 8.0 and 7.0, 4,000 11.4 and 11.5, 16,384 29 and 38; 512 lanes,
// 4,000 19.1 and 17.5, 8,192 30.2 and 31.7; 768 lanes, 8,192 45.0 and 45.2, 16,384 88.5 and
// 88.2; 1,280 lanes, 8,192 78 and 73, 16,384 152 and 151.  fp32: 128 lanes, 1,000 4.4 and
// 4.4, 16,384 30 and 39; 256 lanes, 1,000 6.7 and 5.5, 4,000 16.4 and 17.0, 16,384 58 and 61;
// 384 lanes, 8,192 46 and 42, 16,384 89 and 82.
inline bool wave_a_token(const arbor_geom_t *g, int n_tokens) {
  const int64_t lanes = (int64_t)g->num_kv_heads * (g->q_per_kv + 2) * (g->head_dim / 8);
  return n_tokens >= 16 * lanes && lanes <= (g->dtype == ARBOR_BF16 ? 512 : 256);
}

}  // namespace

int launch_append(const arbor_geom_t *geom, const arbor_tree_t *tree, arbor_pool_t *pool,
                  int32_t layer, const arbor_append_t *a, int32_t n_tokens, int32_t *status,
                  hipStream_t stream) {
  if (n_tokens == 0) return ARBOR_OK;
  const AppendArgs args{make_pool(geom, pool), *a, tree->num_tokens, layer, n_tokens, status};
  const bool many = wave_a_token(geom, n_tokens);
#define ARBOR_APPEND_WHOLE(T, D, HALVES)                                                         \
  do {                                                                                           \
    if (many)                                                                                    \
      hipLaunchKernelGGL((append_whole<T, D, HALVES, 64>), dim3(n_tokens), dim3(64), 0, stream,  \
                         args);                                                                  \
    else                                                                                         \
      hipLaunchKernelGGL((append_whole<T, D, HALVES, 256>), dim3(n_tokens), dim3(256), 0,        \
                         stream, args);                                                          \
  } while (0)
#define ARBOR_APPEND_LAUNCH(T, D)                                                                \
  do {                                                                                           \
    if (a->interleaved || a->rotary_dim == 0)                                                    \
      ARBOR_APPEND_WHOLE(T, D, false);                                                           \
    else if (a->rotary_dim == geom->head_dim)                                                    \
      ARBOR_APPEND_WHOLE(T, D, true);                                                            \
    else                                                                                         \
      hipLaunchKernelGGL((append_rows<T, D>), dim3(n_tokens), dim3(256), 0, stream, args);       \
  } while (0)
  if (geom->dtype == ARBOR_BF16) {
    if (geom->head_dim == 128) ARBOR_APPEND_LAUNCH(__bf16, 128);
    else ARBOR_APPEND_LAUNCH(__bf16, 64);
  } else {
    if (geom->head_dim == 128) ARBOR_APPEND_LAUNCH(float, 128);
    else ARBOR_APPEND_LAUNCH(float, 64);
  }
#undef ARBOR_APPEND_LAUNCH
#undef ARBOR_APPEND_WHOLE
  return hip_ok(hipGetLastError());
}

}  // namespace arbor
