// arbor_append: norm of each query and key head, rotation by position, and the K/V
// rows of new tokens into the paged pool, in one pass over the projections.
//
// A workgroup takes one token.  Its angles are formed once, in 64 bits (a far
// position times a frequency does not fit 24 bits of mantissa: at position 10^5 an
// fp32 angle is off by up to 4e-3), reduced by whole turns, and their sines and
// cosines shared through LDS; then every group of D / 8 lanes takes one head, eight
// elements a lane, as two pieces of four such that the pairs (a, b) of the rotation
// lie in one lane: pieces 4 q and rotary_dim / 2 + 4 q of a half-split head, 8 q and
// 8 q + 4 otherwise.  The sum of squares crosses the lanes by DPP; nothing but the
// angles goes through LDS, and each element is read and written once: HBM-bound.
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
template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
  v += dpp_move<dpp::kQuadXor1>(v);
  v += dpp_move<dpp::kQuadXor2>(v);
  v += dpp_move<dpp::kRowHalfMirror>(v);
  if constexpr (LPR == 16) v += dpp_move<dpp::kRowMirror>(v);
  return v;
}

template <class T, int D>
__global__ __launch_bounds__(256) void append_rows(AppendArgs args) {
  constexpr int LPR = D / 8;                    // lanes of a head
  constexpr int RPS = 256 / LPR;                // heads a step
  constexpr int UNROLL = 4;                     // steps whose loads are in flight together
  typedef typename Piece<T>::reg reg;
  __shared__ float sh_cos[D / 2], sh_sin[D / 2];
  const arbor_append_t &a = args.a;
  const Pool &pl = args.pl;
  if (status_failed(args.status)) return;
  const int64_t t = blockIdx.x;
  const int64_t slot = a.slots[t];
  if (slot == -1) return;
  const int64_t rec = a.record_k ? a.tokens[t] : 0;
  if (slot < 0 || slot >= pl.num_pages * pl.P || rec < 0 ||
      (a.record_k && rec >= args.num_tokens)) {
    if (threadIdx.x == 0) status_error(args.status, ARBOR_EINVAL);
    return;
  }
  const int tid = threadIdx.x, q8 = tid % LPR;
  const int rd = a.rotary_dim, half = rd / 2;
  const bool split = !a.interleaved && q8 < rd / 8;    // this lane's pieces lie half apart
  const int ca = split ? 4 * q8 : 8 * q8, cb = split ? half + 4 * q8 : 8 * q8 + 4;
  const bool turns = q8 < rd / 8;
  const int Hq = pl.Hkv * pl.G, heads = Hq + 2 * pl.Hkv;
  auto row_of = [&](int h) -> const T * {
    const T *p = static_cast<const T *>(h < Hq ? a.q : h < Hq + pl.Hkv ? a.k : a.v);
    const int64_t stride = h < Hq ? a.q_stride : h < Hq + pl.Hkv ? a.k_stride : a.v_stride;
    const int hh = h < Hq ? h : h < Hq + pl.Hkv ? h - Hq : h - Hq - pl.Hkv;
    return p + t * stride + (int64_t)hh * D;
  };
  // the first heads' loads are on their way while the angles are formed
  reg xa[UNROLL], xb[UNROLL];
  auto load = [&](int h0) {
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int h = h0 + u * RPS;
      if (h < heads) {
        const T *p = row_of(h);
        xa[u] = *reinterpret_cast<const reg *>(p + ca);
        xb[u] = *reinterpret_cast<const reg *>(p + cb);
      }
    }
  };
  int h0 = tid / LPR;
  load(h0);
  if (rd > 0) {
    if (tid < half) {
      // in turns: x = pos f / (2 pi) in fp64 is off by 2^-53 relative, 1e-10 turns
      // at position 10^6, and its fraction is exact
      const double x = (double)a.positions[t] * (double)a.inv_freq[tid] * 0.15915494309189535;
      const float f = (float)(x - rint(x)) * 2.0f;       // half turns, in [-1, 1]
      float s, c;
      sincospif(f, &s, &c);
      sh_cos[tid] = c;
      sh_sin[tid] = s;
    }
    __syncthreads();
  }
  // elements (a, b) of pair e of this lane: split (xa[e], xb[e]); otherwise
  // (xa[0], xa[1]), (xa[2], xa[3]), (xb[0], xb[1]), (xb[2], xb[3]): pair 4 q8 + e either way
  float co[4], si[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    co[e] = turns ? sh_cos[4 * q8 + e] : 1.0f;
    si[e] = turns ? sh_sin[4 * q8 + e] : 0.0f;
  }
  const int64_t page = slot / pl.P, row = slot % pl.P;
  for (; h0 < heads; h0 += UNROLL * RPS) {
    if (h0 >= UNROLL * RPS) load(h0);
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
        if (w) {
          float ss = 0.0f;
#pragma unroll
          for (int e = 0; e < 4; ++e) ss += va[e] * va[e] + vb[e] * vb[e];
          ss = row_sum<LPR>(ss);
          const float r = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
          const reg wa = *reinterpret_cast<const reg *>(static_cast<const T *>(w) + ca);
          const reg wb = *reinterpret_cast<const reg *>(static_cast<const T *>(w) + cb);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            va[e] *= r * (float)wa[e];
            vb[e] *= r * (float)wb[e];
          }
        }
        if (split) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ya[e] = (T)(va[e] * co[e] - vb[e] * si[e]);
            yb[e] = (T)(vb[e] * co[e] + va[e] * si[e]);
          }
        } else if (turns) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            ya[2 * e] = (T)(va[2 * e] * co[e] - va[2 * e + 1] * si[e]);
            ya[2 * e + 1] = (T)(va[2 * e + 1] * co[e] + va[2 * e] * si[e]);
            yb[2 * e] = (T)(vb[2 * e] * co[2 + e] - vb[2 * e + 1] * si[2 + e]);
            yb[2 * e + 1] = (T)(vb[2 * e + 1] * co[2 + e] + vb[2 * e] * si[2 + e]);
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            ya[e] = (T)va[e];
            yb[e] = (T)vb[e];
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
                 ((rec * pl.L + args.layer) * pl.Hkv + g) * D;
          *reinterpret_cast<reg *>(r + ca) = ya;
          *reinterpret_cast<reg *>(r + cb) = yb;
        }
      }
      *reinterpret_cast<reg *>(out + ca) = ya;
      *reinterpret_cast<reg *>(out + cb) = yb;
    }
  }
}

}  // namespace

int launch_append(const arbor_geom_t *geom, const arbor_tree_t *tree, arbor_pool_t *pool,
                  int32_t layer, const arbor_append_t *a, int32_t n_tokens, int32_t *status,
                  hipStream_t stream) {
  if (n_tokens == 0) return ARBOR_OK;
  const AppendArgs args{make_pool(geom, pool), *a, tree->num_tokens, layer, n_tokens, status};
#define ARBOR_APPEND_LAUNCH(T, D) \
  hipLaunchKernelGGL((append_rows<T, D>), dim3(n_tokens), dim3(256), 0, stream, args)
  if (geom->dtype == ARBOR_BF16) {
    if (geom->head_dim == 128) ARBOR_APPEND_LAUNCH(__bf16, 128);
    else ARBOR_APPEND_LAUNCH(__bf16, 64);
  } else {
    if (geom->head_dim == 128) ARBOR_APPEND_LAUNCH(float, 128);
    else ARBOR_APPEND_LAUNCH(float, 64);
  }
#undef ARBOR_APPEND_LAUNCH
  return hip_ok(hipGetLastError());
}

}  // namespace arbor
