// Queries and keys of a projection, each head normalised and rotated, with the tree rows' keys and
// values written into the cache: y = x / sqrt(mean(x^2) + eps) * gain over a head's dims, then the
// rotation of (y_i, y_{i + hd/2}) by position * base^(-2i/hd), in one pass over the projection.
//
// Memory bound (the projection read once, rotated queries, keys and values written once); with few
// rows the chain of loads.  A lane holds 8 dims of a head's lower half and their partners in the
// upper half, so that a pair never crosses lanes and the sum of squares is 3 lane swaps (2 for
// head dim 64).  A workgroup takes some rows of a session and some of the heads: angles are
// evaluated in 64 bits once a row and frequency, kept in LDS and used for all its heads (a row's
// hd / 2 sines in double cost as much as some 10 heads' loads).
#include "common.h"

namespace {

constexpr int QT = 256;       // threads
constexpr int QROWS = 16;     // rows of a session in a workgroup, at most

template <typename T> AS_DEVICE void load8(float (&x)[8], const T *p) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  const t8 v = *(const t8 *)p;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = to_f32<T>(v[e]);
}
template <typename T> AS_DEVICE void store8(T *p, const float (&x)[8]) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  t8 v;
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = from_f32<T>(x[e]);
  *(t8 *)p = v;
}
// the k-slices of a product, summed in order
template <typename T> AS_DEVICE void load_slices(float (&x)[8], const T *p, int nsl, size_t slice) {
  load8(x, p);
  for (int s = 1; s < nsl; ++s) {
    float y[8];
    load8(y, p + s * slice);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] += y[e];
  }
}

// grid: (groups of hpw heads out of H + 2 Hkv, chunks of rpw rows, sessions).  META: positions,
// slots and angles are there (meta, rot); else they follow from the parents.
template <typename TW, typename TIN, typename TQ, int HD, bool META>
__global__ __launch_bounds__(QT) void qk_norm_rope_kernel(
    const TIN *__restrict__ qkv, int nsl, const TW *__restrict__ q_gain,
    const TW *__restrict__ k_gain, float eps, const double *__restrict__ inv_freq, TreeMeta meta,
    const int32_t *__restrict__ parents, const int32_t *__restrict__ prefix_len, SharedArgs sh,
    int32_t *__restrict__ status, TQ *__restrict__ q_out, TW *__restrict__ ck,
    TW *__restrict__ cv, const float2 *__restrict__ rot, int n1, int H, int Hkv, int capacity,
    int hpw, int rpw) {
  constexpr int HALF = HD / 2, LPH = HD / 16;   // lanes a head
  __shared__ float2 s_rot[QROWS][HALF];
  __shared__ int s_par[128];
  const int b = blockIdx.z, r0 = blockIdx.y * rpw, nr = min(rpw, n1 - r0), tid = threadIdx.x;
  const int h0 = blockIdx.x * hpw, h1 = min(h0 + hpw, H + 2 * Hkv);
  const size_t row0 = (size_t)b * n1 + r0, W = (size_t)(H + 2 * Hkv) * HD;
  const size_t slice = W * n1 * gridDim.z;
  int S;
  if (META) {
    S = meta.sess_S[b];
    for (int e = tid; e < nr * HALF; e += QT)
      s_rot[e / HALF][e % HALF] = rot[(row0 + e / HALF) * HALF + e % HALF];
  } else {
    S = prefix_len[b];
    int front = 0;
    bool ok = S >= 0 && S <= (long long)capacity - n1;
    if (sh.of) {
      const int p = sh.of[b];
      const bool in = p >= 0 && p < sh.P;
      if (in) front = sh.len[p];
      ok = ok && (in || p == -1) && front >= 0 && front <= sh.cap;
      front = min(max(front, 0), sh.cap);
    }
    const int pr = tid < n1 ? parents[(size_t)b * n1 + tid] : 0;
    if (tid < n1) s_par[tid] = pr;
    ok = __syncthreads_and(ok && (tid >= n1 || (tid == 0 ? pr == -1 : pr >= 0 && pr < tid)));
    if (blockIdx.x == 0 && blockIdx.y == 0 && tid == 0)
      status[b] = ok ? ACESPEC_OK : ACESPEC_EBADTREE;
    if (!ok) return;   // nothing of the session is written
    for (int e = tid; e < nr * HALF; e += QT) {
      const int r = e / HALF, i = e % HALF;
      int depth = 0;
      for (int j = r0 + r; j > 0; j = s_par[j]) ++depth;
      double sd, cd;
      sincos((double)(front + S + depth) * inv_freq[i], &sd, &cd);
      s_rot[r][i] = make_float2((float)cd, (float)sd);
    }
  }
  __syncthreads();
  // queries and keys: LPH lanes a (row, head), heads next to each other
  const int hq = min(h1, H + Hkv) - h0;
  const int l8 = tid % LPH * 8;
  for (int e = tid / LPH; e < nr * hq; e += QT / LPH) {   // (whole groups of LPH lanes)
    const int r = e / hq, h = h0 + e - r * hq;
    const TIN *src = qkv + (row0 + r) * W + (size_t)h * HD + l8;
    float a[8], c[8];
    load_slices(a, src, nsl, slice);
    load_slices(c, src + HALF, nsl, slice);
    const TW *gain = h < H ? q_gain : k_gain;
    if (gain) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += a[i] * a[i] + c[i] * c[i];
#pragma unroll
      for (int x = 1; x < LPH; x <<= 1) ss += __shfl_xor(ss, x);
      const float inv = 1.0f / sqrtf(ss / (float)HD + eps);
      float ga[8], gc[8];
      load8(ga, gain + l8);
      load8(gc, gain + HALF + l8);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a[i] = a[i] * inv * ga[i];
        c[i] = c[i] * inv * gc[i];
      }
    }
    float y1[8], y2[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 cs = s_rot[r][l8 + i];
      y1[i] = a[i] * cs.x - c[i] * cs.y;
      y2[i] = c[i] * cs.x + a[i] * cs.y;
    }
    if (h < H) {
      TQ *dst = q_out + ((row0 + r) * H + h) * HD + l8;
      store8(dst, y1);
      store8(dst + HALF, y2);
    } else {
      TW *dst = ck + (((size_t)b * Hkv + h - H) * capacity + S + r0 + r) * HD + l8;
      store8(dst, y1);
      store8(dst + HALF, y2);
    }
  }
  // values: rows next to each other, so that a wave's two-byte stores are runs of slots
  const int v0 = max(h0, H + Hkv), hv = h1 - v0;
  const int pr2 = nr > 8 ? 16 : nr > 4 ? 8 : nr > 2 ? 4 : nr > 1 ? 2 : 1;   // lanes a column of rows
  for (int e = tid; e < hv * (HD / 8) * pr2; e += QT) {
    const int r = e % pr2, x = e / pr2, d = x % (HD / 8) * 8, h = v0 + x / (HD / 8);
    if (r >= nr) continue;
    float v[8];
    load_slices(v, qkv + (row0 + r) * W + (size_t)h * HD + d, nsl, slice);
    TW *dst = cv + (((size_t)b * Hkv + h - H - Hkv) * HD + d) * capacity + S + r0 + r;
#pragma unroll
    for (int i = 0; i < 8; ++i) dst[(size_t)i * capacity] = from_f32<TW>(v[i]);
  }
}

}  // namespace

namespace acespec {

template <typename TW, typename TIN, typename TQ>
hipError_t launch_qk_norm_rope(const TIN *qkv, int nsl, const TW *q_gain, const TW *k_gain,
                               float eps, const double *inv_freq, const TreeMeta &meta,
                               const int32_t *parents, const int32_t *prefix_len,
                               const SharedArgs &sh, int32_t *status, TQ *q_out, TW *ck, TW *cv,
                               const float2 *rot, int B, int n1, int H, int Hkv, int hd,
                               int capacity, hipStream_t s) {
  if ((hd != 64 && hd != 128) || H % Hkv || n1 > 65 || B > 65535) return hipErrorInvalidValue;
  const int chunks = (n1 + QROWS - 1) / QROWS, rpw = (n1 + chunks - 1) / chunks;
  const int heads = H + 2 * Hkv, groups = (heads + 11) / 12, hpw = (heads + groups - 1) / groups;
  const dim3 grid((heads + hpw - 1) / hpw, chunks, B);
  auto kernel = parents ? (hd == 64 ? qk_norm_rope_kernel<TW, TIN, TQ, 64, false>
                                    : qk_norm_rope_kernel<TW, TIN, TQ, 128, false>)
                        : (hd == 64 ? qk_norm_rope_kernel<TW, TIN, TQ, 64, true>
                                    : qk_norm_rope_kernel<TW, TIN, TQ, 128, true>);
  hipLaunchKernelGGL(kernel, grid, dim3(QT), 0, s, qkv, nsl, q_gain, k_gain, eps, inv_freq, meta,
                     parents, prefix_len, sh, status, q_out, ck, cv, rot, n1, H, Hkv, capacity, hpw,
                     rpw);
  return hipGetLastError();
}

#define QK_NORM(TW, TIN, TQ)                                                                    \
  template hipError_t launch_qk_norm_rope<TW, TIN, TQ>(                                         \
      const TIN *, int, const TW *, const TW *, float, const double *, const TreeMeta &,        \
      const int32_t *, const int32_t *, const SharedArgs &, int32_t *, TQ *, TW *, TW *,        \
      const float2 *, int, int, int, int, int, int, hipStream_t);
QK_NORM(bf16, bf16, bf16)
QK_NORM(bf16, float, f16)
QK_NORM(float, float, float)
#undef QK_NORM

}  // namespace acespec
