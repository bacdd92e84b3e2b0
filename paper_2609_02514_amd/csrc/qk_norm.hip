// Queries and keys of a projection, each head normalised and rotated, with the tree rows' keys and
// values written into the cache: y = x / sqrt(mean(x^2) + eps) * gain over a head's dims, then the
// rotation of (y_i, y_{i + hd/2}) by position * base^(-2i/hd), in one pass over the projection.
//
// Bound by the chain of loads (the projection read once, rotated queries, keys and values written once:
// 64 sessions of 17 rows, 32 query and 8 kv heads of 128 dims 11 us, where the bytes alone take 4: 9
// rows of 8 heads are 576 lanes' work for a workgroup of 256, three rounds of which each asks for its
// loads when the one before is computed; one row 4.2).  A lane holds 8 dims of a head's lower half and their partners in the
// upper half, so that a pair never crosses lanes and the sum of squares is 3 lane swaps (2 for
// head dim 64).  A workgroup takes some rows of a session and some query and key heads, whose loads
// are under way while it evaluates the rows' angles; or one value head of a session.
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

// cos and sin of pos * freq: the product and its distance from a multiple of 2 pi in 64 bits (a
// position times a frequency of 1 loses 2 pi's fraction in 32), the functions in 32 on that
// distance's upper part, its lower one to first order.  Off by 2^-23; sines in double took as long
// as ten heads' loads.
AS_DEVICE float2 cos_sin(int pos, double freq) {
  constexpr double TWO_PI = 6.283185307179586, TWO_PI_LOW = 2.4492935982947064e-16;
  const double x = (double)pos * freq, n = rint(x * (1 / TWO_PI));
  const double r = fma(-n, TWO_PI_LOW, fma(-n, TWO_PI, x));
  const float hi = (float)r, lo = (float)(r - (double)hi);
  float s, c;
  sincosf(hi, &s, &c);
  return make_float2(fmaf(-lo, s, c), fmaf(lo, c, s));
}

// grid: (groups of hpw heads out of H + Hkv for each of `chunks` chunks of rpw rows, then the value
// heads; sessions).  META: positions, slots and angles are there (meta, rot); else they follow from
// the parents.
template <typename TW, typename TIN, typename TQ, int HD, bool META>
__global__ __launch_bounds__(QT) void qk_norm_rope_kernel(
    const TIN *__restrict__ qkv, int nsl, const TW *__restrict__ q_gain,
    const TW *__restrict__ k_gain, float eps, const double *__restrict__ inv_freq, TreeMeta meta,
    const int32_t *__restrict__ parents, const int32_t *__restrict__ prefix_len, SharedArgs sh,
    int32_t *__restrict__ status, TQ *__restrict__ q_out, TW *__restrict__ ck,
    TW *__restrict__ cv, const float2 *__restrict__ rot, int n1, int H, int Hkv, int capacity,
    int hpw, int rpw, int chunks, int groups) {
  constexpr int HALF = HD / 2, LPH = HD / 16;   // lanes a head
  __shared__ float2 s_rot[QROWS][HALF + 1];
  __shared__ int s_par[128];
  const int b = blockIdx.y, x = blockIdx.x, tid = threadIdx.x;
  const bool values = x >= groups * chunks;
  const int chunk = values ? 0 : x / groups;
  const int r0 = chunk * rpw, nr = values ? n1 : min(rpw, n1 - r0);
  const int h0 = (x - chunk * groups) * hpw, hq = values ? 0 : min(hpw, H + Hkv - h0);
  const size_t row0 = (size_t)b * n1 + r0, W = (size_t)(H + 2 * Hkv) * HD;
  const size_t slice = W * n1 * gridDim.y;
  const TIN *rows = qkv + row0 * W;

  // queries and keys: LPH lanes a (row, head), heads next to each other; the first ones' loads go
  // out before anything else is known
  const int l8 = tid % LPH * 8, e0 = tid / LPH, tasks = nr * hq;
  float a[8], c[8];
  auto load = [&](int e) {
    const int r = e / hq, h = h0 + e - r * hq;
    const TIN *src = rows + r * W + (size_t)h * HD + l8;
    load_slices(a, src, nsl, slice);
    load_slices(c, src + HALF, nsl, slice);
  };
  if (e0 < tasks) load(e0);

  int S;
  if (META) {
    S = meta.sess_S[b];
    if (!values)
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
    }
    const int pr = tid < n1 ? parents[(size_t)b * n1 + tid] : 0;
    if (tid < n1) s_par[tid] = pr;
    ok = __syncthreads_and(ok && (tid >= n1 || (tid == 0 ? pr == -1 : pr >= 0 && pr < tid)));
    if (x == 0 && tid == 0) status[b] = ok ? ACESPEC_OK : ACESPEC_EBADTREE;
    if (!ok) return;   // nothing of the session is written
    if (!values)
      for (int e = tid; e < nr * HALF; e += QT) {
        const int r = e / HALF, i = e % HALF;
        int depth = 0;
        for (int j = r0 + r; j > 0; j = s_par[j]) ++depth;
        s_rot[r][i] = cos_sin(front + S + depth, inv_freq[i]);
      }
  }
  if (values) {
    // rows next to each other, so that a wave's two-byte stores are runs of slots
    const int g = x - groups * chunks;
    const TIN *src = rows + (size_t)(H + Hkv + g) * HD;
    TW *dst = cv + ((size_t)b * Hkv + g) * HD * capacity + S;
#pragma unroll 2
    for (int e = tid; e < n1 * (HD / 8); e += QT) {
      const int p = e / n1, r = e - p * n1;
      float v[8];
      load_slices(v, src + r * W + p * 8, nsl, slice);
#pragma unroll
      for (int i = 0; i < 8; ++i) dst[(size_t)(p * 8 + i) * capacity + r] = from_f32<TW>(v[i]);
    }
    return;
  }
  __syncthreads();
  for (int e = e0; e < tasks;) {   // (whole groups of LPH lanes)
    const int r = e / hq, h = h0 + e - r * hq;
    const TW *gain = h < H ? q_gain : k_gain;
    if (gain) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss += a[i] * a[i] + c[i] * c[i];
#pragma unroll
      for (int o = 1; o < LPH; o <<= 1) ss += __shfl_xor(ss, o);
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
    e += QT / LPH;
    if (e < tasks) load(e);
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
  const int heads = H + Hkv, hpw = heads < 8 ? heads : 8, groups = (heads + hpw - 1) / hpw;
  const dim3 grid(groups * chunks + Hkv, B);
  auto kernel = parents ? (hd == 64 ? qk_norm_rope_kernel<TW, TIN, TQ, 64, false>
                                    : qk_norm_rope_kernel<TW, TIN, TQ, 128, false>)
                        : (hd == 64 ? qk_norm_rope_kernel<TW, TIN, TQ, 64, true>
                                    : qk_norm_rope_kernel<TW, TIN, TQ, 128, true>);
  hipLaunchKernelGGL(kernel, grid, dim3(QT), 0, s, qkv, nsl, q_gain, k_gain, eps, inv_freq, meta,
                     parents, prefix_len, sh, status, q_out, ck, cv, rot, n1, H, Hkv, capacity, hpw,
                     rpw, chunks, groups);
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
