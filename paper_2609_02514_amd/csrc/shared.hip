// Moves between caches: a session's first slots into the store of shared prefixes, and sessions
// that take over another session's slots.
//
// Both are copies, bound by memory (a take-over of 8 layers of two prefixes of up to 8192 slots 112 us,
// 468 MB past the caches; sixteen sessions that go on four's up to 2048 slots 213, 886 MB).  The store keeps records of 64 slots in the order in which the
// attention over them multiplies (fp16 for a bf16 model: the values that the products take anyway),
// so that a prefix is brought into that order once and read by every step from then on.
#include "common.h"

namespace {

constexpr int ST = 256;   // threads
// Past the caches, for what is not touched again here (6.4 TB/s against the 5.0 of plain copies).
template <typename P> AS_DEVICE P ld_nt(const P *p) { return __builtin_nontemporal_load(p); }
template <typename P> AS_DEVICE void st_nt(P *p, P x) { __builtin_nontemporal_store(x, p); }

// One workgroup a record.  grid: records x prefixes x (layer, kv head), records fastest.
template <typename T, int HD>
__global__ __launch_bounds__(ST) void share_kernel(const T *__restrict__ k, const T *__restrict__ v,
                                                   const int32_t *__restrict__ prefix_len, int B,
                                                   int cap, void *__restrict__ blocks, SharedArgs sh,
                                                   const int32_t *__restrict__ from,
                                                   const int32_t *__restrict__ count,
                                                   int32_t *__restrict__ new_len, int Hkv) {
  constexpr int REC = 128 * HD;
  const int nblk = sh.cap >> 6;
  const long long item = blockIdx.x / nblk;
  const int c = (int)(blockIdx.x - item * nblk), p = (int)(item % sh.P), lg = (int)(item / sh.P);
  const int l = lg / Hkv, g = lg - l * Hkv, tid = threadIdx.x;
  const int src = from[p];
  int n = -1;
  if (src >= 0 && src < B) {
    const int len = prefix_len[src];
    n = count ? count[p] : len;
    if (len < 0 || len > cap || n < 0 || n > len || n > sh.cap) n = -1;
  }
  if (lg == 0 && c == 0 && tid == 0) new_len[p] = src == -1 ? sh.len[p] : n;
  if (c * 64 >= n) return;
  const size_t plane = ((size_t)l * B + src) * Hkv + g;
  const T *kp = k + (plane * cap + c * 64) * HD, *vp = v + plane * HD * cap + c * 64;
  const size_t rec = (((size_t)l * sh.P + p) * Hkv + g) * nblk + c;
  const int valid = min(64, n - c * 64);
  constexpr int PE = 16 / sizeof(T);
  typedef T piece __attribute__((ext_vector_type(PE)));
  if constexpr (sizeof(T) == 4) {
    float *dst = (float *)blocks + rec * REC;
    for (int e = tid; e < 64 * HD / PE; e += ST) {
      const int slot = e / (HD / PE);
      piece x{};
      if (slot < valid) x = ld_nt((const piece *)(kp + (size_t)e * PE));
      st_nt((piece *)(dst + e * PE), x);
    }
    for (int e = tid; e < 64 * HD / PE; e += ST) {
      const int d = e / (64 / PE), s0 = e % (64 / PE) * PE;
      piece x{};
      if (s0 < valid) x = ld_nt((const piece *)(vp + (size_t)d * cap + s0));
#pragma unroll
      for (int i = 0; i < PE; ++i)
        if (s0 + i >= valid) x[i] = 0.f;
      st_nt((piece *)(dst + REC / 2 + e * PE), x);
    }
  } else {
    // read in the cache's order and written in the record's, both in whole lines, through LDS
    __shared__ __attribute__((aligned(16))) f16 rec_s[REC];
#pragma unroll 4
    for (int e = tid; e < 64 * HD / 8; e += ST) {
      const int slot = e / (HD / 8), d8 = e % (HD / 8);
      f16x8 x{};
      if (slot < valid) x = bf16x8_to_f16x8(ld_nt((const bf16x8 *)(kp + (size_t)e * 8)));
      // row r of a 32 x 32 operand holds slot 16 r4 + 8 r2 + 4 r3 + r10 of its half
      const int lane = (d8 & 1) * 32 + (slot & 16) + ((slot >> 3) & 1) * 4 + ((slot >> 2) & 1) * 8 + (slot & 3);
      *(f16x8 *)(rec_s + (((slot >> 5) * (HD / 16) + (d8 >> 1)) * 64 + lane) * 8) = x;
    }
#pragma unroll 4
    for (int e = tid; e < 64 * HD / 8; e += ST) {
      const int d = e >> 3, s8 = e & 7;
      f16x8 x{};
      if (s8 * 8 < valid) x = bf16x8_to_f16x8(ld_nt((const bf16x8 *)(vp + (size_t)d * cap + s8 * 8)));
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (s8 * 8 + i >= valid) x[i] = (f16)0.f;
      const int lane = (s8 & 1) * 32 + (d & 31);
      *(f16x8 *)(rec_s + REC / 2 + (((s8 >> 1) * (HD / 32) + (d >> 5)) * 64 + lane) * 8) = x;
    }
    __syncthreads();
    f16 *dst = (f16 *)blocks + rec * REC;
#pragma unroll 4
    for (int e = tid; e < REC / 8; e += ST) st_nt((f16x8 *)(dst + e * 8), *(const f16x8 *)(rec_s + e * 8));
  }
}

// 16 bytes at any element's address
template <typename T> AS_DEVICE u32x4 load_any(const T *p) {
  struct __attribute__((packed, aligned(sizeof(T)))) U { u32x4 x; };
  return ((const U *)p)->x;
}

// One workgroup takes FCH slots of a plane (layer, kv head) of a source: read once, written for all
// the sessions that take over from it (16 rows from 4 sources, 0.78 GB written: a workgroup a session
// 232 us, the source read again through L2, this 213).  The first of these sessions' workgroup does
// it, the others leave.
constexpr int FCH = acespec::kForkSlots;
template <typename T, int HD>
__global__ __launch_bounds__(ST) void fork_kernel(const T *__restrict__ sk, const T *__restrict__ sv,
                                                  const int32_t *__restrict__ src_len, int Bs,
                                                  int scap, T *dk, T *dv,
                                                  const int32_t *__restrict__ dst_len, int Bd,
                                                  int dcap, const int32_t *__restrict__ from,
                                                  const int32_t *__restrict__ first,
                                                  int32_t *__restrict__ new_len, int Hkv,
                                                  int chunks, int same) {
  constexpr int PE = 16 / sizeof(T), NP = FCH * HD / PE / ST, VR = FCH / PE;   // pieces a thread, a value row
  // (neighbours on one XCD: dealt round-robin, the first sessions of 16 fell on four of the eight)
  const int id = xcd_tile(blockIdx.x, gridDim.x), b = id % Bd, rest = id / Bd;
  const int c = rest % chunks, lg = rest / chunks, l = lg / Hkv, g = lg - l * Hkv;
  const int tid = threadIdx.x, lane = tid & 63;
  const int src = from[b], lo = c * FCH;
  const bool there = src >= 0 && src < Bs;
  const int len = there ? src_len[src] : -1;
  // (a session that receives slots itself is no source)
  const int up = there && same ? from[src] : -1;
  const bool source = there && len >= 0 && len <= scap && (up == -1 || up == src);
  // slots of session d and where they begin, -1: refused
  auto slots = [&](int d, int *x0) {
    *x0 = first ? first[d] : 0;
    if (same && d == src) return *x0 == 0 ? len : -1;
    return source && *x0 >= 0 && *x0 <= len && len - *x0 <= dcap ? len - *x0 : -1;
  };
  if (lg == 0 && c == 0 && tid == 0) {
    int x0;
    new_len[b] = src == -1 ? dst_len[b] : there && len >= 0 && len <= scap ? slots(b, &x0) : -1;
  }
  if (!source || lo >= len) return;
  u32x4 kx[NP], vx[NP];
  int held = -1;   // the offset whose slots are in kx, vx
  for (int d0 = 0; d0 < Bd; d0 += 64) {
    const int f = d0 + lane < Bd ? from[d0 + lane] : -1;
    for (uint64_t rest = __ballot(f == src); rest; rest &= rest - 1) {
      const int d = d0 + __builtin_ctzll(rest);
      if (d < b) return;   // another session's workgroup is the first
      int x0;
      const int n = slots(d, &x0), m = min(FCH, n - lo);
      if (m <= 0 || (same && d == src)) continue;
      const size_t sp = ((size_t)l * Bs + src) * Hkv + g, dp = ((size_t)l * Bd + d) * Hkv + g;
      const T *ks = sk + (sp * scap + x0 + lo) * HD, *vs = sv + sp * HD * scap + x0 + lo;
      T *kd = dk + (dp * dcap + lo) * HD, *vd = dv + dp * HD * dcap + lo;
      const int kp = m * (HD / PE), full = m / PE;   // pieces of keys, whole ones of a value row
      if (x0 != held) {
        held = x0;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int e = tid + i * ST;
          if (e < kp) kx[i] = ((const u32x4 *)ks)[e];
          if (e % VR < full) vx[i] = load_any(vs + (size_t)(e / VR) * scap + e % VR * PE);
        }
      }
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int e = tid + i * ST;
        if (e < kp) st_nt((u32x4 *)kd + e, kx[i]);
        if (e % VR < full) st_nt((u32x4 *)(vd + (size_t)(e / VR) * dcap + e % VR * PE), vx[i]);
      }
      if (m % PE)   // the last, broken piece of each value row
        for (int e = tid; e < HD * (m % PE); e += ST) {
          const int r = e / (m % PE), j = full * PE + e % (m % PE);
          vd[(size_t)r * dcap + j] = vs[(size_t)r * scap + j];
        }
    }
  }
}

}  // namespace

namespace acespec {

template <typename T>
hipError_t launch_share_prefix(const T *k, const T *v, const int32_t *prefix_len, int B, int cap,
                               void *blocks, const SharedArgs &sh, const int32_t *from,
                               const int32_t *count, int32_t *new_len, int L, int Hkv, int hd,
                               hipStream_t s) {
  const long long wgs = (long long)L * Hkv * sh.P * (sh.cap / 64);
  if ((hd != 64 && hd != 128) || wgs > 0xffffffffLL / ST) return hipErrorInvalidValue;
  auto kernel = hd == 64 ? share_kernel<T, 64> : share_kernel<T, 128>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(ST), 0, s, k, v, prefix_len, B, cap, blocks, sh,
                     from, count, new_len, Hkv);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_fork_kv(const T *sk, const T *sv, const int32_t *src_len, int Bs, int scap, T *dk,
                          T *dv, const int32_t *dst_len, int Bd, int dcap, const int32_t *from,
                          const int32_t *first, int32_t *new_len, int L, int Hkv, int hd,
                          hipStream_t s) {
  const int chunks = ((scap < dcap ? scap : dcap) + FCH - 1) / FCH;
  const long long wgs = fork_workgroups(L, Hkv, Bd, scap, dcap);
  if ((hd != 64 && hd != 128) || wgs > 0xffffffffLL / ST) return hipErrorInvalidValue;
  const int same = sk == dk && sv == dv;
  auto kernel = hd == 64 ? fork_kernel<T, 64> : fork_kernel<T, 128>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(ST), 0, s, sk, sv, src_len, Bs, scap, dk, dv,
                     dst_len, Bd, dcap, from, first, new_len, Hkv, chunks, same);
  return hipGetLastError();
}

#define MOVES(T)                                                                                   \
  template hipError_t launch_share_prefix<T>(const T *, const T *, const int32_t *, int, int,      \
                                             void *, const SharedArgs &, const int32_t *,          \
                                             const int32_t *, int32_t *, int, int, int,            \
                                             hipStream_t);                                         \
  template hipError_t launch_fork_kv<T>(const T *, const T *, const int32_t *, int, int, T *, T *, \
                                        const int32_t *, int, int, const int32_t *,                \
                                        const int32_t *, int32_t *, int, int, int, hipStream_t);
MOVES(bf16)
MOVES(float)
#undef MOVES

}  // namespace acespec
