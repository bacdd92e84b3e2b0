// The 4-bit KV cache: a cache brought to 4 bits, read back, and the commit that brings the
// blocks of 32 slots to 4 bits as the verified path completes them.
//
// All three move bytes: what bounds them is HBM (or, for the commit's few rows, the chain of
// dependent reads before the first store).  A record is written by one wave, each lane from the
// 32 (head dim 64: 16) head dims of a key and the 8 slots of a value row that its operands hold,
// so a key group's maximum is the lane's own (head dim 64: of two lanes) and a value group's
// takes two swaps between lanes; nothing goes through LDS.
#include "quant.h"

namespace {

constexpr int QT = 256;   // threads: four waves

struct QuantDims {
  int B, Hkv, cap, qcap, tcap, ng;   // sessions, kv heads, capacities, workgroups a plane
};

// Whether a session of P slots fits the caches (P < 0: does not).
AS_DEVICE bool fits(int P, const QuantDims &d) {
  return P >= 0 && P <= d.cap && (P & ~(Q4_SLOTS - 1)) <= d.qcap;
}

// Workgroup blockIdx.x = plane * ng + i; a plane is (layer, session, kv head).  The waves of a
// plane's ng workgroups take its blocks in turn, from the one that holds slot first[b] on.  The
// block after the last complete one is the tail: copied as it is.
template <typename T, int HD>
__global__ __launch_bounds__(QT) void quantize_kernel(const T *__restrict__ k,
                                                      const T *__restrict__ v,
                                                      const int32_t *__restrict__ prefix_len,
                                                      const int32_t *__restrict__ first,
                                                      uint8_t *__restrict__ blocks,
                                                      T *__restrict__ tk, T *__restrict__ tv,
                                                      QuantDims d, int32_t *__restrict__ status) {
  const size_t plane = blockIdx.x / d.ng;
  const int grp = blockIdx.x - (int)plane * d.ng, lane = threadIdx.x & 63;
  const int b = (int)(plane / d.Hkv) % d.B;
  const int P = prefix_len[b], F = first ? first[b] : 0;
  const bool ok = fits(P, d) && F >= 0 && F <= P;
  if (status && grp == 0 && plane < (size_t)d.B * d.Hkv && plane % d.Hkv == 0 && threadIdx.x == 0)
    status[b] = ok ? ACESPEC_OK : ACESPEC_EBADTREE;
  if (!ok) return;
  const int full = P / Q4_SLOTS, t = P % Q4_SLOTS;
  const T *kp = k + plane * d.cap * HD, *vp = v + plane * HD * d.cap;
  for (int blk = F / Q4_SLOTS + grp * (QT / 64) + (threadIdx.x >> 6); blk <= full;
       blk += d.ng * (QT / 64)) {
    const int s0 = blk * Q4_SLOTS;
    if (blk < full) {
      q4_encode_block<T, HD>(kp + (size_t)s0 * HD, vp + s0, d.cap,
                             blocks + (plane * (d.qcap / Q4_SLOTS) + blk) * q4_bytes(HD), lane);
      continue;
    }
    T *kd = tk + plane * d.tcap * HD, *vd = tv + plane * HD * d.tcap;
    for (int e = lane; e < t * (HD / 8); e += 64) {
      float x[8];
      load8(kp + (size_t)s0 * HD + e * 8, x);
      store8(kd + e * 8, f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]});
    }
    const int slot = lane & (Q4_SLOTS - 1);
    if (slot < t)
      for (int r = lane >> 5; r < HD; r += 2)
        vd[(size_t)r * d.tcap + slot] = vp[(size_t)r * d.cap + s0 + slot];
  }
}

// The inverse, for slots [first[b] / 32 * 32, prefix_len[b]).
template <typename T, int HD>
__global__ __launch_bounds__(QT) void dequantize_kernel(const uint8_t *__restrict__ blocks,
                                                        const T *__restrict__ tk,
                                                        const T *__restrict__ tv,
                                                        const int32_t *__restrict__ prefix_len,
                                                        const int32_t *__restrict__ first,
                                                        T *__restrict__ k, T *__restrict__ v,
                                                        QuantDims d, int32_t *__restrict__ status) {
  constexpr int LD = HD / 4, NB = HD / 16;
  const size_t plane = blockIdx.x / d.ng;
  const int grp = blockIdx.x - (int)plane * d.ng, lane = threadIdx.x & 63;
  const int lr = lane & 15, lg = lane >> 4;
  const int b = (int)(plane / d.Hkv) % d.B;
  const int P = prefix_len[b], F = first ? first[b] : 0;
  const bool ok = fits(P, d) && F >= 0 && F <= P;
  if (status && grp == 0 && plane < (size_t)d.B * d.Hkv && plane % d.Hkv == 0 && threadIdx.x == 0)
    status[b] = ok ? ACESPEC_OK : ACESPEC_EBADTREE;
  if (!ok) return;
  const int full = P / Q4_SLOTS, t = P % Q4_SLOTS;
  T *kp = k + plane * d.cap * HD, *vp = v + plane * HD * d.cap;
  for (int blk = F / Q4_SLOTS + grp * (QT / 64) + (threadIdx.x >> 6); blk <= full;
       blk += d.ng * (QT / 64)) {
    const int s0 = blk * Q4_SLOTS;
    if (blk < full) {
      Q4Regs<HD> r;
      q4_load<HD>(r, blocks + (plane * (d.qcap / Q4_SLOTS) + blk) * q4_bytes(HD), lane);
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int j = 0; j < LD / 8; ++j)
          store8(kp + (size_t)(s0 + q4_key(kk, lr)) * HD + lg * LD + j * 8,
                 q4_decode_f32(q4_kword<HD>(r, kk, j), q4_kscale<HD>(r, kk)));
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
        store8(vp + (size_t)(nb * 16 + lr) * d.cap + s0 + lg * 8,
               q4_decode_f32(q4_vword<HD>(r, nb), q4_vscale<HD>(r, nb)));
      continue;
    }
    const T *ks = tk + plane * d.tcap * HD, *vs = tv + plane * HD * d.tcap;
    for (int e = lane; e < t * (HD / 8); e += 64) {
      float x[8];
      load8(ks + e * 8, x);
      store8(kp + (size_t)s0 * HD + e * 8, f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]});
    }
    const int slot = lane & (Q4_SLOTS - 1);
    if (slot < t)
      for (int r = lane >> 5; r < HD; r += 2)
        vp[(size_t)r * d.cap + s0 + slot] = vs[(size_t)r * d.tcap + slot];
  }
}

// Commit (Algorithm 1, COMPACT_KV).  With t = P % 32 the session's committed slots are the
// tail's [0, t], the root among them, and the kept rows t + path[i]: t + 1 + np slots in that
// order, of which every complete 32 become a record and the rest the tail's front.  One
// workgroup per plane.  All that moves goes through LDS first, as a destination may be another
// entry's source.
template <typename T, int HD>
__global__ __launch_bounds__(QT) void commit_quant_kernel(
    uint8_t *__restrict__ blocks, T *__restrict__ tk, T *__restrict__ tv,
    const int32_t *__restrict__ prefix_len, const int32_t *__restrict__ path,
    const int32_t *__restrict__ path_len, const int32_t *__restrict__ status, int n1,
    QuantDims d, int pitch, int32_t *__restrict__ new_len) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int src[96];                 // slot of the tail that committed slot i comes from
  const size_t plane = blockIdx.x;
  const int b = (int)(plane / d.Hkv) % d.B, tid = threadIdx.x;
  const int P = prefix_len[b], np = path_len[b];
  const int t = P & (Q4_SLOTS - 1), end = t + 1 + np, nblk = end / Q4_SLOTS;
  const bool ok = (status == nullptr || status[b] == ACESPEC_OK) && P >= 0 && np >= 0 && np < n1 &&
                  P / Q4_SLOTS + nblk <= d.qcap / Q4_SLOTS;
  const int32_t row = tid < n1 - 1 ? path[(size_t)b * n1 + tid] : 0;
  const bool bad = __syncthreads_or(!ok || (tid < np && (row < 1 || row >= n1)));
  if (plane < (size_t)d.B * d.Hkv && plane % d.Hkv == 0 && tid == 0) new_len[b] = bad ? -1 : P + 1 + np;
  if (bad) return;
  // What moves: from slot `lo` on (without a complete block only the kept rows do).
  const int lo = nblk ? 0 : t + 1;
  if (tid <= t) src[tid] = tid;
  if (tid < np) src[t + 1 + tid] = t + row;
  __syncthreads();
  T *kd = tk + plane * d.tcap * HD, *vd = tv + plane * HD * d.tcap;
  T *kx = (T *)smem, *vx = kx + (size_t)pitch * HD;   // [slot][HD], [HD][pitch]
  for (int e = tid; e < (end - lo) * (HD / 8); e += QT) {
    const int i = lo + e / (HD / 8), c = e % (HD / 8) * 8;
    float x[8];
    load8(kd + (size_t)src[i] * HD + c, x);
    store8(kx + i * HD + c, f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]});
  }
  for (int r = tid >> 5; r < HD; r += QT / 32)
    for (int i = lo + (tid & 31); i < end; i += 32) vx[r * pitch + i] = vd[(size_t)r * d.tcap + src[i]];
  __syncthreads();
  const int wave = tid >> 6;
  if (wave < nblk)
    q4_encode_block<T, HD>(kx + wave * Q4_SLOTS * HD, vx + wave * Q4_SLOTS, pitch,
                           blocks + (plane * (d.qcap / Q4_SLOTS) + P / Q4_SLOTS + wave) * q4_bytes(HD),
                           tid & 63);
  const int from = nblk ? nblk * Q4_SLOTS : lo, to = nblk ? 0 : lo;
  for (int e = tid; e < (end - from) * (HD / 8); e += QT) {
    const int i = e / (HD / 8), c = e % (HD / 8) * 8;
    float x[8];
    load8(kx + (from + i) * HD + c, x);
    store8(kd + (size_t)(to + i) * HD + c, f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]});
  }
  for (int r = tid >> 5; r < HD; r += QT / 32)
    for (int i = tid & 31; i < end - from; i += 32)
      vd[(size_t)r * d.tcap + to + i] = vx[r * pitch + from + i];
}

// Workgroups a plane: all its blocks' waves at once, but no more in all than keep every CU
// busy several times over (a read-back of a few slots would else launch a workgroup for every
// block of the capacity).
int groups_of(long long planes, int blocks) {
  const long long want = (32768 + planes - 1) / planes;
  const int most = (blocks + QT / 64 - 1) / (QT / 64);
  return want < most ? (int)want : most;
}

}  // namespace

namespace acespec {

template <typename T>
hipError_t launch_quantize_kv(const T *k, const T *v, const int32_t *prefix_len,
                              const int32_t *first, uint8_t *blocks, T *tk, T *tv, int L, int B,
                              int Hkv, int hd, int cap, int qcap, int tcap, int32_t *status,
                              hipStream_t s) {
  const long long planes = (long long)L * B * Hkv;
  const QuantDims d{B, Hkv, cap, qcap, tcap,
                    groups_of(planes, (cap < qcap + Q4_SLOTS ? cap : qcap + Q4_SLOTS) / Q4_SLOTS + 1)};
  auto kernel = hd == 64 ? quantize_kernel<T, 64> : quantize_kernel<T, 128>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(planes * d.ng)), dim3(QT), 0, s, k, v, prefix_len,
                     first, blocks, tk, tv, d, status);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_dequantize_kv(const uint8_t *blocks, const T *tk, const T *tv,
                                const int32_t *prefix_len, const int32_t *first, T *k, T *v,
                                int L, int B, int Hkv, int hd, int cap, int qcap, int tcap,
                                int32_t *status, hipStream_t s) {
  const long long planes = (long long)L * B * Hkv;
  const QuantDims d{B, Hkv, cap, qcap, tcap,
                    groups_of(planes, (cap < qcap + Q4_SLOTS ? cap : qcap + Q4_SLOTS) / Q4_SLOTS + 1)};
  auto kernel = hd == 64 ? dequantize_kernel<T, 64> : dequantize_kernel<T, 128>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(planes * d.ng)), dim3(QT), 0, s, blocks, tk, tv,
                     prefix_len, first, k, v, d, status);
  return hipGetLastError();
}

template <typename T>
hipError_t launch_commit_quant(uint8_t *blocks, T *tk, T *tv, const int32_t *prefix_len,
                               const int32_t *path, const int32_t *path_len,
                               const int32_t *status, int L, int B, int n1, int Hkv, int hd,
                               int qcap, int tcap, int32_t *new_len, hipStream_t s) {
  if (n1 > 65) return hipErrorInvalidValue;
  const QuantDims d{B, Hkv, 0, qcap, tcap, 1};
  const int pitch = (Q4_SLOTS - 1 + n1 + 7) / 8 * 8;   // 16-byte rows; up to 96 slots
  const size_t lds = (size_t)2 * pitch * hd * sizeof(T);
  auto kernel = hd == 64 ? commit_quant_kernel<T, 64> : commit_quant_kernel<T, 128>;
  if (lds > 65536) {   // fp32, trees of more than 32 rows: up to 96 KB
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)((long long)L * B * Hkv)), dim3(QT), lds, s, blocks, tk,
                     tv, prefix_len, path, path_len, status, n1, d, pitch, new_len);
  return hipGetLastError();
}

#define INSTANTIATE(T)                                                                            \
  template hipError_t launch_quantize_kv<T>(const T *, const T *, const int32_t *, const int32_t *, \
                                            uint8_t *, T *, T *, int, int, int, int, int, int, int, \
                                            int32_t *, hipStream_t);                              \
  template hipError_t launch_dequantize_kv<T>(const uint8_t *, const T *, const T *,              \
                                              const int32_t *, const int32_t *, T *, T *, int,    \
                                              int, int, int, int, int, int, int32_t *,            \
                                              hipStream_t);                                       \
  template hipError_t launch_commit_quant<T>(uint8_t *, T *, T *, const int32_t *,                \
                                             const int32_t *, const int32_t *, const int32_t *,   \
                                             int, int, int, int, int, int, int, int32_t *,        \
                                             hipStream_t);
INSTANTIATE(float)
INSTANTIATE(bf16)

}  // namespace acespec
