// The 4-bit KV cache: a cache brought to 4 bits, read back, and the commit that brings the
// blocks of 32 slots to 4 bits as the verified path completes them.
//
// All three move bytes, and HBM bounds them: 4 layers x 16 sessions x 8 kv heads of 128, up to
// 2048 slots, 429 MB of bf16: 104 us to 4 bits (5.4 TB/s), 77 us back.  After a commit (32 layers
// x 48 sessions x 8, 1 to 9 slots each) it is lines: a value row has a few two-byte slots in
// each 128, and 268 MB move in 74 us (commit), 424 MB in 138 (read-back).  A workgroup takes the keys, or the values, of 64
// slots of a plane (layer, session, kv head): the unquantized side is read or written in whole
// 128-byte lines through LDS, the records in runs of 1 KB, and each wave converts one operand
// (keys) or half of them (values) of one of the two blocks.  A key group's maximum is the
// lane's own (head dim 64: of two lanes), a value group's takes two swaps between lanes.
#include "quant.h"

namespace {

constexpr int QT = 256;      // threads: four waves
constexpr int GROUP = 64;    // slots of a workgroup's turn: a 128-byte line of a bf16 value row
constexpr int PAD = 16;      // bytes behind an LDS row: 16 rows then start in different banks

struct QuantDims {
  int B, Hkv, cap, qcap, tcap, ng;   // sessions, kv heads, capacities, workgroups a plane and kind
};

// Which plane, kind and turns a workgroup has, and its session's lengths.
struct Share {
  size_t plane;
  int grp, values, full, t, first, last;   // first block; last group of 64 slots
  bool ok;
};
AS_DEVICE Share share_of(const QuantDims &d, const int32_t *prefix_len, const int32_t *first,
                         int32_t *status) {
  Share s;
  s.plane = blockIdx.x / (2 * d.ng);
  const int rest = blockIdx.x - (int)s.plane * (2 * d.ng);
  s.values = rest & 1;
  s.grp = rest >> 1;
  const int b = (int)(s.plane / d.Hkv) % d.B;
  const int P = prefix_len[b], F = first ? first[b] : 0;
  s.ok = P >= 0 && P <= d.cap && (P & ~(Q4_SLOTS - 1)) <= d.qcap && F >= 0 && F <= P;
  if (status && rest == 0 && s.plane < (size_t)d.B * d.Hkv && s.plane % d.Hkv == 0 && threadIdx.x == 0)
    status[b] = s.ok ? ACESPEC_OK : ACESPEC_EBADTREE;
  s.full = P / Q4_SLOTS;
  s.t = P % Q4_SLOTS;
  s.first = F / Q4_SLOTS;
  s.last = (P - 1) >> 6;
  return s;
}

template <typename T> AS_DEVICE void copy8(T *dst, const T *src) {
  Raw8<T> x;
  x.load(src);
  x.store(dst);
}
template <typename T> AS_DEVICE void copy8_once(T *dst, const T *src) {
  Raw8<T> x;
  x.load(src);
  x.store_once(dst);
}
// The t slots of the last, incomplete block, between the cache (slots from s0 on) and the tail.
template <typename T, int HD>
AS_DEVICE void copy_tail_keys(T *dst, const T *src, int t) {
#pragma unroll 2
  for (int e = threadIdx.x; e < t * (HD / 8); e += QT) copy8(dst + e * 8, src + e * 8);
}
template <typename T, int HD>
AS_DEVICE void copy_tail_values(T *dst, size_t dpitch, const T *src, size_t spitch, int t) {
#pragma unroll
  for (int e = threadIdx.x; e < HD * 4; e += QT) {
    const int r = e >> 2, c = (e & 3) * 8;
    if (c + 8 <= t) {
      copy8(dst + r * dpitch + c, src + r * spitch + c);
    } else if (c < t) {
      Raw8<T> x;   // (the source's row goes on: both sides' rows are whole pieces)
      x.load(src + r * spitch + c);
      x.store_first(dst + r * dpitch + c, t - c);
    }
  }
}

template <typename T, int HD> struct Stage {   // 64 slots of keys or values in LDS
  static constexpr int KP = HD + PAD / (int)sizeof(T), VP = GROUP + PAD / (int)sizeof(T);
  static constexpr int N = GROUP * KP > HD * VP ? GROUP * KP : HD * VP;
  __attribute__((aligned(16))) T x[N];
};

// The next turn's loads are in flight while this one's are converted.
template <typename T, int HD>
__global__ __launch_bounds__(QT) void quantize_kernel(const T *__restrict__ k,
                                                      const T *__restrict__ v,
                                                      const int32_t *__restrict__ prefix_len,
                                                      const int32_t *__restrict__ first,
                                                      uint8_t *__restrict__ blocks,
                                                      T *__restrict__ tk, T *__restrict__ tv,
                                                      QuantDims d, int32_t *__restrict__ status) {
  typedef Stage<T, HD> St;
  constexpr int N = GROUP * HD / 8 / QT;   // pieces a thread moves in a turn
  __shared__ St st;
  const Share s = share_of(d, prefix_len, first, status);
  if (!s.ok) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = wave & 1;
  const int off = (wave >> 1) * Q4_SLOTS;
  const T *src = s.values ? v + s.plane * HD * d.cap : k + s.plane * d.cap * HD;
  uint8_t *rec0 = blocks + s.plane * (d.qcap / Q4_SLOTS) * q4_bytes(HD);
  auto held = [&](int g) { return min(GROUP, s.full * Q4_SLOTS - g * GROUP); };   // in whole blocks
  Raw8<T> x[N];
  auto fetch = [&](int g) {
    const int n = held(g);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = tid + i * QT;
      if (s.values) {
        const int r = e >> 3, c = (e & 7) * 8;
        if (c < n) x[i].load_once(src + (size_t)r * d.cap + g * GROUP + c);
      } else {
        const int r = e / (HD / 8), c = e % (HD / 8) * 8;
        if (r < n) x[i].load_once(src + (size_t)(g * GROUP + r) * HD + c);
      }
    }
  };
  int g = (s.first >> 1) + s.grp;
  if (g <= s.last) fetch(g);
  for (; g <= s.last; g += d.ng) {
    const int n = held(g), blk = 2 * g + (wave >> 1);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = tid + i * QT;
      x[i].store(st.x + (s.values ? (e >> 3) * St::VP + (e & 7) * 8 : e / (HD / 8) * St::KP + e % (HD / 8) * 8));
    }
    __syncthreads();
    if (g + d.ng <= s.last) fetch(g + d.ng);
    if (off < n && blk >= s.first) {
      uint8_t *rec = rec0 + (size_t)blk * q4_bytes(HD);
      if (s.values)
        q4_encode_values<T, HD>([&](int dim, int slot) {
          Raw8<T> y;
          y.load(st.x + dim * St::VP + off + slot);
          return y;
        }, half, rec, lane);
      else
        q4_encode_keys<T, HD>([&](int slot, int dim) {
          Raw8<T> y;
          y.load(st.x + (off + slot) * St::KP + dim);
          return y;
        }, half, rec, lane);
    }
    __syncthreads();
    if (s.t && g == s.full >> 1) {
      const int s0 = s.full * Q4_SLOTS;
      if (s.values)
        copy_tail_values<T, HD>(tv + s.plane * HD * d.tcap, d.tcap, src + s0, d.cap, s.t);
      else
        copy_tail_keys<T, HD>(tk + s.plane * d.tcap * HD, src + (size_t)s0 * HD, s.t);
    }
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
  typedef Stage<T, HD> St;
  constexpr int N = GROUP * HD / 8 / QT;
  __shared__ St st;
  const Share s = share_of(d, prefix_len, first, status);
  if (!s.ok) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = wave & 1;
  const int off = (wave >> 1) * Q4_SLOTS;
  T *dst = s.values ? v + s.plane * HD * d.cap : k + s.plane * d.cap * HD;
  const uint8_t *rec0 = blocks + s.plane * (d.qcap / Q4_SLOTS) * q4_bytes(HD);
  Q4Part<HD> part;
  auto mine = [&](int g) {   // whether this wave has a block of turn g
    const int blk = 2 * g + (wave >> 1);
    return g <= s.last && blk < s.full && blk >= s.first;
  };
  auto fetch = [&](int g) {
    const uint8_t *rec = rec0 + (size_t)(2 * g + (wave >> 1)) * q4_bytes(HD);
    if (s.values) part.load_values(rec, half, lane);
    else part.load_keys(rec, half, lane);
  };
  int g = (s.first >> 1) + s.grp;
  if (mine(g)) fetch(g);
  for (; g <= s.last; g += d.ng) {
    const int n = min(GROUP, s.full * Q4_SLOTS - g * GROUP);
    const int lo = s.first > 2 * g ? Q4_SLOTS : 0;         // a block below `first`
    if (n > lo) {
      if (mine(g)) {
        if (s.values)
          part.template decode_values<T>([&](int dim, int slot, const Raw8<T> &y) {
            y.store(st.x + dim * St::VP + off + slot);
          }, half, lane);
        else
          part.template decode_keys<T>([&](int slot, int dim, const Raw8<T> &y) {
            y.store(st.x + (off + slot) * St::KP + dim);
          }, half, lane);
      }
      __syncthreads();
      if (mine(g + d.ng)) fetch(g + d.ng);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int e = tid + i * QT;
        if (s.values) {
          const int r = e >> 3, c = (e & 7) * 8;
          if (c < n && c >= lo) copy8_once(dst + (size_t)r * d.cap + g * GROUP + c, st.x + r * St::VP + c);
        } else {
          const int r = e / (HD / 8), c = e % (HD / 8) * 8;
          if (r < n && r >= lo) copy8_once(dst + (size_t)(g * GROUP + r) * HD + c, st.x + r * St::KP + c);
        }
      }
      __syncthreads();
    }
    if (s.t && g == s.full >> 1) {
      const int s0 = s.full * Q4_SLOTS;
      if (s.values)
        copy_tail_values<T, HD>(dst + s0, d.cap, tv + s.plane * HD * d.tcap, d.tcap, s.t);
      else
        copy_tail_keys<T, HD>(dst + (size_t)s0 * HD, tk + s.plane * d.tcap * HD, s.t);
    }
  }
}

// Commit (Algorithm 1, COMPACT_KV).  With t = P % 32 the session's committed slots are the
// tail's [0, t], the root among them, and the kept rows t + path[i]: t + 1 + np slots in that
// order, of which every complete 32 become a record and the rest the tail's front.  One
// workgroup per plane.  All that moves goes through LDS first, as a destination may be another
// entry's source: keys row by row, values as the 16-byte pieces of each row that hold a slot
// that moves or is moved to (a row's other slots are written back as they were: nothing else
// writes this plane).
template <typename T, int HD>
__global__ __launch_bounds__(QT) void commit_quant_kernel(
    uint8_t *__restrict__ blocks, T *__restrict__ tk, T *__restrict__ tv,
    const int32_t *__restrict__ prefix_len, const int32_t *__restrict__ path,
    const int32_t *__restrict__ path_len, const int32_t *__restrict__ status, int n1,
    QuantDims d, int vpitch, int32_t *__restrict__ new_len) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  __shared__ int src[96];                 // slot of the tail that committed slot i comes from
  const size_t plane = blockIdx.x;
  const int b = (int)(plane / d.Hkv) % d.B, tid = threadIdx.x;
  const int32_t row = tid < n1 - 1 ? path[(size_t)b * n1 + tid] : 0;
  const int P = prefix_len[b], np = path_len[b];
  const int st = status ? status[b] : ACESPEC_OK;
  const int t = P & (Q4_SLOTS - 1);
  const bool ok = st == ACESPEC_OK && P >= 0 && np >= 0 && np < n1;
  const int end = ok ? t + 1 + np : 0, nblk = end / Q4_SLOTS;
  const bool fits = ok && P / Q4_SLOTS + nblk <= d.qcap / Q4_SLOTS;
  const bool bad = __syncthreads_or(!fits || (tid < np && (row < 1 || row >= n1)));
  if (plane < (size_t)d.B * d.Hkv && plane % d.Hkv == 0 && tid == 0) new_len[b] = bad ? -1 : P + 1 + np;
  if (bad || (np == 0 && nblk == 0)) return;
  // What moves: from slot `lo` on (without a complete block only the kept rows do).
  const int lo = nblk ? 0 : t + 1;
  if (tid <= t) src[tid] = tid;
  if (tid < np) src[t + 1 + tid] = t + row;
  __syncthreads();
  T *kd = tk + plane * d.tcap * HD, *vd = tv + plane * HD * d.tcap;
  T *vx = (T *)smem, *kx = vx + (size_t)HD * vpitch;       // [HD][slots from 8 p0], [slot - lo][HD]
  const int p0 = lo / 8, np8 = (t + n1 + 7) / 8 - p0;      // pieces of a value row
#pragma unroll 4
  for (int e = tid; e < HD * np8; e += QT) {
    const int r = e / np8, c = (e - r * np8) * 8;
    copy8(vx + r * vpitch + c, vd + (size_t)r * d.tcap + p0 * 8 + c);
  }
#pragma unroll 4
  for (int e = tid; e < (end - lo) * (HD / 8); e += QT) {
    const int i = e / (HD / 8), c = e % (HD / 8) * 8;
    copy8(kx + i * HD + c, kd + (size_t)src[lo + i] * HD + c);
  }
  __syncthreads();
  auto gather = [&](int dim, int i) -> Raw8<T> {           // committed slots i .. i + 8 of a row
    __attribute__((aligned(16))) T y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = vx[dim * vpitch + src[i + j]];
    Raw8<T> r;
    r.load(y);
    return r;
  };
  for (int x = tid >> 6; x < 4 * nblk; x += QT / 64) {     // operands of the new records
    const int blk = x >> 2, s0 = blk * Q4_SLOTS;
    uint8_t *rec = blocks + (plane * (d.qcap / Q4_SLOTS) + P / Q4_SLOTS + blk) * q4_bytes(HD);
    if (x & 2)
      q4_encode_values<T, HD>([&](int dim, int slot) { return gather(dim, s0 + slot); }, x & 1, rec,
                              tid & 63);
    else
      q4_encode_keys<T, HD>([&](int slot, int dim) {
        Raw8<T> y;
        y.load(kx + (s0 + slot) * HD + dim);
        return y;
      }, x & 1, rec, tid & 63);
  }
  // Committed slots from `from` on move to the tail's slots from `to` on.
  const int from = nblk ? nblk * Q4_SLOTS : lo, to = nblk ? 0 : lo, cnt = end - from;
#pragma unroll 4
  for (int e = tid; e < cnt * (HD / 8); e += QT)
    copy8(kd + (size_t)to * HD + e * 8, kx + (size_t)(from - lo) * HD + e * 8);
  const int q0 = to / 8, nq8 = (to + cnt + 7) / 8 - q0;
#pragma unroll 4
  for (int e = tid; e < HD * nq8; e += QT) {
    const int r = e / nq8, c = (q0 + e - r * nq8) * 8;     // first slot of the piece
    __attribute__((aligned(16))) T y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = c + j - to;                            // the moved slot that lands here
      y[j] = vx[r * vpitch + (i >= 0 && i < cnt ? src[from + i] : c + j) - p0 * 8];
    }
    copy8(vd + (size_t)r * d.tcap + c, y);
  }
}

// Workgroups a plane and kind: a turn each, but no more in all than fill the chip several times
// over.  With `first` most sessions have a few slots to move, and more workgroups than planes
// only come and go (32 layers x 48 sessions x 8 heads, a few slots each: 172 us with one a
// plane, 260 with two); without, each turn is worth a workgroup (400 MB: 107 us, and 120 with a
// quarter of them).
int groups_of(long long planes, int slots, bool appended) {
  const long long want = ((appended ? 4096 : 16384) + planes - 1) / planes;
  const int most = (slots + GROUP - 1) / GROUP;
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
                    groups_of(planes, cap < qcap + Q4_SLOTS ? cap : qcap + Q4_SLOTS, first != nullptr)};
  auto kernel = hd == 64 ? quantize_kernel<T, 64> : quantize_kernel<T, 128>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(planes * 2 * d.ng)), dim3(QT), 0, s, k, v, prefix_len,
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
                    groups_of(planes, cap < qcap + Q4_SLOTS ? cap : qcap + Q4_SLOTS, first != nullptr)};
  auto kernel = hd == 64 ? dequantize_kernel<T, 64> : dequantize_kernel<T, 128>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(planes * 2 * d.ng)), dim3(QT), 0, s, blocks, tk, tv,
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
  // LDS: rows of values with the tail's slots (whole pieces, and one behind them against bank
  // conflicts), and the keys' rows
  const int slots = Q4_SLOTS - 1 + n1, vpitch = (slots + 7) / 8 * 8 + 8;
  const size_t lds = (size_t)(vpitch + slots) * hd * sizeof(T);
  auto kernel = hd == 64 ? commit_quant_kernel<T, 64> : commit_quant_kernel<T, 128>;
  if (lds > 65536) {   // fp32, trees of more than 32 rows: up to 100 KB
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)((long long)L * B * Hkv)), dim3(QT), lds, s, blocks, tk,
                     tv, prefix_len, path, path_len, status, n1, d, vpitch, new_len);
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
