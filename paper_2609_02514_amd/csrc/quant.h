// Device helpers of the 4-bit KV cache (acespec_kv_quant): the block record and its groups.
//
// A record holds 32 slots of one (layer, session, kv head) as the operands of the attention's
// matrix instructions, so that a lane reads what it multiplies with 16-byte loads and every
// load of a wave is one contiguous run.  Lane l of a wave has lr = l % 16 and lg = l / 16.
//   offset 0         key codes.  Key row lr of operand kk (kk = 0, 1) is slot
//                    q4_key(kk, lr); the lane holds its head dims lg * hd/4 .. + hd/4.
//                    hd 128: [kk][lane][16 bytes], hd 64: [lane][kk][8 bytes]
//   offset 16 hd     value codes.  Value row lr of operand nb is head dim 16 nb + lr; the lane
//                    holds its slots 8 lg .. + 8.  [nb / 4][lane][nb % 4][4 bytes]
//   offset 32 hd     key scales [lr][group of 32 head dims][kk], a byte each
//   offset 33 hd     value scales [lr][nb], a byte each
// 34 hd bytes in all (17/32 byte an element where bf16 takes 2).  Codes are e2m1, the first of
// two in the low half of the byte; a scale byte s is 2^(s - 127), 255 marks a group that holds
// something not finite, and reads as NaN.  Both groups run along the axis the attention's
// products contract over (head dims of a key, slots of a value row), so one scale serves all
// eight codes of an operand's register.
#pragma once
#include "common.h"

constexpr int Q4_SLOTS = 32;
constexpr int q4_bytes(int hd) { return 34 * hd; }
constexpr uint32_t Q4_BAD = 255;
constexpr uint32_t Q4_MIN = 127 - 13;   // smallest scale: 2^-14 is its half step, fp16's least normal

// Slot (within a block) of key row m of operand kk: the scores' output row 4 lg + e of operand
// kk is then slot 8 lg + 4 kk + e, so a lane's scores of both operands are 8 consecutive slots,
// the ones its value operands hold.
AS_DEVICE int q4_key(int kk, int m) { return (m >> 2) * 8 + kk * 4 + (m & 3); }

AS_DEVICE float q4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes times their scale; exact in fp16 (scales are 2^-13 .. 2^13) and fp32.
AS_DEVICE f16x8 q4_decode_f16(uint32_t c, float s) {
  typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 0);
  const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 1);
  const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 2);
  const f16x2 e = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(c, s, 3);
  return f16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}
typedef float f32x8 __attribute__((ext_vector_type(8)));
AS_DEVICE f32x8 q4_decode_f32(uint32_t c, float s) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0);
  const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
  const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2);
  const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
  return f32x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

// The scale byte of a group whose largest magnitude has the bits `top` (an integer maximum
// over the magnitudes' bits, so that NaN and inf win): 2^(floor(log2 top) - 2), one power more
// from 1.75 times the power of two on, where 6 would be further off than a doubled step.
AS_DEVICE uint32_t q4_group_scale(uint32_t top) {
  if (top >= 0x47600000u) return Q4_BAD;                 // 57344 = 7 * 2^13, inf or NaN
  const uint32_t e = (top + 0x00200000u) >> 23;          // biased; the addition carries at 1.75
  return e < Q4_MIN + 2 ? Q4_MIN : e - 2;
}
AS_DEVICE uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Eight elements as they are stored, the largest of their magnitudes' bits (as fp32), and their
// codes: the nearest, ties to the even code, at most 6.
template <typename T> struct Raw8;
template <> struct Raw8<bf16> {
  u32x4 w;
  AS_DEVICE uint32_t top() const {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 m = __builtin_bit_cast(u16x2, w[0] & 0x7fff7fffu);
#pragma unroll
    for (int i = 1; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu));
    return (uint32_t)(m[0] > m[1] ? m[0] : m[1]) << 16;
  }
  AS_DEVICE uint32_t encode(float s) const {
    const bf16x8 v = __builtin_bit_cast(bf16x8, w);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_shufflevector(v, v, 0, 1), s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_shufflevector(v, v, 2, 3), s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_shufflevector(v, v, 4, 5), s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_shufflevector(v, v, 6, 7), s, 3);
    return c;
  }
  static AS_DEVICE u32x4 decoded(uint32_t c, float s) {   // exact in bf16
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
    return r;
  }
  AS_DEVICE void decode(uint32_t c, float s) { w = decoded(c, s); }
  AS_DEVICE void load(const bf16 *p) { w = *(const u32x4 *)p; }
  // (of memory that the kernel touches once: past L2 and the MALL)
  AS_DEVICE void load_once(const bf16 *p) { w = __builtin_nontemporal_load((const u32x4 *)p); }
  AS_DEVICE void store_once(bf16 *p) const { __builtin_nontemporal_store(w, (u32x4 *)p); }
  AS_DEVICE void store(bf16 *p) const { *(u32x4 *)p = w; }
  AS_DEVICE void store_first(bf16 *p, int n) const {   // n < 8 of them
    if (n & 4) *(uint2 *)p = make_uint2(w[0], w[1]);
    const uint32_t a = n & 4 ? w[2] : w[0], b = n & 4 ? w[3] : w[1];
    if (n & 2) *(uint32_t *)(p + (n & 4)) = a;
    if (n & 1) *(uint16_t *)(p + (n & 6)) = (uint16_t)(n & 2 ? b : a);
  }
};
template <> struct Raw8<float> {
  u32x4 w[2];
  AS_DEVICE uint32_t top() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, w[i >> 2][i & 3] & 0x7fffffffu);
    return m;
  }
  AS_DEVICE uint32_t encode(float s) const {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i >> 2][i & 3]);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
    return c;
  }
  AS_DEVICE void decode(uint32_t c, float s) {
    const f32x8 v = q4_decode_f32(c, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2][i & 3] = __float_as_uint(v[i]);
  }
  AS_DEVICE void load(const float *p) { w[0] = *(const u32x4 *)p; w[1] = *(const u32x4 *)(p + 4); }
  AS_DEVICE void load_once(const float *p) {
    w[0] = __builtin_nontemporal_load((const u32x4 *)p);
    w[1] = __builtin_nontemporal_load((const u32x4 *)(p + 4));
  }
  AS_DEVICE void store_once(float *p) const {
    __builtin_nontemporal_store(w[0], (u32x4 *)p);
    __builtin_nontemporal_store(w[1], (u32x4 *)(p + 4));
  }
  AS_DEVICE void store_first(float *p, int n) const {
    uint32_t *q = (uint32_t *)p;
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) q[i] = w[i >> 2][i & 3];
  }
  AS_DEVICE void store(float *p) const { *(u32x4 *)p = w[0]; *(u32x4 *)(p + 4) = w[1]; }
};

AS_DEVICE uint32_t max4_u32(uint32_t v) {   // over the lanes l, l^16, l^32, l^48
  v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return max(v, (uint32_t)__shfl_xor((int)v, 32));
}

// One wave writes the key codes and scales of operand kk of a record; load(slot, dim) gives 8
// head dims of a slot of the block.
template <typename T, int HD, typename F>
AS_DEVICE void q4_encode_keys(F &&load, int kk, uint8_t *rec, int lane) {
  constexpr int LD = HD / 4;   // head dims a lane holds of a key
  const int lr = lane & 15, lg = lane >> 4;
  Raw8<T> x[LD / 8];
  uint32_t top = 0, c[LD / 8];
#pragma unroll
  for (int j = 0; j < LD / 8; ++j) {
    x[j] = load(q4_key(kk, lr), lg * LD + j * 8);
    top = max(top, x[j].top());
  }
  if (HD == 64) top = max(top, (uint32_t)__shfl_xor((int)top, 16));   // two lanes a group
  const uint32_t sb = q4_group_scale(top);
#pragma unroll
  for (int j = 0; j < LD / 8; ++j) c[j] = sb == Q4_BAD ? 0u : x[j].encode(q4_scale(sb));
  if constexpr (HD == 128) {
    *(u32x4 *)(rec + kk * 1024 + lane * 16) = u32x4{c[0], c[1], c[2], c[3]};
    rec[32 * HD + (lr * 4 + lg) * 2 + kk] = (uint8_t)sb;
  } else {
    *(uint2 *)(rec + lane * 16 + kk * 8) = make_uint2(c[0], c[1]);
    if ((lg & 1) == 0) rec[32 * HD + (lr * 2 + (lg >> 1)) * 2 + kk] = (uint8_t)sb;
  }
}
// ... and half `h` of its value operands; load(dim, slot) gives 8 slots of a head dim.
template <typename T, int HD, typename F>
AS_DEVICE void q4_encode_values(F &&load, int h, uint8_t *rec, int lane) {
  constexpr int N = HD / 32;   // operands
  const int lr = lane & 15, lg = lane >> 4;
  uint32_t c[N], vs = 0;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const Raw8<T> x = load((h * N + n) * 16 + lr, lg * 8);
    const uint32_t sb = q4_group_scale(max4_u32(x.top()));
    vs |= sb << (8 * n);
    c[n] = sb == Q4_BAD ? 0u : x.encode(q4_scale(sb));
  }
  if constexpr (HD == 128) {
    *(u32x4 *)(rec + 16 * HD + h * 1024 + lane * 16) = u32x4{c[0], c[1], c[2], c[3]};
    if (lg == 0) *(uint32_t *)(rec + 33 * HD + lr * 8 + h * 4) = vs;
  } else {
    *(uint2 *)(rec + 16 * HD + lane * 16 + h * 8) = make_uint2(c[0], c[1]);
    if (lg == 0) *(uint16_t *)(rec + 33 * HD + lr * 4 + h * 2) = (uint16_t)vs;
  }
}

// What a lane holds of a record's operand kk of the keys, or half h of its values: codes (16
// bytes; head dim 64: 8) and scale bytes.
template <int HD> struct Q4Part {
  u32x4 c;
  uint32_t s;
  AS_DEVICE void load_keys(const uint8_t *rec, int kk, int lane) {
    const int lr = lane & 15, lg = lane >> 4;
    if constexpr (HD == 128) {
      c = *(const u32x4 *)(rec + kk * 1024 + lane * 16);
    } else {
      const uint2 v = *(const uint2 *)(rec + lane * 16 + kk * 8);
      c = u32x4{v.x, v.y, 0, 0};
    }
    s = rec[32 * HD + (lr * (HD / 32) + (HD == 128 ? lg : lg >> 1)) * 2 + kk];
  }
  AS_DEVICE void load_values(const uint8_t *rec, int h, int lane) {
    const int lr = lane & 15;
    if constexpr (HD == 128) {
      c = *(const u32x4 *)(rec + 16 * HD + h * 1024 + lane * 16);
      s = *(const uint32_t *)(rec + 33 * HD + lr * 8 + h * 4);
    } else {
      const uint2 v = *(const uint2 *)(rec + 16 * HD + lane * 16 + h * 8);
      c = u32x4{v.x, v.y, 0, 0};
      s = *(const uint16_t *)(rec + 33 * HD + lr * 4 + h * 2);
    }
  }
  // store(slot, dim, values) takes 8 head dims of a slot, store(dim, slot, values) 8 slots of
  // a head dim
  template <typename T, typename F> AS_DEVICE void decode_keys(F &&store, int kk, int lane) const {
#pragma unroll
    for (int j = 0; j < HD / 32; ++j) {
      Raw8<T> x;
      x.decode(c[j], q4_scale(s));
      store(q4_key(kk, lane & 15), (lane >> 4) * (HD / 4) + j * 8, x);
    }
  }
  template <typename T, typename F> AS_DEVICE void decode_values(F &&store, int h, int lane) const {
#pragma unroll
    for (int n = 0; n < HD / 32; ++n) {
      Raw8<T> x;
      x.decode(c[n], q4_scale((s >> (8 * n)) & 255u));
      store((h * (HD / 32) + n) * 16 + (lane & 15), (lane >> 4) * 8, x);
    }
  }
};
