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

// Eight elements to codes: the nearest, ties to the even code, at most 6.
AS_DEVICE uint32_t q4_encode(const float *x, float s) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  return c;
}

AS_DEVICE uint32_t max4_u32(uint32_t v) {   // over the lanes l, l^16, l^32, l^48
  v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return max(v, (uint32_t)__shfl_xor((int)v, 32));
}

// Eight consecutive elements as floats, and back (16-byte aligned).
AS_DEVICE void load8(const bf16 *p, float *x) {
  const bf16x8 v = *(const bf16x8 *)p;
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
}
AS_DEVICE void load8(const float *p, float *x) {
  const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
}
AS_DEVICE void store8(bf16 *p, f32x8 x) {
  bf16x8 v;
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = (bf16)x[i];
  *(bf16x8 *)p = v;
}
AS_DEVICE void store8(float *p, f32x8 x) {
  *(f32x4 *)p = f32x4{x[0], x[1], x[2], x[3]};
  *(f32x4 *)(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// One wave writes a record from 32 slots: keys k[slot * HD + dim], values v[dim * vstride +
// slot], both 16-byte aligned.
template <typename T, int HD>
AS_DEVICE void q4_encode_block(const T *k, const T *v, size_t vstride, uint8_t *rec, int lane) {
  constexpr int LD = HD / 4, NB = HD / 16;   // head dims a lane holds of a key; value operands
  const int lr = lane & 15, lg = lane >> 4;
  uint32_t kc[2][LD / 8];
  uint32_t ks[2];
#pragma unroll
  for (int kk = 0; kk < 2; ++kk) {
    float x[LD];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < LD / 8; ++j) load8(k + (size_t)q4_key(kk, lr) * HD + lg * LD + j * 8, x + j * 8);
#pragma unroll
    for (int j = 0; j < LD; ++j) top = max(top, abs_bits(x[j]));
    if (HD == 64) top = max(top, (uint32_t)__shfl_xor((int)top, 16));   // two lanes a group
    ks[kk] = q4_group_scale(top);
    const float s = q4_scale(ks[kk]);
#pragma unroll
    for (int j = 0; j < LD / 8; ++j) kc[kk][j] = ks[kk] == Q4_BAD ? 0u : q4_encode(x + j * 8, s);
  }
  uint32_t vc[NB];
  uint64_t vs = 0;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float x[8];
    uint32_t top = 0;
    load8(v + (size_t)(nb * 16 + lr) * vstride + lg * 8, x);
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, abs_bits(x[j]));
    const uint32_t sb = q4_group_scale(max4_u32(top));
    vs |= (uint64_t)sb << (8 * nb);
    vc[nb] = sb == Q4_BAD ? 0u : q4_encode(x, q4_scale(sb));
  }
  if constexpr (HD == 128) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk)
      *(u32x4 *)(rec + kk * 1024 + lane * 16) = u32x4{kc[kk][0], kc[kk][1], kc[kk][2], kc[kk][3]};
    *(uint16_t *)(rec + 32 * HD + (lr * 4 + lg) * 2) = (uint16_t)(ks[0] | (ks[1] << 8));
    if (lg == 0) *(uint2 *)(rec + 33 * HD + lr * 8) = make_uint2((uint32_t)vs, (uint32_t)(vs >> 32));
  } else {
    *(u32x4 *)(rec + lane * 16) = u32x4{kc[0][0], kc[0][1], kc[1][0], kc[1][1]};
    if ((lg & 1) == 0)
      *(uint16_t *)(rec + 32 * HD + (lr * 2 + (lg >> 1)) * 2) = (uint16_t)(ks[0] | (ks[1] << 8));
    if (lg == 0) *(uint32_t *)(rec + 33 * HD + lr * 4) = (uint32_t)vs;
  }
#pragma unroll
  for (int h = 0; h < NB / 4; ++h)
    *(u32x4 *)(rec + 16 * HD + h * 1024 + lane * 16) =
        u32x4{vc[h * 4], vc[h * 4 + 1], vc[h * 4 + 2], vc[h * 4 + 3]};
}

// What a lane holds of a record.
template <int HD> struct Q4Regs {
  u32x4 k[HD / 64], v[HD / 64];
  uint32_t ks;           // bytes kk = 0, 1
  uint32_t vs[HD / 64];  // byte nb % 4 of word nb / 4
};
template <int HD> AS_DEVICE void q4_load(Q4Regs<HD> &r, const uint8_t *rec, int lane) {
  const int lr = lane & 15, lg = lane >> 4;
#pragma unroll
  for (int h = 0; h < HD / 64; ++h) {
    r.k[h] = *(const u32x4 *)(rec + h * 1024 + lane * 16);
    r.v[h] = *(const u32x4 *)(rec + 16 * HD + h * 1024 + lane * 16);
  }
  r.ks = *(const uint16_t *)(rec + 32 * HD + (lr * (HD / 32) + (HD == 128 ? lg : lg >> 1)) * 2);
  if constexpr (HD == 128) {
    const uint2 t = *(const uint2 *)(rec + 33 * HD + lr * 8);
    r.vs[0] = t.x;
    r.vs[1] = t.y;
  } else {
    r.vs[0] = *(const uint32_t *)(rec + 33 * HD + lr * 4);
  }
}
// Word j of the lane's key codes of operand kk: head dims lg * HD/4 + 8 j .. + 8.
template <int HD> AS_DEVICE uint32_t q4_kword(const Q4Regs<HD> &r, int kk, int j) {
  return HD == 128 ? r.k[kk * (HD / 128)][j] : r.k[0][kk * 2 + j];
}
template <int HD> AS_DEVICE float q4_kscale(const Q4Regs<HD> &r, int kk) {
  return q4_scale((r.ks >> (8 * kk)) & 255u);
}
template <int HD> AS_DEVICE uint32_t q4_vword(const Q4Regs<HD> &r, int nb) { return r.v[nb >> 2][nb & 3]; }
template <int HD> AS_DEVICE float q4_vscale(const Q4Regs<HD> &r, int nb) {
  return q4_scale((r.vs[nb >> 2] >> (8 * (nb & 3))) & 255u);
}
