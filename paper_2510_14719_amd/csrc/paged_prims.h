// Device parts that the kernels around the paged cache share: the batch, exchange between lane groups, LDS layout of cached rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gfx950_prims.h"
#include "paged_launch.h"

namespace {

// New tokens and length of a sequence, brought into the bounds of the call whatever the arrays hold.
struct SeqRange {
    int q0, n, kv;
};
__device__ __forceinline__ SeqRange seq_range(const int* q_start, const int* kv_len, int s, int tokens, int max_q, int max_kv)
{
    const int q0 = min(max(q_start[s], 0), tokens), q1 = min(max(q_start[s + 1], q0), tokens);
    return {q0, min(q1 - q0, max_q), min(max(kv_len[s], 0), max_kv)};
}

// The last sequence that starts at or before token t, found by the 64 lanes of a wave together (two steps up to 4096 sequences);
// -1 if none does.
__device__ __forceinline__ int seq_of_token(const int* q_start, int sequences, int t, int lane)
{
    int lo = 0, n = sequences;
    while (n > 0) {
        const int step = (n + 63) / 64, i = lane * step;
        const unsigned long long below = __builtin_amdgcn_ballot_w64(i < n && q_start[lo + min(i, n - 1)] <= t);
        if (below == 0) return lo - 1;
        // (starts do not fall; if they do all the same, some sequence of the range comes out)
        const int last = 63 - __builtin_clzll(below);
        lo += last * step;
        n = min(step, n - last * step);
        if (step == 1) return lo;
    }
    return -1;
}

// Exchange with lane^32 and lane^16: v_permlane32_swap swaps the upper 32 lanes of its first operand with the lower 32 of its second,
// v_permlane16_swap odd rows of 16 lanes with even ones.  (Inline asm: the compiler folds the two results of the builtins into one when
// both inputs are the same value; the s_nop covers the VALU-write -> permlane-read hazard.)
__device__ __forceinline__ void lanes32(float x, float& a, float& b) {
    a = x;
    b = x;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
}
__device__ __forceinline__ void lanes16(float x, float& a, float& b) {
    a = x;
    b = x;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
}
// Maximum and sum over the four lanes that share lane % 16.
__device__ __forceinline__ float groups_max(float x) {
    float a, b;
    lanes16(x, a, b);
    lanes32(__builtin_fmaxf(a, b), a, b);
    return __builtin_fmaxf(a, b);
}
__device__ __forceinline__ float groups_sum(float x) {
    float a, b;
    lanes16(x, a, b);
    lanes32(a + b, a, b);
    return a + b;
}

// Eight E4M3 values as eight 16-bit ones (exact: every E4M3 value is one of both types).
template <int DTYPE> __device__ __forceinline__ s16x8 widen8(u32x2 w)
{
    typedef typename Elem<DTYPE>::v2 v2;
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (DTYPE == 0) {
            r[2 * i] = __builtin_bit_cast(unsigned, (v2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, false));
            r[2 * i + 1] = __builtin_bit_cast(unsigned, (v2)__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[i], 1.0f, true));
        } else {
            r[2 * i] = __builtin_bit_cast(unsigned, (v2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, false));
            r[2 * i + 1] = __builtin_bit_cast(unsigned, (v2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.0f, true));
        }
    }
    return __builtin_bit_cast(s16x8, r);
}

template <int DTYPE> __device__ __forceinline__ float to_float(uint16_t x)
{
    if constexpr (DTYPE == 0) return (float)__builtin_bit_cast(_Float16, x);
    else return __builtin_bit_cast(float, (unsigned)x << 16);
}

// LDS layout of ROWS cached rows (K or V), a multiple of 32: [group of LINE bytes of a row][row][LINE], 16-byte columns of a line permuted.
//
// The order of the keys.  S^T = K Q^T by 16x16x32 MFMAs leaves lane group g = lane / 16 with the rows 4 g ... 4 g + 3 of each of the two
// 16-row blocks of 32 keys.  Block kb takes as its row r the key 8 (r / 4) + 4 kb + r % 4 of the 32, so the group holds the keys 8 g ... 8 g + 7, in
// order: just what one lane of the second product's V^T operand holds, and what the transposing reads bring (8 keys of one 8-bit
// feature, or twice 4 of a 16-bit one).
//
// The permutation of the columns (a column c of row r stands at c ^ swK(r) or c ^ swV(r)): 16 lanes that read one column of K's rows {8 a +
// 4 kb + b}, and the 8 or 16 rows that half a wave of a transposing read touches, cover all 64 banks.
template <int D, int ES, int ROWS> struct CachedRows {
    static constexpr int ROW = D * ES, LINE = ROW < 128 ? ROW : 128, GROUPS = ROW / LINE, COLS = LINE / 16;
    static constexpr int BYTES = ROWS * ROW;
    static constexpr int PER_PIECE = 64 / COLS;              // rows that one copy of 64 x 16 bytes brings: 8, or 16 short ones
    static __device__ __forceinline__ int sw_k(int r) { return LINE == 128 ? ((r >> 3) & 3) * 2 + ((r >> 1) & 1) : (r >> 3) & 3; }
    static __device__ __forceinline__ int sw_v(int r) {
        if (ES == 2) return (((r >> 3) & 1) * 2 + ((r >> 1) & 1)) * 2;       // (32-byte pairs of columns stay together)
        return LINE == 128 ? ((r >> 3) & 1) * 4 + ((r >> 1) & 3) : ((r >> 3) & 1) * 2 + ((r >> 2) & 1);
    }
    // K operand of 16 keys x 32 features: block kb (of 32 keys), features kk * 32 ...
    template <int DTYPE> static __device__ __forceinline__ s16x8 k_operand(const char* k, int kb, int kk, int lane) {
        const int lc = lane & 15, lg = lane >> 4, r = (kb >> 1) * 32 + (lc >> 2) * 8 + (kb & 1) * 4 + (lc & 3);
        const int byte = kk * 32 * ES + lg * 8 * ES, line = byte / LINE, col = byte % LINE / 16;
        const char* const at = k + line * (ROWS * LINE) + r * LINE + ((col ^ sw_k(r)) * 16) + byte % 16;
        if constexpr (ES == 2) return *reinterpret_cast<const s16x8*>(at);
        else return widen8<DTYPE>(*reinterpret_cast<const u32x2*>(at));
    }
    // V^T operand of 16 features x 32 keys: features fb * 16 ..., keys kc * 32 ...
    template <int DTYPE> static __device__ __forceinline__ s16x8 v_operand(const char* v, int kc, int fb, int lane) {
        const int lc = lane & 15, lg = lane >> 4;
        if constexpr (ES == 2) {
            const int r = kc * 32 + lg * 8 + (lc >> 2), byte = fb * 32, line = byte / LINE, col = byte % LINE / 16;
            const char* const at = v + line * (ROWS * LINE) + r * LINE + ((col ^ sw_v(r)) * 16) + (lc & 3) * 8;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(at));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS s16x4*)(at + 4 * LINE));   // (the same permutation)
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            typedef int i32x2 __attribute__((ext_vector_type(2)));
            const int r = kc * 32 + lg * 8 + (lc >> 1), byte = fb * 16, line = byte / LINE, col = byte % LINE / 16;
            const char* const at = v + line * (ROWS * LINE) + r * LINE + ((col ^ sw_v(r)) * 16) + (lc & 1) * 8;
            const i32x2 x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((LDS_AS i32x2*)(at));
            return widen8<DTYPE>(__builtin_bit_cast(u32x2, x));
        }
    }
    // One value of V.
    template <int DTYPE> static __device__ __forceinline__ float v_value(const char* v, int r, int f) {
        const int byte = f * ES, line = byte / LINE, col = byte % LINE / 16;
        const char* const at = v + line * (ROWS * LINE) + r * LINE + ((col ^ sw_v(r)) * 16) + byte % 16;
        if constexpr (ES == 2) return to_float<DTYPE>(*reinterpret_cast<const uint16_t*>(at));
        else return __builtin_amdgcn_cvt_f32_fp8(*reinterpret_cast<const uint8_t*>(at), 0);
    }
};

// Non-finite values of a V^T operand: which halves of w have all exponent bits set, as a mask of the whole halves.
template <int DTYPE> __device__ __forceinline__ unsigned not_finite(unsigned w)
{
    constexpr unsigned E = DTYPE == 0 ? 0x7c00u : 0x7f80u;
    return ((w & E) == E ? 0xffffu : 0u) | ((w >> 16 & E) == E ? 0xffff0000u : 0u);
}

}  // namespace
