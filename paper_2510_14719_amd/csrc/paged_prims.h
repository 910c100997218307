// Device parts that the kernels around the paged cache share: the batch, exchange between lane groups, LDS layout of cached rows.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gfx950_prims.h"
#include "paged_launch.h"

namespace {

// New tokens of a sequence, what it has in all and the position of its first new token, brought into the bounds of the call whatever the arrays hold: of too many new tokens the
// first max_q are left, of a sequence that is too long those at positions below max_kv.  Both keep their positions (negative where there are more new tokens than tokens).
struct SeqRange {
    int q0, n, kv, first;
};
__device__ __forceinline__ SeqRange seq_range(const int* q_start, const int* kv_len, int s, int tokens, int max_q, int max_kv)
{
    const int q0 = min(max(q_start[s], 0), tokens), all = min(max(q_start[s + 1], q0), tokens) - q0, first = max(kv_len[s], 0) - all;
    int n = min(all, max_q);
    if (first > max_kv - n) n = max(max_kv - first, 0);
    return {q0, n, min(max(first + n, 0), max_kv), first};
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

// ---- how the sequences of small tiles are cut along their keys
//
// Where their workgroups are fewer than the chip has places (few_room > 0), every wave finds for itself the shortest of some lengths whose pieces, of all
// sequences together, still have a place each, and which piece its workgroup has.  (One token each, 32 heads on 8,
// d 128, with pieces of one length that the host chose from the longest sequence / so: 11 of 9000 102 / 76 us, 3 of 9000 34.8 / 27.3, 9 of 2000 ... 9000 54 / 40.)
// Pieces of a sequence, cut for 1 / inverse keys (a row tile of it has as many, of its own keys).
__device__ __forceinline__ int few_pieces(float inverse, int kv) { return max(1, (int)__builtin_ceilf(__builtin_fmaf((float)kv, inverse, -0.001f))); }
__device__ __forceinline__ int few_tiles(const PagedArgs& a, const SeqRange& seq)
{
    const int rows = seq.n * a.group;
    return rows > a.few_rows ? 0 : (rows + a.rows - 1) / a.rows;
}
__device__ __forceinline__ SeqRange few_seq(const PagedArgs& a, int s)
{
    return s < a.sequences ? seq_range(a.q_start, a.kv_len, s, a.tokens, a.max_q, a.max_kv) : SeqRange{0, 0, 0, 0};
}
// (`first`: the first 64 sequences, a lane each; a lane has a length)
__device__ inline float few_cut(const PagedArgs& a, const SeqRange& first, int lane)
{
    if (a.few_fixed) {
        int pieces = 0;
        for (int s0 = 0; s0 < a.sequences; s0 += 64) {
            const SeqRange seq = s0 == 0 ? first : few_seq(a, s0 + lane);
            pieces += few_tiles(a, seq) * few_pieces(a.few_finest, seq.kv);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) pieces += __shfl_xor(pieces, d);
        if (__builtin_amdgcn_readfirstlane(pieces) <= a.few_room) return a.few_finest;
    }
    const float inverse = lane == 63 ? a.few_coarsest : a.few_finest * __builtin_amdgcn_exp2f(-a.few_step * lane);
    int pieces = 0;
    for (int s0 = 0; s0 < a.sequences; s0 += 64) {
        const SeqRange seq = s0 == 0 ? first : few_seq(a, s0 + lane);
        const int tiles = few_tiles(a, seq);
        unsigned long long there = __builtin_amdgcn_ballot_w64(tiles > 0);
        while (there) {
            const int i = __builtin_ctzll(there);
            there &= there - 1;
            pieces += __builtin_amdgcn_readlane(tiles, i) * few_pieces(inverse, __builtin_amdgcn_readlane(seq.kv, i));
        }
    }
    const unsigned long long fits = __builtin_amdgcn_ballot_w64(lane == 63 || pieces <= a.few_room);     // (the longest: the host has seen to it)
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, inverse), __builtin_ctzll(fits)));
}
// The piece with a number; s = -1 behind the last.
struct FewPiece {
    int s, tile, piece, pieces;
    SeqRange seq;
};
__device__ inline FewPiece few_numbered(const PagedArgs& a, const SeqRange& first, float inverse, int left, int lane)
{
    for (int s0 = 0; s0 < a.sequences; s0 += 64) {
        const SeqRange seq = s0 == 0 ? first : few_seq(a, s0 + lane);
        const int pieces = few_pieces(inverse, seq.kv), own = few_tiles(a, seq) * pieces;
        int sum = own;                          // with those of the lanes before
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(sum, d);
            if (lane >= d) sum += x;
        }
        const unsigned long long beyond = __builtin_amdgcn_ballot_w64(sum > left);
        if (beyond) {
            const int at = __builtin_ctzll(beyond), n = __builtin_amdgcn_readlane(pieces, at), inside = left - (__builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(own, at));
            return {s0 + at, inside / n, inside % n, n, 
                    {__builtin_amdgcn_readlane(seq.q0, at), __builtin_amdgcn_readlane(seq.n, at), __builtin_amdgcn_readlane(seq.kv, at), __builtin_amdgcn_readlane(seq.first, at)}};
        }
        left -= __builtin_amdgcn_readlane(sum, 63);
    }
    return {-1, 0, 0, 1, {0, 0, 0, 0}};
}
// Keys of a piece of a row tile with so many keys.
__device__ __forceinline__ int few_piece_keys(int pieces, int keys) { return max(((keys + pieces - 1) / pieces + 63) / 64 * 64, 64); }

// ---- how chunks are cut along their keys
//
// Chunks of the sequences with more rows than few_rows are numbered through, the last one of a sequence first.  Where they are fewer than the chip has compute
// units, those of long sequences are cut into pieces; which length to cut for is found on the device, from the lengths that are there, by every wave of the
// kernel for itself: of 64 lengths, the longest sequence's x 2^(-3c/32), the shortest that still makes no more pieces than there are compute units, if that
// is worth the joining.  (On MI355X a tile of 64 keys takes 1.6 us, leaving partial results 6, joining them 8.  us cut / not, all by chunks: 12 sequences of 1 ... 777 new tokens,
// 900 ... 4001 keys, 16 heads on 4, d 128 64 / 97 (69 with 15 lengths a fourth of an octave apart); 8 of 64 new tokens, 4000 keys, the same heads 40 / 96; one of 1024, 1024 keys 28 / 34;
// one of 5, 16384 keys, 32 heads on 4 25 (33 with 16 pieces at most).)
constexpr int CHUNK_PARTS = 256;                // most pieces: a round of the compute units
constexpr int CHUNK_UNCUT = 512;                // sequences up to this length are not cut
constexpr float CHUNK_SAVES = 9.f, CHUNK_LEAST = 4.f;            // tiles that cutting has to save, and leaves in a piece at least

struct ChunkSeq {
    int chunks, tiles;                          // chunks of the sequence, key tiles of its longest
};
__device__ __forceinline__ ChunkSeq chunk_seq(const PagedArgs& a, int s)
{
    if (s >= a.sequences) return {0, 0};
    const SeqRange seq = seq_range(a.q_start, a.kv_len, s, a.tokens, a.max_q, a.max_kv);
    const int rows = seq.n * a.group;
    if (rows <= a.few_rows) return {0, 0};
    return {(rows + PAGED_CHUNK_ROWS - 1) / PAGED_CHUNK_ROWS, (seq.kv + 63) / 64};
}
// Calls f(chunks, tiles) for every sequence that goes by chunks; `first`: those of the first 64, a lane each.
template <typename F> __device__ __forceinline__ void each_chunk_seq(const PagedArgs& a, const ChunkSeq& first, int lane, F f)
{
    for (int s0 = 0; s0 < a.sequences; s0 += 64) {
        const ChunkSeq q = s0 == 0 ? first : chunk_seq(a, s0 + lane);
        unsigned long long there = __builtin_amdgcn_ballot_w64(q.chunks > 0);
        while (there) {
            const int i = __builtin_ctzll(there);
            there &= there - 1;
            f(__builtin_amdgcn_readlane(q.chunks, i), __builtin_amdgcn_readlane(q.tiles, i));
        }
    }
}
// Pieces of a chunk of a sequence of so many tiles, where it is cut for 1 / inverse tiles.
__device__ __forceinline__ int chunk_pieces(float inverse, int tiles) { return max(1, (int)__builtin_ceilf((float)tiles * inverse - 0.001f)); }
// 1 / the length to cut for (0: not at all), and how many chunks there are in that case.
struct ChunkCut {
    float inverse;
    int chunks;
};
__device__ inline ChunkCut chunk_cut(const PagedArgs& a, const ChunkSeq& first, int key_heads, int lane)
{
    if (a.chunk_parts == 0) return {0.f, 0};
    int longest = 0, chunks = 0;
    each_chunk_seq(a, first, lane, [&](int n, int tiles) {
        longest = max(longest, tiles);
        chunks += n;
    });
    if (longest <= CHUNK_UNCUT / 64 || chunks * key_heads >= a.chunk_parts) return {0.f, 0};
    const float length = (float)longest * __builtin_amdgcn_exp2f(-0.09375f * (1 + lane)), inverse = 1.f / length;
    int pieces = 0;
    each_chunk_seq(a, first, lane, [&](int n, int tiles) { pieces += n * chunk_pieces(inverse, tiles); });
    const unsigned long long fits = __builtin_amdgcn_ballot_w64(pieces * key_heads <= a.chunk_parts && (float)longest - length > CHUNK_SAVES && length >= CHUNK_LEAST);
    if (fits == 0) return {0.f, 0};
    return {__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, inverse), 63 - __builtin_clzll(fits))), chunks};
}
// Sequence, chunk and piece with a number, and the chunk's number; s = -1 behind the last.
struct ChunkPiece {
    int s, chunk, piece, pieces, number;
};
__device__ inline ChunkPiece chunk_numbered(const PagedArgs& a, const ChunkSeq& first, float inverse, int left, int lane)
{
    int number = 0;
    for (int s0 = 0; s0 < a.sequences; s0 += 64) {
        const ChunkSeq q = s0 == 0 ? first : chunk_seq(a, s0 + lane);
        const int pieces = chunk_pieces(inverse, q.tiles);
        int sum = q.chunks * pieces, before = q.chunks;      // with those of the lanes before
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int x = __shfl_up(sum, d), y = __shfl_up(before, d);
            if (lane >= d) {
                sum += x;
                before += y;
            }
        }
        const unsigned long long beyond = __builtin_amdgcn_ballot_w64(sum > left);
        if (beyond) {
            const int at = __builtin_ctzll(beyond), n = __builtin_amdgcn_readlane(pieces, at), chunks = __builtin_amdgcn_readlane(q.chunks, at);
            const int inside = left - (__builtin_amdgcn_readlane(sum, at) - chunks * n);
            return {s0 + at, chunks - 1 - inside / n, inside % n, n, number + __builtin_amdgcn_readlane(before, at) - chunks + inside / n};
        }
        left -= __builtin_amdgcn_readlane(sum, 63);
        number += __builtin_amdgcn_readlane(before, 63);
    }
    return {-1, 0, 0, 1, 0};
}
// Key tiles per piece.
__device__ __forceinline__ int chunk_piece_tiles(int pieces, int keys) { return max(1, ((keys + 63) / 64 + pieces - 1) / pieces); }

// ---- the same for prompts, whose chunks see different numbers of keys under the mask: each is cut for its own (see launch)
struct OwnSeq {
    int chunks, tiles;                          // chunks of the sequence, key tiles of its last, which are the most
    float head;                                 // tiles less in the one before that; each further one has 4 / group less
};
__device__ __forceinline__ OwnSeq own_seq(const PagedArgs& a, int s)
{
    const ChunkSeq q = chunk_seq(a, s);
    if (q.chunks == 0) return {0, 0, 0.f};
    const SeqRange seq = seq_range(a.q_start, a.kv_len, s, a.tokens, a.max_q, a.max_kv);
    return {q.chunks, q.tiles, (float)(seq.n * a.group - (q.chunks - 1) * PAGED_CHUNK_ROWS) / (float)(64 * a.group)};
}
// Sequence i of those that the lanes have.
__device__ __forceinline__ OwnSeq own_of(const OwnSeq& q, int i)
{
    return {__builtin_amdgcn_readlane(q.chunks, i), __builtin_amdgcn_readlane(q.tiles, i), __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, q.head), i))};
}
// How many of the chunks, from the last one on, have more than j pieces when they are cut for so many tiles.
__device__ __forceinline__ int own_layer(const PagedArgs& a, const OwnSeq& q, float length, int j)
{
    if (j == 0) return q.chunks;
    const float y = __builtin_fmaf(-length, (float)j, (float)q.tiles - 0.01f);
    if (y <= 0.f) return 0;
    return 1 + max(0, min(q.chunks - 1, (int)__builtin_fminf(__builtin_ceilf((y - q.head) * (0.25f * a.group)), 1e6f)));
}
constexpr float OWN_WHOLE = 1e9f;               // a length that no chunk is cut for
constexpr int OWN_MOST = 4;                     // sequences of a call, at most
struct OwnCut {
    float length;
    int chunks;
};
// (`all`: the sequences, a lane each; a lane has a length.)
__device__ inline OwnCut own_cut(const PagedArgs& a, const OwnSeq& all, int key_heads, int lane)
{
    int longest = 0, chunks = 0;
    float least = 0.f;                          // tiles of all chunks
    for (int i = 0; i < a.sequences; ++i) {
        const OwnSeq q = own_of(all, i);
        longest = max(longest, q.tiles);
        chunks += q.chunks;
        least += (float)(q.chunks * q.tiles) - max(q.chunks - 1, 0) * (q.head + 2.f / a.group * (q.chunks - 2));
    }
    if (longest <= CHUNK_UNCUT / 64 || chunks * key_heads >= a.chunk_parts) return {OWN_WHOLE, 0};
    const float length = (float)longest * __builtin_amdgcn_exp2f(-0.09375f * (1 + lane));
    const int room = a.chunk_parts / key_heads;
    // (lengths that are too short are not counted out: a chunk has nearly half a piece more than its tiles make)
    int pieces = (float)longest - length > CHUNK_SAVES && length >= CHUNK_LEAST && least + 0.4f * length * chunks <= length * room ? 0 : room + 1;
    for (int i = 0; i < a.sequences; ++i) {
        const OwnSeq q = own_of(all, i);
        for (int j = 0, n; pieces <= room && (n = own_layer(a, q, length, j)) > 0; ++j) pieces += n;
    }
    const unsigned long long fits = __builtin_amdgcn_ballot_w64(pieces <= room);
    if (fits == 0) return {OWN_WHOLE, 0};
    return {__builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, length), 63 - __builtin_clzll(fits))), chunks};
}
__device__ inline ChunkPiece own_numbered(const PagedArgs& a, const OwnSeq& all, float length, int left, int lane)
{
    int number = 0;
    for (int s = 0; s < a.sequences; ++s) {
        const OwnSeq q = own_of(all, s);
        for (int i0 = 0; i0 < q.chunks; i0 += 64) {          // a chunk a lane, the last one first
            const int i = i0 + lane;
            int start = 0, pieces = 0;
            for (int j = 0, n; (n = own_layer(a, q, length, j)) > 0; ++j) {
                start += min(i, n);
                pieces += i < n;
            }
            const unsigned long long here = __builtin_amdgcn_ballot_w64(start <= left && left < start + pieces);
            if (here) {
                const int l = __builtin_ctzll(here);
                return {s, q.chunks - 1 - (i0 + l), left - __builtin_amdgcn_readlane(start, l), __builtin_amdgcn_readlane(pieces, l), number + i0 + l};
            }
        }
        for (int j = 0, n; (n = own_layer(a, q, length, j)) > 0; ++j) left -= n;
        number += q.chunks;
    }
    return {-1, 0, 0, 1, 0};
}

// What a score is multiplied by.  Not zero, where the product of the call's scale and the keys' may be: hidden scores are -infinity.
__device__ __forceinline__ float score_scale(float product) { return product < 0x1p-126f ? 0x1p-126f : product; }

// ---- the sums of a row's weights
//
// The product with V takes the weights rounded to the type of the tokens.  O is divided by the sum of the same rounded weights, so that it is a mean of rows of V and
// the rounding of a row that few keys dominate cancels (divided by the sum of the weights as they are, values of 1 ... 1.06 in bf16 come out up to 5.8e-3 off, where half a step is 3.9e-3); the LSE is
// that of the weights as they are.
template <int DTYPE> __device__ __forceinline__ s16x8 all_ones()
{
    s16x8 x;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = Elem<DTYPE>::ONE;
    return x;
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

// Whether any of the values of a tile in the LDS is not finite (16-bit ones, or E4M3 where C8).
template <int DTYPE, bool C8, int BYTES> __device__ __forceinline__ bool holds_not_finite(const char* tile, int lane)
{
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    unsigned worst[4] = {};
#pragma unroll
    for (int i = 0; i < BYTES / 1024; ++i) {
        const u32x4 w = *reinterpret_cast<const u32x4*>(tile + i * 1024 + lane * 16);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (C8) worst[k] |= (w[k] & 0x7f7f7f7fu) + 0x01010101u;      // (only S.1111.111 carries into the sign)
            else worst[k] = __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, worst[k]), __builtin_bit_cast(u16x2, w[k] & 0x7fff7fffu)));
        }
    }
    bool found = false;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        constexpr unsigned E = DTYPE == 0 ? 0x7c00u : 0x7f80u;
        found |= C8 ? (worst[k] & 0x80808080u) != 0 : (worst[k] & 0xffffu) >= E || worst[k] >> 16 >= E;
    }
    return __builtin_amdgcn_ballot_w64(found) != 0;
}
// Non-finite values of a V^T operand: which halves of w have all exponent bits set, as a mask of the whole halves.
template <int DTYPE> __device__ __forceinline__ unsigned not_finite(unsigned w)
{
    constexpr unsigned E = DTYPE == 0 ? 0x7c00u : 0x7f80u;
    return ((w & E) == E ? 0xffffu : 0u) | ((w >> 16 & E) == E ? 0xffff0000u : 0u);
}

}  // namespace
