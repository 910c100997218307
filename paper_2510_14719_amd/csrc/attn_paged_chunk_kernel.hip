// Attention of chunks of new tokens over a paged cache (include/kv_cache.h), many query rows at a time, for gfx950 (MI355X).
//
// A workgroup takes 256 rows, (token, query head) pairs that share a key head, 32 to a wave, and walks the keys in tiles of 64.  Its two
// groups of four waves (one wave of each on a SIMD) run half a period apart:
//     group A after barrier j:  [U_{j-1}, T_j] on the matrix cores, then C_j on the vector ALU
//     group B after barrier j:  C_j on the vector ALU, then [U_j, T_{j+1}] on the matrix cores
// with T = Q K^T, C = softmax against a running reference, U = P V of a tile, so that one wave of a SIMD streams MFMAs while the other does its softmax.
// Keys and values come by direct-to-LDS copies into a ring of four stages (K tile s + 1 and V tile s are stage s), two tiles ahead; a page has at
// least 16 tokens, so the 8 or 16 rows of a copy lie in one page.
//
// Tiles that some row sees only in part (the diagonal, the end, missing pages) come last or are rare: a loop of their own masks the scores and
// keeps values that are not finite out of the product (see careful_u).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "launch_once.h"
#include "paged_launch.h"
#include "paged_prims.h"

namespace {

constexpr float MOVE_LOG2 = 8.0f;               // the reference moves when a maximum grew by more than this many powers of two
constexpr int NW = 8, BM = PAGED_CHUNK_ROWS, BN = 64, STAGES = 4, QB = 2, KB = BN / 16;
constexpr int AHEAD = 2;                        // LDS operands requested ahead of their MFMA

template <int DTYPE, bool C8, int D, bool OWN>
__global__ __launch_bounds__(NW * 64)
void attn_paged_chunk(PagedArgs a)
{
    typedef Elem<DTYPE> E;
    typedef CachedRows<D, 2, BN> Rows;                       // in the LDS: 16-bit values, whatever the cache holds
    constexpr int KK = D / 32, FB = D / 16, STAGE = 2 * Rows::BYTES;
    constexpr int COLS = D * (C8 ? 1 : 2) / 16 < 8 ? D * (C8 ? 1 : 2) / 16 : 8;          // 16-byte columns of a cached row that a copy takes
    constexpr int PER_PIECE = 64 / COLS;                     // rows of a copy of 64 x 16 bytes
    constexpr int PPW = 2 * BN * D * (C8 ? 1 : 2) / 1024 / NW;           // copies of a stage that a wave issues: 4 (K, K, V, V), 2 (K, V) or 1
    extern __shared__ __attribute__((aligned(1024))) char smem[];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lc = lane & 15, lg = lane >> 4;
    const bool group_b = wave >= NW / 2;

    // ---- which chunk, and which piece of its keys
    const int key_heads = a.heads / a.group, h = blockIdx.x % key_heads;
    int cut_chunks;                             // how many there are, if they are cut
    ChunkPiece mine;
    if constexpr (OWN) {
        const OwnSeq all = own_seq(a, lane);
        const OwnCut cut = own_cut(a, all, key_heads, lane);
        mine = own_numbered(a, all, cut.length, blockIdx.x / key_heads, lane);
        cut_chunks = cut.chunks;
    } else {
        const ChunkSeq first = chunk_seq(a, lane);
        const ChunkCut cut = chunk_cut(a, first, key_heads, lane);
        mine = chunk_numbered(a, first, cut.inverse, blockIdx.x / key_heads, lane);
        cut_chunks = cut.chunks;
    }
    const int s = __builtin_amdgcn_readfirstlane(mine.s), tile = __builtin_amdgcn_readfirstlane(mine.chunk);
    int keys = 0, per = 0;                      // keys of the chunk, of a piece
    SeqRange seq = {0, 0, 0, 0};
    if (s >= 0) {
        seq = seq_range(a.q_start, a.kv_len, s, a.tokens, a.max_q, a.max_kv);
        keys = __builtin_amdgcn_readfirstlane(paged_tile_keys(tile, BM, seq.n, a.group, seq.first, seq.kv, a.causal));
        per = chunk_piece_tiles(mine.pieces, keys) * BN;
    }
    if (threadIdx.x == 0 && a.chunk_parts > 0) {                         // for attn_paged_join_chunks
        if (blockIdx.x == 0) a.chunk_what[a.chunk_parts * 4] = cut_chunks * key_heads;
        if (cut_chunks > 0 && s >= 0 && mine.piece == 0)
            *reinterpret_cast<u32x4*>(a.chunk_what + (mine.number * key_heads + h) * 4) =
                u32x4{(unsigned)s, (unsigned)tile, (unsigned)(per < keys ? (keys + per - 1) / per : 1), blockIdx.x};
    }
    if (s < 0) return;
    const int k0 = __builtin_amdgcn_readfirstlane(mine.piece * per), k1 = __builtin_amdgcn_readfirstlane(min(keys, k0 + per));
    if (mine.piece > 0 && k0 >= keys) return;
    const bool whole = per >= keys;

    // ---- rows of this wave, lane % 16 of each 16-row block
    const int wq0 = tile * BM + wave * (QB * 16);
    s16x8 Qf[QB][KK];
    int last_key[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r = wq0 + qb * 16 + lc, tok = r / a.group, head = h * a.group + r % a.group;
        const bool real = tok < seq.n;
        const int t = seq.q0 + (real ? tok : seq.n - 1);
        const char* const at = a.q + t * a.q_token + head * a.q_head + lg * 16;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) Qf[qb][kk] = *reinterpret_cast<const s16x8*>(at + kk * 64);
        last_key[qb] = a.causal ? min(seq.first + tok, keys - 1) : keys - 1;
    }
    // keys of the split that any row of this wave sees, and those that all of them see, in tiles
    int nt = (k1 - k0 + BN - 1) / BN, nt_w, nt_full;
    {
        const int first_tok = wq0 / a.group, last_tok = min((wq0 + QB * 16 - 1) / a.group, seq.n - 1);
        const int w_end = first_tok >= seq.n ? 0 : a.causal ? min(k1, seq.first + last_tok + 1) : k1;
        const int w_all = a.causal ? min(k1, seq.first + first_tok + 1) : k1;
        nt = max(nt, 0);
        nt_w = w_end > k0 ? (w_end - k0 + BN - 1) / BN : 0;
        nt_full = w_all > k0 ? min((w_all - k0) / BN, nt_w) : 0;
    }
    nt = __builtin_amdgcn_readfirstlane(nt);
    nt_w = __builtin_amdgcn_readfirstlane(nt_w);
    nt_full = __builtin_amdgcn_readfirstlane(nt_full);

    const float scale = score_scale(a.scale * (C8 && a.k_scale ? a.k_scale[h] : 1.f)), c = scale * 1.4426950408889634f;
    const float m_none = c > 1.f ? -0x1.fffff0p127f / c : -__FLT_MAX__;  // (the most negative float whose scaled value is finite)

    // ---- copies.  A wave's pieces are rows of one 16-key block of the tile and one 128-byte group of a row.
    const bool copies_k = PPW > 1 || wave < NW / 2, copies_v = PPW > 1 || wave >= NW / 2;
    const int block = PPW == 2 ? wave >> 1 : wave & 3;       // 16-key block
    const int group = PPW == 4 ? wave >> 2 : 0;
    constexpr int SUBS = PPW == 4 ? 2 : 1;                   // pieces of K (and of V)
    const int sub0 = PPW == 2 ? wave & 1 : 0;
    unsigned k_off[SUBS], v_off[SUBS];                       // source offsets of the lane inside 16 whole rows
    int piece_row[SUBS];                                     // row of the lane among the 16
#pragma unroll
    for (int i = 0; i < SUBS; ++i) {
        const int r = (sub0 + i) * PER_PIECE + lane / COLS, col = lane % COLS;
        piece_row[i] = r;
        k_off[i] = (unsigned)((C8 ? col : col ^ Rows::sw_k(block * 16 + r)) * 16 + group * 128) + r * (unsigned)a.token_bytes;
        v_off[i] = (unsigned)((C8 ? col : col ^ Rows::sw_v(block * 16 + r)) * 16 + group * 128) + r * (unsigned)a.token_bytes;
    }
    const unsigned lds = (unsigned)(size_t)(LDS_AS void*)smem;
    const int to0 = group * (BN * Rows::LINE) + (block * 16 + sub0 * PER_PIECE) * Rows::LINE;
    const int* const table = a.table + (long long)s * a.table_stride;
    const int page_mask = (1 << a.page_shift) - 1, token_bytes = (int)a.token_bytes;
    const long long k_base = reinterpret_cast<long long>(uniform_ptr(a.k + h * a.head_bytes)), v_minus_k = reinterpret_cast<long long>(uniform_ptr(a.v)) - reinterpret_cast<long long>(uniform_ptr(a.k));
    const int inside = __builtin_amdgcn_readfirstlane(keys - 16 - block * 16 - k0 < 0 ? 0 : (keys - 16 - block * 16 - k0) / BN + 1);   // tiles whose 16 keys all exist
    // Lane i: where the first of this wave's keys of tile i of the current 64 stands in K.  (Addresses are worked out for 64 tiles at a time: with every tile for itself a
    // wave was held 500 cycles by its copies, of 3100 a tile; 4096 new tokens of 16384, 32 heads on 8, d 128: 769 us that way, 753 so.)
    unsigned place_lo = 0, place_hi = 0;
    bool any_bad = false;                       // a page of the tiles so far is none
    auto load_places = [&](int t0) __attribute__((always_inline)) {
        const int key = k0 + (t0 + lane) * BN, first_key = min(key + block * 16, keys - 1);
        bool bad = false;
#pragma unroll
        for (int b = 0; b < KB; ++b) bad |= (unsigned)table[min(key + b * 16, keys - 1) >> a.page_shift] >= (unsigned)a.pages;
        any_bad |= __builtin_amdgcn_ballot_w64(bad) != 0;
        int page = table[first_key >> a.page_shift];
        page = (unsigned)page < (unsigned)a.pages ? page : 0;
        const unsigned long long place = k_base + page * a.page_bytes + (first_key & page_mask) * token_bytes;
        place_lo = (unsigned)place;
        place_hi = (unsigned)(place >> 32);
    };
    unsigned long long place_k = 0, place_v = 0;             // of the K tile of the stage; in K too, of its V tile
    // Where the lane's 16 bytes of piece i stand, in tile t of K or V (rows behind the last key: that one again; they are masked, or never read).
    auto source = [&](unsigned long long place, int t, const unsigned (&off)[SUBS], int i, unsigned& lane_off) __attribute__((always_inline)) -> const char* {
        lane_off = off[i];
        const char* base = reinterpret_cast<const char*>(place);
        if (t >= inside) {
            const int key = k0 + min(t, nt - 1) * BN + block * 16;
            base -= (min(key, keys - 1) & page_mask) * token_bytes;
            lane_off += (unsigned)(((min(key + piece_row[i], keys - 1) & page_mask) - piece_row[i]) * token_bytes);
        }
        return base;
    };
    // Moves on to the K tile of stage st (in order, from -1 on) and the V tile of the same stage.
    auto advance = [&](int st) __attribute__((always_inline)) {
        const int t = st + 1;
        place_v = place_k;
        if (t < nt) {
            if ((t & 63) == 0) load_places(t);
            place_k = (unsigned)__builtin_amdgcn_readlane(place_lo, t & 63) | (unsigned long long)(unsigned)__builtin_amdgcn_readlane(place_hi, t & 63) << 32;
        }
    };
    // A 16-bit cache: straight into the LDS.
    auto issue_stage = [&](int st) __attribute__((always_inline)) {
        advance(st);
        const unsigned dst = lds + ((st + STAGES) % STAGES) * STAGE + to0;
        // (behind the last tile, and before the first, something is copied all the same: the waits count copies)
#pragma unroll
        for (int i = 0; i < SUBS; ++i) {
            unsigned off;
            const char* const from = source(place_k, st + 1, k_off, i, off);
            dma16(from, off, dst + i * (PER_PIECE * Rows::LINE));
        }
#pragma unroll
        for (int i = 0; i < SUBS; ++i) {
            unsigned off;
            const char* const from = source((st < 0 ? place_k : place_v) + v_minus_k, max(st, 0), v_off, i, off);
            dma16(from, off, dst + Rows::BYTES + i * (PER_PIECE * Rows::LINE));
        }
    };
    // An 8-bit cache: into registers a stage ahead, widened once and written to the LDS (widened by every wave as it reads, the same values take the vector ALU longer
    // than the products take the matrix cores: 4096 new tokens of 16384, 32 heads on 8, d 128: 1015 us that way, 848 so, and 885 with the sums of the rounded weights).
    u32x4 raw_k, raw_v;
    auto fetch_stage = [&](int st) __attribute__((always_inline)) {
        advance(st);
        unsigned off;
        if (copies_k) {
            const char* const from = source(place_k, st + 1, k_off, 0, off);
            raw_k = *reinterpret_cast<const u32x4*>(from + off);
        }
        if (copies_v) {
            const char* const from = source((st < 0 ? place_k : place_v) + v_minus_k, max(st, 0), v_off, 0, off);
            raw_v = *reinterpret_cast<const u32x4*>(from + off);
        }
    };
    auto write_stage = [&](int st) __attribute__((always_inline)) {
        char* const dst = smem + ((st + STAGES) % STAGES) * STAGE;
        const int r = block * 16 + piece_row[0], byte = lane % COLS * 32, line = byte / Rows::LINE, col = byte % Rows::LINE / 16;
        char* const to = dst + line * (BN * Rows::LINE) + r * Rows::LINE;
        if (copies_k) {
            *reinterpret_cast<s16x8*>(to + (col ^ Rows::sw_k(r)) * 16) = widen8<DTYPE>(u32x2{raw_k[0], raw_k[1]});
            *reinterpret_cast<s16x8*>(to + ((col + 1) ^ Rows::sw_k(r)) * 16) = widen8<DTYPE>(u32x2{raw_k[2], raw_k[3]});
        }
        if (copies_v) {
            *reinterpret_cast<s16x8*>(to + Rows::BYTES + (col ^ Rows::sw_v(r)) * 16) = widen8<DTYPE>(u32x2{raw_v[0], raw_v[1]});
            *reinterpret_cast<s16x8*>(to + Rows::BYTES + ((col + 1) ^ Rows::sw_v(r)) * 16) = widen8<DTYPE>(u32x2{raw_v[2], raw_v[3]});
        }
    };
    // At barrier j every wave's share of stages <= j has landed (8 bits: of stages <= j + 1) and nobody reads stage j - 2 any more, so that stage takes
    // stage j + 2.
    auto wait_stage = [&](int j) __attribute__((always_inline)) {
        if (C8) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        else if (j + 1 < nt) wait_vmcnt<PPW>();
        else wait_vmcnt<0>();
        __builtin_amdgcn_s_barrier();
    };
    auto next = [&](int j) __attribute__((always_inline)) {
        if (j + 2 >= nt) return;
        if constexpr (C8) {
            write_stage(j + 2);
            if (j + 3 < nt) fetch_stage(j + 3);
        } else {
            issue_stage(j + 2);
        }
    };
    auto stage_ptr = [&](int st) __attribute__((always_inline)) -> const char* { return smem + ((st + STAGES) % STAGES) * STAGE; };

    f32x4 O[FB][QB], S[KB][QB];
    u32x4 pw[KB / 2][QB];
    float m_run[QB], neg_mc[QB], L[QB];
    // Sums of the rounded weights, from the matrix cores: the first element.  (4096 new tokens of 16384, 32 heads on 8, d 128, us: without them 778, so 781 ... 799, with vector instructions
    // 825; d 64, 4096 of 8192: 234 / 242 / 272.)
    f32x4 R[QB];
    const s16x8 ones = all_ones<DTYPE>();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        m_run[qb] = m_none;
        neg_mc[qb] = -m_none * c;
        L[qb] = 0.f;
        R[qb] = f32x4(0.f);
#pragma unroll
        for (int fb = 0; fb < FB; ++fb) O[fb][qb] = f32x4(0.f);
    }

    // ---- U and / or T on one stage as one stream of MFMAs, operands requested AHEAD MFMAs before their use
    auto burst = [&](auto do_u, auto do_t, const char* st) __attribute__((always_inline)) {
        constexpr int NU = decltype(do_u)::value ? KB / 2 * FB : 0, NT = decltype(do_t)::value ? KB * KK : 0, NF = NU + NT;
        s16x8 fr[NF];
        auto fetch = [&](int f) __attribute__((always_inline)) {
            if (f < NU) fr[f] = Rows::template v_operand<DTYPE>(st + Rows::BYTES, f / FB, f % FB, lane);
            else fr[f] = Rows::template k_operand<DTYPE>(st, (f - NU) % KB, (f - NU) / KB, lane);
        };
#pragma unroll
        for (int f = 0; f < AHEAD; ++f) fetch(f);
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            if (f + AHEAD < NF) fetch(f + AHEAD);
            if (f < NU) {
                if (f % FB == FB - 1) {
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) R[qb] = E::mfma16(ones, __builtin_bit_cast(s16x8, pw[f / FB][qb]), R[qb]);
                }
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) O[f % FB][qb] = E::mfma16(fr[f], __builtin_bit_cast(s16x8, pw[f / FB][qb]), O[f % FB][qb]);
            } else {
                const int kb = (f - NU) % KB, kk = (f - NU) / KB;
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) S[kb][qb] = E::mfma16(fr[f], Qf[qb][kk], kk == 0 ? f32x4(0.f) : S[kb][qb]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // The 16-key blocks of a tile that lie in no page.
    auto no_pages = [&](int j) __attribute__((always_inline)) {
        unsigned bad = 0;
        if (any_bad) {
#pragma unroll
            for (int b = 0; b < KB; ++b)
                bad |= (unsigned)__builtin_amdgcn_readfirstlane(table[min(k0 + j * BN + b * 16, keys - 1) >> a.page_shift]) >= (unsigned)a.pages ? 1u << b : 0u;
        }
        return bad;
    };
    // ---- U of a tile that some row may see in part.  Where it holds values that are not finite, 0 x NaN would be NaN: these stay out of the product and are
    // added key by key to the rows that see them, whatever their weight, as the product does where every row sees every key.  (Looking for them costs a wave 16 LDS reads and 140 vector instructions; taking them out
    // always, 1300 a tile: 256 new tokens of 256, 16 heads, d 128, by chunks 16.8 us that way, 15.2 so.)
    auto careful_u = [&](int j) __attribute__((always_inline)) {
        const char* const vt = stage_ptr(j) + Rows::BYTES;
        const bool care = (j >= nt_full || any_bad) && holds_not_finite<DTYPE, false, Rows::BYTES>(vt, lane);
#pragma unroll
        for (int kc = 0; kc < KB / 2; ++kc)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) R[qb] = E::mfma16(ones, __builtin_bit_cast(s16x8, pw[kc][qb]), R[qb]);
#pragma unroll
        for (int kc = 0; kc < KB / 2; ++kc)
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                u32x4 w = __builtin_bit_cast(u32x4, Rows::template v_operand<DTYPE>(vt, kc, fb, lane));
                if (care) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) w[t] &= ~not_finite<DTYPE>(w[t]);
                }
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) O[fb][qb] = E::mfma16(__builtin_bit_cast(s16x8, w), __builtin_bit_cast(s16x8, pw[kc][qb]), O[fb][qb]);
            }
        if (!care) return;
        const unsigned bad = no_pages(j);
        for (int k = 0; k < BN; ++k) {
            float p[QB];
            bool seen[QB];
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                seen[qb] = k0 + j * BN + k <= last_key[qb] && !((bad >> (k >> 4)) & 1);
                unsigned x = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) x = (k >> 3 & 4) + (k >> 1 & 3) == e ? pw[e / 4][qb][e % 4] : x;
                x = __shfl(x, (k >> 3 & 3) * 16 + lc);
                p[qb] = to_float<DTYPE>((uint16_t)(k & 1 ? x >> 16 : x));
            }
#pragma unroll
            for (int fb = 0; fb < FB; ++fb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = Rows::template v_value<DTYPE>(vt, k, fb * 16 + lg * 4 + i);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb) O[fb][qb][i] += __builtin_isfinite(x) || !seen[qb] ? 0.f : p[qb] * x;
                }
        }
    };

    // ---- C of tile j: S into pw
    auto softmax_tile = [&](int j, auto masked) __attribute__((always_inline)) {
        if (decltype(masked)::value) {
            const int key0 = k0 + j * BN;
            const unsigned bad = no_pages(j);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    const int lim = (bad >> ((kb >> 1) * 2 + (lg >> 1))) & 1 ? -1 : last_key[qb];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key0 + (kb >> 1) * 32 + lg * 8 + (kb & 1) * 4 + i > lim) S[kb][qb][i] = -__builtin_inff();
                }
        }
        float mx[QB];
        bool over = false;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            mx[qb] = S[0][qb][0];
#pragma unroll
            for (int e = 1; e < 4 * KB; ++e) mx[qb] = __builtin_fmaxf(mx[qb], S[e / 4][qb][e % 4]);
            over |= __builtin_fmaf(mx[qb], c, neg_mc[qb]) > MOVE_LOG2;
        }
        if (__builtin_amdgcn_ballot_w64(over) != 0) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const float m_old = m_run[qb];
                m_run[qb] = groups_max(__builtin_fmaxf(mx[qb], m_old));
                neg_mc[qb] = -m_run[qb] * c;
                const float alpha = __builtin_amdgcn_exp2f((m_old - m_run[qb]) * c);
                L[qb] *= alpha;
                R[qb][0] *= alpha;
#pragma unroll
                for (int fb = 0; fb < FB; ++fb) O[fb][qb] = O[fb][qb] * alpha;
            }
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[kb][qb][2 * t], c, neg_mc[qb]));
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(S[kb][qb][2 * t + 1], c, neg_mc[qb]));
                    L[qb] += p0;
                    L[qb] += p1;
                    pw[kb / 2][qb][kb % 2 * 2 + t] = E::pack2(p0, p1);
                }
    };

    // ---- the walk
    constexpr std::true_type YES{};
    constexpr std::false_type NO{};
    if (nt > 0) {
#pragma unroll
        for (int st = -1; st < 2; ++st) {
            if constexpr (C8) {
                fetch_stage(st);
                write_stage(st);
            } else {
                issue_stage(st);
            }
        }
        if constexpr (C8) {
            if (2 < nt) fetch_stage(2);
        }
    }
    // (Q is used once here, so that the compiler waits for its loads before the loop, and with them for the copies)
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) asm volatile("" :: "v"(Qf[qb][kk]));
    if (C8) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    else wait_vmcnt<0>();
    __builtin_amdgcn_s_barrier();
    // (the last tile of a wave is none of these: it is always done with care)
    auto whole_tiles = [&](int j) __attribute__((always_inline)) { return j < nt_full && j + 1 < nt_w && !any_bad; };
    if (nt_w == 0) {                            // no row of this wave sees a key of the split: it only copies
        for (int j = 0; j < nt; ++j) {
            wait_stage(j);
            next(j);
        }
    } else if (!group_b) {
        wait_stage(0);
        burst(NO, YES, stage_ptr(-1));                                   // T_0
        next(0);
        int j = 0;                              // C_j is next
        if (whole_tiles(0)) {
            do {                                // (bottom-tested, here and below: the accumulators stay in place)
                softmax_tile(j, NO);
                wait_stage(++j);
                burst(YES, YES, stage_ptr(j - 1));
                next(j);
            } while (whole_tiles(j));
        }
        do {
            softmax_tile(j, YES);
            if (++j < nt) wait_stage(j);
            careful_u(j - 1);
            if (j < nt_w) burst(NO, YES, stage_ptr(j - 1));
            next(j);
        } while (j < nt_w);
        for (++j; j < nt; ++j) {
            wait_stage(j);
            next(j);
        }
    } else {
        burst(NO, YES, stage_ptr(-1));                                   // T_0
        int j = 0;
        if (whole_tiles(0)) {
            do {
                wait_stage(j);
                next(j);
                softmax_tile(j, NO);
                burst(YES, YES, stage_ptr(j));
            } while (whole_tiles(++j));
        }
        do {
            wait_stage(j);
            next(j);
            softmax_tile(j, YES);
            careful_u(j);
            if (j + 1 < nt_w) burst(NO, YES, stage_ptr(j));
        } while (++j < nt_w);
        for (; j < nt; ++j) {
            wait_stage(j);
            next(j);
        }
    }

    // ---- results
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        L[qb] = groups_sum(L[qb]);
        const int r = wq0 + qb * 16 + lc, tok = r / a.group, head = h * a.group + r % a.group, t = seq.q0 + tok;
        if (tok >= seq.n) continue;
        const long long row = (long long)t * a.heads + head;
        if (whole) {
            const float inv = (R[qb][0] == 0.f ? 0.f : 1.f / R[qb][0]) * (C8 && a.v_scale ? a.v_scale[h] : 1.f);
            char* const to = a.o + t * a.o_token + head * a.o_head + lg * 8;
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                const f32x4 x = O[fb][qb] * inv;
                *reinterpret_cast<u32x2*>(to + fb * 32) = u32x2{E::pack2(x[0], x[1]), E::pack2(x[2], x[3])};
            }
            if (a.lse && lg == 0) a.lse[row] = m_run[qb] * scale + __builtin_logf(L[qb]);
        } else {
            const long long at = (long long)blockIdx.x * BM + r % BM;
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) *reinterpret_cast<f32x4*>(a.chunk_o + at * D + fb * 16 + lg * 4) = O[fb][qb];
            if (lg == 0) *reinterpret_cast<f32x4*>(a.chunk_ml + at * 4) = f32x4{m_run[qb] * c, L[qb], R[qb][0], 0.f};
        }
    }
}

template <int DTYPE, bool C8, int D, bool OWN>
int launch_as(const PagedArgs& a, const PagedPlan& plan, hipStream_t stream)
{
    constexpr int SMEM = STAGES * 2 * CachedRows<D, 2, BN>::BYTES;
    auto kern = attn_paged_chunk<DTYPE, C8, D, OWN>;
    static PerDeviceOnce once;
    if (once.prepare(reinterpret_cast<const void*>(kern), SMEM) < 0) return -1;
    PagedArgs arg = a;
    void* args[] = {&arg};
    const long long grid = plan.chunk_tiles > a.chunk_parts ? plan.chunk_tiles : a.chunk_parts;
    return hipLaunchKernel(reinterpret_cast<const void*>(kern), dim3((unsigned)grid), dim3(NW * 64), args, SMEM, stream) == hipSuccess ? 0 : -1;
}

// Whether chunks are cut for the keys that they see themselves: prompts of a few sequences (finding out takes longer the more there are; 6 of up to 1040 tokens, 5 heads on 1, E4M3, d 64 25 us
// without, 29 with) whose chunks differ, the first seeing at least a quarter fewer keys than the last (each has 256 / group tokens more than the one before), and are fewer than the compute
// units.  us without / with, 16-bit: one prompt of 2048, 16 heads, d 128 49.0 / 43.2, of 4096, 8 heads 71.3 / 59.0, of 3000, 16 on 2 81.6 / 70.3; two of 1326, 20 on 4, d 64 61.7 / 62.0 (the
// gain is lost to the longer way of finding out; over E4M3 68.7 / 71.4, the most that it costs).
template <int DTYPE, bool C8, int D>
int launch(const PagedArgs& a, const PagedPlan& plan, hipStream_t stream)
{
    const long long chunks = ((long long)a.max_q * a.group + BM - 1) / BM, all = (long long)a.tokens * a.group / BM + a.sequences, tiles = a.max_kv / 64;
    const bool own = a.causal && a.chunk_parts > 0 && a.sequences <= OWN_MOST && chunks >= 4 && 16 * (chunks - 1) >= a.group * tiles && (all - a.sequences) * (a.heads / a.group) < a.chunk_parts;
    return own ? launch_as<DTYPE, C8, D, true>(a, plan, stream) : launch_as<DTYPE, C8, D, false>(a, plan, stream);
}

}  // namespace

int attn_paged_chunk_launch(const PagedArgs& a, const PagedPlan& plan, int d, int dtype, int cache_dtype, void* stream)
{
    const hipStream_t st = (hipStream_t)stream;
    if (cache_dtype == KV_E4M3) {
        if (dtype == 0) return d == 128 ? launch<0, true, 128>(a, plan, st) : launch<0, true, 64>(a, plan, st);
        return d == 128 ? launch<1, true, 128>(a, plan, st) : launch<1, true, 64>(a, plan, st);
    }
    if (dtype == 0) return d == 128 ? launch<0, false, 128>(a, plan, st) : launch<0, false, 64>(a, plan, st);
    return d == 128 ? launch<1, false, 128>(a, plan, st) : launch<1, false, 64>(a, plan, st);
}
