// Attention of a packed batch of new tokens over a paged cache (include/kv_cache.h), for gfx950 (MI355X).
//
// The rows of a workgroup are (token, query head) pairs that share a key head, so every cached row that comes in serves all of them.
// The waves of a workgroup work on the same rows and share out the keys: each walks 32 keys at a time with a softmax state of its own
// (running reference, sum, O), and the states are joined through the LDS at the end.  Nothing waits for another wave before that.  Rows
// that have few workgroups are also cut along the keys into splits; attn_paged_join joins their results.
//
// A wave's keys and values come by direct-to-LDS copies into a ring of its own, one step ahead.  Pages have at least 16
// tokens, so 16 consecutive keys lie in one page and their address is a scalar.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "launch_once.h"
#include "paged_launch.h"
#include "paged_prims.h"

namespace {

// The softmax reference moves only when a row maximum grew by more than this many powers of two.
constexpr float MOVE_LOG2 = 8.0f;
constexpr int NW = 4;                           // waves of a workgroup

template <int D, int ES, int QB> struct FewLayout {
    typedef CachedRows<D, ES, 32> Rows;
    static constexpr int STAGE = 2 * Rows::BYTES, SLOTS = 2;
    static constexpr int JOIN = NW * (D / 16) * QB * 1024;   // O of every wave
    static constexpr int SUMS = NW * QB * 16 * 16;           // first: reference and sums of every wave's rows
    static constexpr int smem(int stages) { return SUMS + (stages * STAGE > JOIN ? stages * STAGE : JOIN); }
};

template <int DTYPE, bool C8, int D, int QB>
__global__ __launch_bounds__(NW * 64)
void attn_paged_few(PagedArgs a)
{
    typedef Elem<DTYPE> E;
    typedef FewLayout<D, C8 ? 1 : 2, QB> Layout;
    typedef typename Layout::Rows Rows;
    constexpr int KK = D / 32, FB = D / 16, ROWS = QB * 16;
    constexpr int SUBS = 16 / Rows::PER_PIECE;               // pieces of 16 keys and a line of their rows
    constexpr int PIECES = 2 * Rows::BYTES / 1024;           // copies of a step
    extern __shared__ __attribute__((aligned(1024))) char smem[];

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, lc = lane & 15, lg = lane >> 4;
    const int key_heads = a.heads / a.group;
    int id = blockIdx.x;
    const int h = id % key_heads;
    id /= key_heads;
    FewPiece mine;
    if (a.few_room > 0) {
        const SeqRange first = few_seq(a, lane);
        const float inverse = few_cut(a, first, lane);
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.few_inverse = inverse;
        mine = few_numbered(a, first, inverse, id, lane);
        if (mine.s < 0) return;
    } else {
        mine.piece = id % a.splits;
        id /= a.splits;
        mine.tile = a.row_tiles - 1 - id % a.row_tiles;
        mine.s = id / a.row_tiles;
        mine.pieces = 0;
        mine.seq = seq_range(a.q_start, a.kv_len, mine.s, a.tokens, a.max_q, a.max_kv);
    }
    const int s = __builtin_amdgcn_readfirstlane(mine.s), tile = __builtin_amdgcn_readfirstlane(mine.tile), sp = __builtin_amdgcn_readfirstlane(mine.piece);
    const SeqRange seq = {__builtin_amdgcn_readfirstlane(mine.seq.q0), __builtin_amdgcn_readfirstlane(mine.seq.n), __builtin_amdgcn_readfirstlane(mine.seq.kv), __builtin_amdgcn_readfirstlane(mine.seq.first)};
    if (tile * ROWS >= seq.n * a.group || seq.n * a.group > a.few_rows) return;
    const int keys = paged_tile_keys(tile, ROWS, seq.n, a.group, seq.first, seq.kv, a.causal), per = a.few_room > 0 ? few_piece_keys(mine.pieces, keys) : paged_piece_keys(keys, a.split);
    const int k0 = sp * per, k1 = min(keys, k0 + per);
    if (sp > 0 && k0 >= keys) return;
    const bool whole = keys <= per;
    if (a.few_first && sp == 0 && h == 0 && threadIdx.x == 0) a.few_first[s * a.row_tiles + tile] = blockIdx.x / key_heads;

    // ---- the wave's steps are 32 keys each, every NW-th of the piece's
    const int* const table = a.table + (long long)s * a.table_stride;
    auto entries_of = [&](int step) __attribute__((always_inline)) {     // lane 2 i + hf: page of half hf of the i-th step from here
        const int key = max(min(k0 + ((step + (lane >> 1)) * NW + wave) * 32 + (lane & 1) * 16, keys - 1), 0);
        return table[key >> a.page_shift];
    };
    int entries = entries_of(0);

    // ---- rows: lane % 16 of each 16-row block
    s16x8 Qf[QB][KK];
    int last_key[QB];                           // the last key that the row sees
    long long o_row[QB];                        // token * heads + head, -1 behind the last row
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int r = tile * ROWS + qb * 16 + lc, tok = r / a.group, head = h * a.group + r % a.group;
        const bool real = tok < seq.n;
        const int t = seq.q0 + (real ? tok : seq.n - 1);
        const char* const at = a.q + t * a.q_token + head * a.q_head + lg * 16;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) Qf[qb][kk] = *reinterpret_cast<const s16x8*>(at + kk * 64);
        last_key[qb] = a.causal ? min(seq.first + tok, keys - 1) : keys - 1;
        o_row[qb] = real ? (long long)t * a.heads + head : -1;
    }
    const int first_last = a.causal ? seq.first + tile * ROWS / a.group : keys - 1;   // what the first row sees

    const float scale = score_scale(a.scale * (C8 && a.k_scale ? a.k_scale[h] : 1.f)), c = scale * 1.4426950408889634f;
    // The reference before the first score: the most negative float whose scaled value is finite.  (-inf would make NaN of rows whose
    // first keys are hidden.)
    const float m_none = c > 1.f ? -0x1.fffff0p127f / c : -__FLT_MAX__;
    f32x4 O[FB][QB];
    // Sums of the weights: as they are, for the LSE, and as the product with V takes them, rounded, for O (see paged_prims.h).  The latter comes from the matrix cores,
    // a block of ones in the place of V^T; its first element is read.
    float m_run[QB], neg_mc[QB], L[QB];
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

    const int blocks = (k1 - k0 + 31) / 32, steps = blocks > wave ? (blocks - wave + NW - 1) / NW : 0;
    const int page_mask = (1 << a.page_shift) - 1;
    // per-lane source offsets of a copy inside 16 keys: row and (permuted) column
    unsigned k_off[2][SUBS], v_off[2][SUBS];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub) {
            const int r = sub * Rows::PER_PIECE + lane / Rows::COLS, col = lane % Rows::COLS;
            k_off[hf][sub] = (unsigned)(r * a.token_bytes) + ((col ^ Rows::sw_k(hf * 16 + r)) * 16);
            v_off[hf][sub] = (unsigned)(r * a.token_bytes) + ((col ^ Rows::sw_v(hf * 16 + r)) * 16);
        }
    const char* const ring = smem + Layout::SUMS + wave * Layout::STAGE;        // slot-major: a short piece uses the first stages only
    const char* const kh = uniform_ptr(a.k + h * a.head_bytes);
    const char* const vh = uniform_ptr(a.v + h * a.head_bytes);
    auto issue = [&](int step) __attribute__((always_inline)) -> unsigned {      // the halves of the step that lie in no page
        const unsigned dst = (unsigned)(size_t)(LDS_AS const void*)(ring + (step & 1) * (NW * Layout::STAGE));
        const int key = k0 + (step * NW + wave) * 32;
        unsigned bad = 0;
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const int k_half = key + hf * 16;
            // (a half behind the last key takes the other one's page: the last key's)
            int page = __builtin_amdgcn_readlane(entries, (step & 31) * 2 + (k_half < keys ? hf : 0));
            if ((unsigned)page >= (unsigned)a.pages) {
                page = 0;
                bad |= 1u << hf;
            }
            long long off = page * a.page_bytes;
            if (k_half + 16 <= keys) {
                off += (k_half & page_mask) * a.token_bytes;
#pragma unroll
                for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
                    for (int g = 0; g < Rows::GROUPS; ++g) {
                        const unsigned to = dst + g * (32 * Rows::LINE) + (hf * 16 + sub * Rows::PER_PIECE) * Rows::LINE;
                        dma16(kh + off + g * 128, k_off[hf][sub], to);
                        dma16(vh + off + g * 128, v_off[hf][sub], to + Rows::BYTES);
                    }
            } else {                            // rows behind the last key: that one again (they are masked)
#pragma unroll
                for (int sub = 0; sub < SUBS; ++sub) {
                    const int r = sub * Rows::PER_PIECE + lane / Rows::COLS, col = lane % Rows::COLS;
                    const unsigned row = (unsigned)((min(k_half + r, keys - 1) & page_mask) * a.token_bytes);
                    const unsigned ko = row + ((col ^ Rows::sw_k(hf * 16 + r)) * 16), vo = row + ((col ^ Rows::sw_v(hf * 16 + r)) * 16);
#pragma unroll
                    for (int g = 0; g < Rows::GROUPS; ++g) {
                        const unsigned to = dst + g * (32 * Rows::LINE) + (hf * 16 + sub * Rows::PER_PIECE) * Rows::LINE;
                        dma16(kh + off + g * 128, ko, to);
                        dma16(vh + off + g * 128, vo, to + Rows::BYTES);
                    }
                }
            }
        }
        return bad;
    };

    // Q is used once here, so that the compiler waits for its loads before the first copy and not for all copies later.
#pragma unroll
    for (int qb = 0; qb < QB; ++qb)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) asm volatile("" :: "v"(Qf[qb][kk]));
    unsigned bad = steps > 0 ? issue(0) : 0, bad_next = steps > 1 ? issue(1) : 0;

    for (int step = 0; step < steps; ++step) {
        if (step + 1 < steps) wait_vmcnt<PIECES>(); else wait_vmcnt<0>();
        const char* const kt = ring + (step & 1) * (NW * Layout::STAGE);
        const char* const vt = kt + Rows::BYTES;
        const int key = k0 + (step * NW + wave) * 32;
        f32x4 S[2][QB];
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const s16x8 kf = Rows::template k_operand<DTYPE>(kt, kb, kk, lane);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) S[kb][qb] = E::mfma16(kf, Qf[qb][kk], kk == 0 ? f32x4(0.f) : S[kb][qb]);
            }
        const bool masked = bad != 0 || key + 32 > keys || key + 31 > first_last;
        if (masked) {
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                const int lim = (bad >> (lg >> 1)) & 1 ? -1 : last_key[qb];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key + lg * 8 + kb * 4 + i > lim) S[kb][qb][i] = -__builtin_inff();
            }
        }
        u32x4 P[QB];
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            float mx = S[0][qb][0];
#pragma unroll
            for (int e = 1; e < 8; ++e) mx = __builtin_fmaxf(mx, S[e / 4][qb][e % 4]);
            if (__builtin_amdgcn_ballot_w64(__builtin_fmaf(mx, c, neg_mc[qb]) > MOVE_LOG2) != 0) {
                const float m_old = m_run[qb];
                m_run[qb] = groups_max(__builtin_fmaxf(mx, m_old));
                neg_mc[qb] = -m_run[qb] * c;
                const float alpha = __builtin_amdgcn_exp2f((m_old - m_run[qb]) * c);
                L[qb] *= alpha;
                R[qb][0] *= alpha;
#pragma unroll
                for (int fb = 0; fb < FB; ++fb) O[fb][qb] = O[fb][qb] * alpha;
            }
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    S[kb][qb][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[kb][qb][i], c, neg_mc[qb]));
                    L[qb] += S[kb][qb][i];
                }
#pragma unroll
            for (int t = 0; t < 4; ++t) P[qb][t] = E::pack2(S[t / 2][qb][t % 2 * 2], S[t / 2][qb][t % 2 * 2 + 1]);
            R[qb] = E::mfma16(ones, __builtin_bit_cast(s16x8, P[qb]), R[qb]);
        }
        if (!masked || !holds_not_finite<DTYPE, C8, Rows::BYTES>(vt, lane)) {
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                const s16x8 vf = Rows::template v_operand<DTYPE>(vt, 0, fb, lane);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) O[fb][qb] = E::mfma16(vf, __builtin_bit_cast(s16x8, P[qb]), O[fb][qb]);
            }
        } else {
            // Where some row does not see some key, 0 x NaN would be NaN: there, values that are not finite stay out of the product and
            // are added key by key to the rows that see them, whatever their weight, as the product does where every row sees every key.
#pragma unroll
            for (int fb = 0; fb < FB; ++fb) {
                u32x4 w = __builtin_bit_cast(u32x4, Rows::template v_operand<DTYPE>(vt, 0, fb, lane));
#pragma unroll
                for (int t = 0; t < 4; ++t) w[t] &= ~not_finite<DTYPE>(w[t]);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) O[fb][qb] = E::mfma16(__builtin_bit_cast(s16x8, w), __builtin_bit_cast(s16x8, P[qb]), O[fb][qb]);
            }
            for (int j = 0; j < 32; ++j) {
                float p[QB];
                bool seen[QB];
#pragma unroll
                for (int qb = 0; qb < QB; ++qb) {
                    seen[qb] = key + j <= last_key[qb] && !((bad >> (j >> 4)) & 1);
                    float x = S[0][qb][0];
#pragma unroll
                    for (int e = 1; e < 8; ++e) x = (j & 7) == e ? S[e / 4][qb][e % 4] : x;
                    p[qb] = __shfl(x, (j >> 3) * 16 + lc);
                }
#pragma unroll
                for (int fb = 0; fb < FB; ++fb)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float x = Rows::template v_value<DTYPE>(vt, j, fb * 16 + lg * 4 + i);
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb) O[fb][qb][i] += __builtin_isfinite(x) || !seen[qb] ? 0.f : p[qb] * x;
                    }
            }
        }
        bad = bad_next;
        if (step + 2 < steps) {
            if (((step + 2) & 31) == 0) entries = entries_of(step + 2);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");           // every read of the slot is done
            bad_next = issue(step + 2);
        }
    }

    // ---- join the waves: each takes its share of the features
    float* const sums = reinterpret_cast<float*>(smem);
    char* const join = smem + Layout::SUMS;
    __syncthreads();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        L[qb] = groups_sum(L[qb]);
#pragma unroll
        for (int fb = 0; fb < FB; ++fb) *reinterpret_cast<f32x4*>(join + ((wave * FB + fb) * QB + qb) * 1024 + lane * 16) = O[fb][qb];
        if (lg == 0) *reinterpret_cast<f32x4*>(sums + ((wave * QB + qb) * 16 + lc) * 4) = f32x4{m_run[qb], L[qb], R[qb][0], 0.f};
    }
    __syncthreads();
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        f32x4 ml[NW];
        float m = m_none, l = 0.f, rounded = 0.f, w[NW];
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            ml[v] = *reinterpret_cast<const f32x4*>(sums + ((v * QB + qb) * 16 + lc) * 4);
            m = __builtin_fmaxf(m, ml[v][0]);
        }
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            w[v] = __builtin_amdgcn_exp2f((ml[v][0] - m) * c);
            l += ml[v][1] * w[v];
            rounded += ml[v][2] * w[v];
        }
        const bool real = o_row[qb] >= 0;
        const int t = real ? (int)(o_row[qb] / a.heads) : 0, head = real ? (int)(o_row[qb] % a.heads) : 0;
        const int r = tile * ROWS + qb * 16 + lc;
        const long long at = a.few_first ? (long long)blockIdx.x * ROWS + qb * 16 + lc
                                         : sp * a.part_rows + (a.part_most > 0 ? ((long long)s * key_heads + h) * a.part_most + r : o_row[qb]);
        const float inv = (rounded == 0.f ? 0.f : 1.f / rounded) * (C8 && a.v_scale ? a.v_scale[h] : 1.f);
#pragma unroll
        for (int f = 0; f < FB / NW; ++f) {
            const int fb = wave * (FB / NW) + f;
            f32x4 x = f32x4(0.f);
#pragma unroll
            for (int v = 0; v < NW; ++v) x += *reinterpret_cast<const f32x4*>(join + ((v * FB + fb) * QB + qb) * 1024 + lane * 16) * w[v];
            if (!real) continue;
            if (whole) {
                const u32x2 y = {E::pack2(x[0] * inv, x[1] * inv), E::pack2(x[2] * inv, x[3] * inv)};
                *reinterpret_cast<u32x2*>(a.o + t * a.o_token + head * a.o_head + (fb * 16 + lg * 4) * 2) = y;
            } else {
                *reinterpret_cast<f32x4*>(a.part_o + at * D + fb * 16 + lg * 4) = x;
            }
        }
        if (real && wave == 0 && lg == 0) {
            if (!whole) *reinterpret_cast<f32x4*>(a.part_ml + at * 4) = f32x4{m * c, l, rounded, 0.f};
            else if (a.lse) a.lse[o_row[qb]] = m * scale + __builtin_logf(l);
        }
    }
}

// ---- the splits of a row joined: WAVES waves (a workgroup) a row.  Groups of D / 4 lanes take 16 bytes each of a part's O, so that several parts are under
// way at a time, and the groups' sums meet in the LDS.
template <int DTYPE, bool C8, int D, int WAVES>
__global__ __launch_bounds__(WAVES * 64)
void attn_paged_join(PagedArgs a)
{
    typedef Elem<DTYPE> E;
    constexpr int LANES = D / 4, GROUPS = WAVES * 64 / LANES;
    __shared__ f32x4 s_x[GROUPS][LANES];
    __shared__ f32x2 s_l[GROUPS];
    const int lane = threadIdx.x & 63, group = threadIdx.x / LANES, e = threadIdx.x % LANES;
    // the r-th row of key head h of sequence s
    const int key_heads = a.heads / a.group, most = min(a.row_tiles * a.rows, a.max_q * a.group), r = blockIdx.x % most, h = blockIdx.x / most % key_heads;
    const long long sequence = blockIdx.x / most / key_heads;
    const int first = a.few_first ? a.few_first[sequence * a.row_tiles + r / a.rows] : 0;      // (on its way under what follows; of a tile without pieces anything)
    const SeqRange seq = seq_range(a.q_start, a.kv_len, (int)sequence, a.tokens, a.max_q, a.max_kv);
    if (r >= seq.n * a.group || seq.n * a.group > a.few_rows) return;
    const int keys = paged_tile_keys(r / a.rows, a.rows, seq.n, a.group, seq.first, seq.kv, a.causal);
    const int per = a.few_room > 0 ? few_piece_keys(few_pieces(*a.few_inverse, seq.kv), keys) : paged_piece_keys(keys, a.split);
    if (keys <= per) return;
    const int n = (keys + per - 1) / per, t = seq.q0 + r / a.group, head = h * a.group + r % a.group;
    const long long row = (long long)t * a.heads + head;
    const long long all = a.few_first ? (long long)key_heads * a.rows : a.part_rows;                 // slots from a piece to the next
    const long long slot = a.few_first ? ((long long)first * key_heads + h) * a.rows + r % a.rows
                         : a.part_most > 0 ? (sequence * key_heads + h) * a.part_most + r : row;
    const float* const part_o = a.part_o + slot * D;
    const float* const part_ml = a.part_ml + slot * 4;
    float m = -__builtin_inff();
    for (int i = lane; i < n; i += 64) m = __builtin_fmaxf(m, part_ml[i * all * 4]);
#pragma unroll
    for (int i = 1; i < 64; i *= 2) m = __builtin_fmaxf(m, __shfl_xor(m, i));
    // (a part without a key has a finite reference; a score of +infinity makes the row NaN here as in a whole one)
    f32x4 x = f32x4(0.f);
    f32x2 l = f32x2(0.f);                       // of the weights, and of the rounded ones
#pragma unroll 4
    for (int i = group; i < n; i += GROUPS) {
        const f32x4 ml = *reinterpret_cast<const f32x4*>(part_ml + i * all * 4);
        const float w = __builtin_amdgcn_exp2f(ml[0] - m);
        l += f32x2{ml[1], ml[2]} * w;
        x += *reinterpret_cast<const f32x4*>(part_o + i * all * D + e * 4) * w;
    }
    s_x[group][e] = x;
    if (e == 0) s_l[group] = l;
    __syncthreads();
    if (threadIdx.x >= LANES) return;
#pragma unroll
    for (int g = 1; g < GROUPS; ++g) {
        x += s_x[g][e];
        l += s_l[g];
    }
    const float inv = (l[1] == 0.f ? 0.f : 1.f / l[1]) * (C8 && a.v_scale ? a.v_scale[h] : 1.f);
    *reinterpret_cast<u32x2*>(a.o + t * a.o_token + head * a.o_head + e * 8) = u32x2{E::pack2(x[0] * inv, x[1] * inv), E::pack2(x[2] * inv, x[3] * inv)};
    if (a.lse && e == 0) a.lse[row] = (m + __builtin_amdgcn_logf(l[0])) * 0.6931471805599453f;
}

// ---- the pieces of a chunk joined: D / 4 lanes a row, so 1024 / D rows by a workgroup
template <int DTYPE, bool C8, int D>
__global__ __launch_bounds__(256)
void attn_paged_join_chunks(PagedArgs a)
{
    typedef Elem<DTYPE> E;
    constexpr int LANES = D / 4;
    const int key_heads = a.heads / a.group, h = blockIdx.x % key_heads, e = threadIdx.x % LANES;
    if ((int)blockIdx.x >= a.chunk_what[a.chunk_parts * 4]) return;
    const u32x4 what = *reinterpret_cast<const u32x4*>(a.chunk_what + blockIdx.x * 4);
    const int s = (int)what[0], n = (int)what[2];
    if (n < 2) return;
    const SeqRange seq = seq_range(a.q_start, a.kv_len, s, a.tokens, a.max_q, a.max_kv);
    const long long step = (long long)key_heads * PAGED_CHUNK_ROWS;      // from a piece to the next
    const int r = blockIdx.y * (256 / LANES) + threadIdx.x / LANES, row = (int)what[1] * PAGED_CHUNK_ROWS + r, tok = row / a.group, head = h * a.group + row % a.group;
    if (tok >= seq.n) return;
    const long long first = (long long)what[3] * PAGED_CHUNK_ROWS + r;
    const int lane = threadIdx.x & 15;          // 16 lanes have 16 pieces' references and sums
    f32x4 ml = *reinterpret_cast<const f32x4*>(a.chunk_ml + (first + min(lane, n - 1) * step) * 4);
    float m = ml[0];
    for (int k = 16 + lane; k < n; k += 16) m = __builtin_fmaxf(m, a.chunk_ml[(first + k * step) * 4]);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) m = __builtin_fmaxf(m, __shfl_xor(m, d));
    f32x2 l = f32x2(0.f);                       // of the weights, and of the rounded ones
    f32x4 x = f32x4(0.f);
    for (int k = 0; k < n; k += 16) {
        if (k > 0) ml = *reinterpret_cast<const f32x4*>(a.chunk_ml + (first + min(k + lane, n - 1) * step) * 4);
        const float w = __builtin_amdgcn_exp2f(ml[0] - m);
        l += k + lane < n ? f32x2{ml[1], ml[2]} * w : f32x2(0.f);
        const int some = min(16, n - k);
        auto add = [&](auto count, int j) __attribute__((always_inline)) {       // so many loads under way
#pragma unroll
            for (int i = j; i < j + decltype(count)::value; ++i) {
                const f32x4 part = *reinterpret_cast<const f32x4*>(a.chunk_o + (first + min(k + i, n - 1) * step) * D + e * 4) * __shfl(w, (threadIdx.x & 48) + i);
                x += i < some ? part : f32x4(0.f);
            }
        };
        int j = 0;
        for (; j + 2 < some; j += 8) add(std::integral_constant<int, 8>(), j);
        if (j < some) add(std::integral_constant<int, 2>(), j);
    }
#pragma unroll
    for (int d = 1; d < 16; d *= 2) l += f32x2{__shfl_xor(l[0], d), __shfl_xor(l[1], d)};
    const int t = seq.q0 + tok;
    const float inv = (l[1] == 0.f ? 0.f : 1.f / l[1]) * (C8 && a.v_scale ? a.v_scale[h] : 1.f);
    *reinterpret_cast<u32x2*>(a.o + t * a.o_token + head * a.o_head + e * 8) = u32x2{E::pack2(x[0] * inv, x[1] * inv), E::pack2(x[2] * inv, x[3] * inv)};
    if (a.lse && e == 0) a.lse[(long long)t * a.heads + head] = (m + __builtin_amdgcn_logf(l[0])) * 0.6931471805599453f;
}

template <int DTYPE, bool C8, int D, int QB>
int launch_few(const PagedArgs& a, hipStream_t stream)
{
    typedef FewLayout<D, C8 ? 1 : 2, QB> Layout;
    auto kern = attn_paged_few<DTYPE, C8, D, QB>;
    static PerDeviceOnce once;
    constexpr int STAGES = NW * Layout::SLOTS;
    if (once.prepare(reinterpret_cast<const void*>(kern), Layout::smem(STAGES)) < 0) return -1;
    PagedArgs arg = a;
    void* args[] = {&arg};
    // Where all keys fit fewer stages, the others are not asked for and more workgroups fit a compute unit.  (us so / with all stages, d 128:
    // 156 sequences of 7 keys, 16 heads 22 / 39; 256 of 100, 32 heads on 8 31 / 48.)
    const int blocks = a.max_kv < STAGES * 32 ? (a.max_kv + 31) / 32 : STAGES, smem = Layout::smem(blocks);
    const long long grid = (a.few_room > 0 ? a.few_room : (long long)a.sequences * a.row_tiles * a.splits) * (a.heads / a.group);
    return hipLaunchKernel(reinterpret_cast<const void*>(kern), dim3((unsigned)grid), dim3(NW * 64), args, smem, stream) == hipSuccess ? 0 : -1;
}

template <int DTYPE, bool C8, int D>
int launch_all(const PagedArgs& a, const PagedPlan& plan, hipStream_t stream)
{
    int rc = 0;
    if (plan.few_rows > 0) rc = plan.rows == 16 ? launch_few<DTYPE, C8, D, 1>(a, stream) : launch_few<DTYPE, C8, D, 2>(a, stream);
    if (rc == 0 && plan.chunk_tiles > 0) rc = attn_paged_chunk_launch(a, plan, D, DTYPE, C8 ? KV_E4M3 : DTYPE, stream);
    PagedArgs arg = a;
    void* args[] = {&arg};
    if (rc == 0 && a.chunk_parts > 0)
        rc = hipLaunchKernel(reinterpret_cast<const void*>(attn_paged_join_chunks<DTYPE, C8, D>), dim3((unsigned)(plan.chunk_tiles < a.chunk_parts ? plan.chunk_tiles : a.chunk_parts), PAGED_CHUNK_ROWS / (1024 / D)), dim3(256), args, 0, stream) == hipSuccess ? 0 : -1;
    if (rc != 0 || a.splits == 1) return rc;
    // (few rows: 4 waves a row, to have many parts under way; many: one)
    const int most = a.max_q * a.group < a.row_tiles * a.rows ? a.max_q * a.group : a.row_tiles * a.rows;
    const long long grid = (long long)a.sequences * (a.heads / a.group) * most;
    const void* const kern = grid <= 1024 ? reinterpret_cast<const void*>(attn_paged_join<DTYPE, C8, D, 4>) : reinterpret_cast<const void*>(attn_paged_join<DTYPE, C8, D, 1>);
    return hipLaunchKernel(kern, dim3((unsigned)grid), dim3(grid <= 1024 ? 256 : 64), args, 0, stream) == hipSuccess ? 0 : -1;
}

}  // namespace

PagedPlan paged_plan(int sequences, int tokens, int max_q, int max_kv, int heads, int key_heads, int d, int cache_bytes)
{
    const int group = heads / key_heads;
    const long long most = (long long)max_q * group;
    const int whole = (max_kv + 127) / 128 * 128;            // one split
    PagedPlan p{};
    p.splits = 1;
    p.split = whole;
    // Small tiles of 16 or 32 rows, or chunks of 256.  The former have many workgroups, fit for short calls, the latter feed the matrix cores better.  In keys that the places
    // of the chip walk through one after the other: chunks of sequences that they are cut for (or are not) cost as much as 400 (900) keys more.  us chunks / small tiles, d 128, 16-bit,
    // 16 heads, one prompt of 64 8.3 / 5.9, 256 15.7 / 7.2, 512 21.4 / 12.6, 1024 26.4 / 25.5, 2048 42.4 / 71.5; 32 heads on 8, 64 tokens of 1000 20.4 / 12.9, 256 of 4000 35.8 / 54,
    // one prompt of 1024 32.7 / 47.
    const long long key_bytes = 2ll * d * cache_bytes;
    auto workgroups = [&](int rows) { return (double)((most + rows - 1) / rows) * sequences * key_heads; };
    auto places = [&](int rows, int kv) {       // what the LDS and the registers hold on 256 compute units
        const int stages = kv < 256 ? (kv + 31) / 32 : 8;
        const long long ring = stages * 32 * key_bytes, join = rows * d * 16, fit = (160 << 10) / (rows * 64 + (ring > join ? ring : join)), regs = rows == 32 ? (d == 128 ? 1 : 2) : d == 128 ? 2 : cache_bytes == 2 ? 3 : 4;
        return 256 * (fit < regs ? fit : regs);
    };
    const double small = workgroups(32), chip = places(16, 256);
    const double keys = max_q < max_kv ? max_kv - 0.5 * max_q : 0.5 * max_kv;        // of a row on the mean, as most calls are
    const bool all_small = most <= 32 || (small <= 256 + chip && small * keys / chip <= (max_kv > 1024 ? 400 : 900) + workgroups(256) * keys / 256);
    // With chunks, sequences of up to 32 rows go by small tiles, in a kernel of their own, where a batch has many workgroups, else by a chunk each.  That kernel costs 10 ... 20 us beside the
    // chunks' and saves what many or long single tokens take longer as chunks.  us chunks for all / both (sequences x key heads): 16 heads on 4, 7 tokens of 4000 beside a prompt of 4096
    // 110 / 131 (32), 8 of 1000 ... 4000 beside 8 prompts of 64 29 / 45 (64), 28 of 300 ... 8000 beside 4 of 1024 148 / 83 (128); 32 heads on 8, 60 of 300 ... 4000 beside 4 of 512 125 / 128 (512),
    // 12 of 300 ... 2000 beside 12 of 256 54 / 63 (192), 7 of 65536 beside one of 2048 1115 / 392 (64): the product tells them apart only roughly, the last two are on the wrong side of it.
    p.few_rows = all_small ? 1 << 30 : (long long)sequences * key_heads > 64 ? 32 : 0;
    // 16 rows where they have a place each (with the pieces of long sequences) or, with more rows, no more rounds than those of 32: a step of 128 keys takes 1.0 us with 16 rows, 1.5 with 32.
    const double parts = max_kv > 1024 ? max_kv / 512. : 1., rounds = parts * workgroups(16) / places(16, max_kv), rounds32 = parts * small / places(32, max_kv);
    p.rows = most <= 16 || (all_small && (rounds <= 1. || (most > 32 && rounds <= rounds32))) ? 16 : 32;
    p.row_tiles = all_small ? (int)((most + p.rows - 1) / p.rows) : 1;
    if (p.few_rows) {
        // Pieces, of 512 keys at least: where the workgroups are fewer than the places, as many as these are, found on the device; where there are 512 workgroups or more
        // anyway, pieces only serve to even out lengths, and have 1.25 MiB of keys and values.  A piece costs 4 us besides its keys, the joining
        // 6.  (us at most keys of a piece 512 / 768 / 1536 / 2560 / 4096, d 128, 32 heads on 8: 64 sequences of 4000 218 / 211 / 197 / 191 / 183; of
        // 300 ... 16384 260 / 232 / 211 / 211 / 251.)
        const long long tiles = (long long)sequences * p.row_tiles, units = tiles * key_heads, even = (5 << 18) / key_bytes;
        if (units >= 512) {
            if (max_kv > even * 8 / 5) p.split = (int)((even + 127) / 128 * 128);
            p.splits = (int)((max_kv + p.split - 1) / p.split);
        } else if (max_kv > 1024) {
            // One piece a place, or two or three one after the other where that evens them out (sequences of 9000 of 4 tokens each over E4M3: 37, 32 heads on 4, d 128 115 / 95 us, 20, 128 heads on 16,
            // d 64 106 / 90) and reading the cache takes less time anyway.
            const double alone = max_kv / 128. * (p.rows == 16 ? 1. : 1.5), reading = (double)units * max_kv * key_bytes / 5.5e6;
            long long room = 0;
            double best = 1e30;
            for (int rounds = 1; rounds <= 3; ++rounds) {
                const long long all = places(p.rows, 256) * rounds, k = all / units;
                const double time = k == 0 ? 1e30 : rounds * (alone / k + 4.);
                if (time < 0.9 * best && best > reading) {
                    best = time;
                    room = all / key_heads;
                }
            }
            if (room > tiles) {                 // (else whole)
                const long long alike = (max_kv + room / tiles - 1) / (room / tiles);
                p.split = 512;
                p.split_max = (int)(alike > 512 ? alike : 512);
                if (sequences > 128) p.split = (p.split_max + 63) / 64 * 64;     // (many: finding out would take longer than it saves)
                else if (p.split_max > 512) p.few_room = (int)room;
                p.splits = (int)((max_kv + p.split - 1) / p.split);
                if (p.few_room > 0 && p.splits > p.few_room) p.splits = p.few_room;
            }
        }
    }
    if (!all_small) {
        const long long each = (most + PAGED_CHUNK_ROWS - 1) / PAGED_CHUNK_ROWS * sequences, all = (long long)tokens * group / PAGED_CHUNK_ROWS + sequences;
        p.chunk_tiles = (each < all ? each : all) * key_heads;
        if (max_kv > CHUNK_UNCUT) p.chunk_parts = CHUNK_PARTS;
    }
    return p;
}

int attn_paged_launch(const PagedArgs& a, const PagedPlan& plan, int d, int dtype, int cache_dtype, void* stream)
{
    const hipStream_t st = (hipStream_t)stream;
    if (cache_dtype == KV_E4M3) {
        if (dtype == 0) return d == 128 ? launch_all<0, true, 128>(a, plan, st) : launch_all<0, true, 64>(a, plan, st);
        return d == 128 ? launch_all<1, true, 128>(a, plan, st) : launch_all<1, true, 64>(a, plan, st);
    }
    if (dtype == 0) return d == 128 ? launch_all<0, false, 128>(a, plan, st) : launch_all<0, false, 64>(a, plan, st);
    return d == 128 ? launch_all<1, false, 128>(a, plan, st) : launch_all<1, false, 64>(a, plan, st);
}
