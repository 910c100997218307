// Rotary positions and the writing of new tokens to a paged cache (include/kv_cache.h), for gfx950 (MI355X).
//
// Both are bound by memory: every element is read once and written once.  The angles of a token serve all of its heads, so a workgroup takes a
// few tokens with all their heads, computes the sines and cosines once into the LDS and streams the heads past them.  An
// angle is position x frequency; at position 10^6 a product in 32 bits would be off by 0.06, so it is formed in 64 bits, in turns, and only the
// part of the last turn goes on in 32.  A thread's unit of work is 16 elements of a head, two times 16 bytes.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paged_launch.h"
#include "paged_prims.h"

namespace {

constexpr int THREADS = 256;

template <int DTYPE> __device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = to_float<DTYPE>((uint16_t)w[i]);
        x[2 * i + 1] = to_float<DTYPE>((uint16_t)(w[i] >> 16));
    }
}
template <int DTYPE> __device__ __forceinline__ u32x4 pack8(const float (&x)[8])
{
    return u32x4{Elem<DTYPE>::pack2(x[0], x[1]), Elem<DTYPE>::pack2(x[2], x[3]), Elem<DTYPE>::pack2(x[4], x[5]), Elem<DTYPE>::pack2(x[6], x[7])};
}

// Cosine and sine of position * freq, times the factors.
__device__ __forceinline__ f32x2 turn(int pos, double freq, float cos_factor, float sin_factor)
{
    const double turns = (double)pos * (freq * 0.15915494309189533577);
    float s, c;
    sincospif((float)(2.0 * (turns - __builtin_rint(turns))), &s, &c);
    return f32x2{c * cos_factor, s * sin_factor};
}

// Unit u has two chunks of 8 elements, half of their part of the head apart (so that neighbouring lanes have neighbouring chunks): u < rot / 16 those of the part
// that is turned, 8 pairs, the others those of the part that is copied.
__device__ __forceinline__ void unit_place(int u, int d, int rot, int& first, int& second)
{
    const bool turned = u < rot / 16;
    first = turned ? u * 8 : rot + (u - rot / 16) * 8;
    second = first + (turned ? rot : d - rot) / 2;
}
// Turns the chunks a and b of unit u; cs: cosine and sine of every pair of the token.
__device__ __forceinline__ void turn_unit(float (&a)[8], float (&b)[8], const f32x2* cs, int u, int rot, int layout)
{
    if (layout == KV_HALF) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x2 t = cs[u * 8 + i];
            const float x = a[i], y = b[i];
            a[i] = x * t[0] - y * t[1];
            b[i] = y * t[0] + x * t[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 t = cs[u * 4 + i], s = cs[rot / 4 + u * 4 + i];
            const float x = a[2 * i], y = a[2 * i + 1], z = b[2 * i], w = b[2 * i + 1];
            a[2 * i] = x * t[0] - y * t[1];
            a[2 * i + 1] = y * t[0] + x * t[1];
            b[2 * i] = z * s[0] - w * s[1];
            b[2 * i + 1] = w * s[0] + z * s[1];
        }
    }
}

// The units of a workgroup: a thread has the same u in all of its rows (threads beyond a multiple of the units of a head have nothing to do).  Of heads
// and tokens the one nearer in memory is numbered innermost, so that a workgroup's accesses lie together (packed tokens of 48 heads into an E4M3 cache, 7800
// tokens, four rows at a time: 76 us with the tokens innermost, 70 so).  The first row's loads are under way while the angles are computed; beyond that it takes many waves, not many
// loads a wave: with 1 / 2 / 4 rows at a time (8, 6, 4 waves a SIMD) these tokens take 60 / 64 / 69 us, 8 x 32 heads, N 8192, d 128 (1.07 GB) 200 / 203 / 219.
struct Walk {
    int u, row, step;                           // u < 0: nothing to do
};
__device__ __forceinline__ Walk walk_of(int units)
{
    const int rows = THREADS / units, tid = threadIdx.x;
    return {tid < rows * units ? tid % units : -1, tid / units, rows};
}

template <int DTYPE>
__global__ __launch_bounds__(THREADS, 8)
void rope_kernel(RopeArgs a, int log_tokens, int head_step)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    f32x2* const cs = reinterpret_cast<f32x2*>(smem);        // [token][rot / 2]
    const int block_tokens = 1 << log_tokens, blocks = (a.tokens + block_tokens - 1) >> log_tokens, b = blockIdx.x / blocks, n0 = (blockIdx.x - b * blocks) << log_tokens;
    const int h0 = blockIdx.y * head_step, heads = min(head_step, a.heads - h0), count = min(block_tokens, a.tokens - n0);
    const int half = a.rot / 2;
    const Walk w = walk_of(a.d / 16);
    int first, second;
    unit_place(max(w.u, 0), a.d, a.rot, first, second);
    const char* const x = a.x + b * a.x_batch + h0 * a.x_head + n0 * a.x_token;
    char* const y = a.y + b * a.y_batch + h0 * a.y_head + n0 * a.y_token;
    const int rows = w.u < 0 ? 0 : heads * count;
    const bool heads_inside = a.x_head < a.x_token;
    u32x4 p, q;
    int n, h;                                   // token and head of the present row
    auto load = [&](int r) __attribute__((always_inline)) {
        if (r >= rows) return;
        const int outer = r / (heads_inside ? heads : count), inner = r - outer * (heads_inside ? heads : count);
        n = heads_inside ? outer : inner;
        h = heads_inside ? inner : outer;
        const char* const from = x + h * a.x_head + n * a.x_token;
        p = *reinterpret_cast<const u32x4*>(from + first * 2);
        q = *reinterpret_cast<const u32x4*>(from + second * 2);
    };
    load(w.row);
    for (int i = threadIdx.x; i < count * half; i += THREADS) {
        const int k = i / half, m = i - k * half;
        cs[i] = turn(a.pos ? a.pos[b * a.pos_stride + n0 + k] : n0 + k, a.freq[m], a.cos_factor, a.sin_factor);
    }
    __syncthreads();
    const bool turned = w.u < a.rot / 16;
    for (int r = w.row; r < rows; r += w.step) {
        if (r != w.row) load(r);
        if (turned) {
            float s[8], t[8];
            unpack8<DTYPE>(p, s);
            unpack8<DTYPE>(q, t);
            turn_unit(s, t, cs + n * half, w.u, a.rot, a.layout);
            p = pack8<DTYPE>(s);
            q = pack8<DTYPE>(t);
        }
        char* const to = y + h * a.y_head + n * a.y_token;
        *reinterpret_cast<u32x4*>(to + first * 2) = p;       // (written through the L2: 0 to 4 % less, with rot 96 a fifth more; past the caches: the next reader pays)
        *reinterpret_cast<u32x4*>(to + second * 2) = q;
    }
}

// Eight values divided by the scale as E4M3: to nearest even, beyond the largest finite value to that one, NaN stays.  The quotient is x times the
// reciprocal and one correction by the remainder, which rounds it as a division does (a division costs four times as much); far beyond 448, where the
// correction might overflow, it does not matter.  (A scale below the normal numbers may have no reciprocal: the values of such a head are brought up with it first.)
__device__ __forceinline__ u32x2 to_e4m3(float (&x)[8], float scale, float reciprocal)
{
    float v[8];
    if (__builtin_expect(scale < 0x1p-126f, 0)) {
        scale *= 0x1p64f;
        reciprocal = 1.f / scale;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= 0x1p64f;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = x[i] * reciprocal, exact = __builtin_fmaf(__builtin_fmaf(-q, scale, x[i]), reciprocal, q);
        v[i] = __builtin_fabsf(q) < 1024.f ? exact : q;
        v[i] = v[i] > 448.f ? 448.f : v[i] < -448.f ? -448.f : v[i];
    }
    u32x2 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        r[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], w, true);
    }
    return r;
}

template <int DTYPE, bool C8>
__global__ __launch_bounds__(THREADS, 6)
void kv_append_kernel(AppendArgs a, int log_tokens)
{
    constexpr int MAX_TOKENS = 16;
    __shared__ int s_pos[MAX_TOKENS];
    __shared__ long long s_place[MAX_TOKENS];                // byte offset of the token in the cache, -1: not stored
    __shared__ int s_real[MAX_TOKENS];
    extern __shared__ __attribute__((aligned(16))) char smem[];
    f32x2* const cs = reinterpret_cast<f32x2*>(smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block_tokens = 1 << log_tokens, t0 = blockIdx.x << log_tokens, count = min(block_tokens, a.tokens - t0);
    for (int i = wave; i < count; i += THREADS / 64) {
        const int t = t0 + i, s = seq_of_token(a.q_start, a.sequences, t, lane);
        bool real = false;
        int pos = 0;
        long long place = -1;
        if (s >= 0) {
            const SeqRange seq = seq_range(a.q_start, a.kv_len, s, a.tokens, a.max_q, a.max_kv);
            real = t >= seq.q0 && t - seq.q0 < seq.n;
            pos = seq.first + (t - seq.q0);
            if (real && pos >= 0) {
                const int page = a.table[(long long)s * a.table_stride + (pos >> a.page_shift)];
                if ((unsigned)page < (unsigned)a.pages) place = page * a.page_bytes + (pos & ((1 << a.page_shift) - 1)) * a.token_bytes;
            }
        }
        if (lane == 0) {
            s_pos[i] = pos;
            s_place[i] = place;
            s_real[i] = real;
        }
    }
    __syncthreads();
    const int half = a.rot / 2, total = a.heads + 2 * a.key_heads;       // rows of a token: heads of Q, K, V
    const Walk w = walk_of(a.d / 16);
    int first, second;
    unit_place(max(w.u, 0), a.d, a.rot, first, second);
    const int rows = w.u < 0 ? 0 : total * count;
    u32x4 p, q;
    int n, h;                                   // token and row of the token that are on
    bool there;                                 // whether there is anything to do for them
    auto load = [&](int r) __attribute__((always_inline)) {
        if (r >= rows) return;
        n = r / total;
        h = r - n * total;
        there = s_real[n] && (h < a.heads || s_place[n] >= 0);
        if (!there) return;
        const int t = t0 + n, kh = h - a.heads, vh = kh - a.key_heads;
        const char* const from = kh < 0 ? a.q + t * a.q_token + h * a.q_head : vh < 0 ? a.k + t * a.k_token + kh * a.k_head : a.v + t * a.v_token + vh * a.v_head;
        p = *reinterpret_cast<const u32x4*>(from + first * 2);
        q = *reinterpret_cast<const u32x4*>(from + second * 2);
    };
    const int start = w.row + blockIdx.y * w.step, stride = gridDim.y * w.step;
    load(start);
    for (int i = threadIdx.x; i < count * half; i += THREADS) {
        const int k = i / half, m = i - k * half;
        cs[i] = turn(s_pos[k], a.freq[m], a.amplitude, a.amplitude);
    }
    __syncthreads();
    for (int r = start; r < rows; r += stride) {
        if (r != start) load(r);
        if (!there) continue;
        const int kh = h - a.heads, vh = kh - a.key_heads;
        const bool turned = vh < 0 && w.u < a.rot / 16, to_cache8 = C8 && kh >= 0;
        char* const place = kh < 0 ? nullptr : vh < 0 ? a.k_cache + s_place[n] + kh * a.head_bytes : a.v_cache + s_place[n] + vh * a.head_bytes;
        if (turned || to_cache8) {
            float s[8], t[8];
            unpack8<DTYPE>(p, s);
            unpack8<DTYPE>(q, t);
            if (turned) turn_unit(s, t, cs + n * half, w.u, a.rot, a.layout);
            if (to_cache8) {
                const float scale = a.k_scale ? vh < 0 ? a.k_scale[kh] : a.v_scale[vh] : 1.f, reciprocal = 1.f / scale;
                *reinterpret_cast<u32x2*>(place + first) = to_e4m3(s, scale, reciprocal);
                *reinterpret_cast<u32x2*>(place + second) = to_e4m3(t, scale, reciprocal);
                continue;
            }
            p = pack8<DTYPE>(s);
            q = pack8<DTYPE>(t);
        }
        char* const to = kh < 0 ? a.q_out + (t0 + n) * a.o_token + h * a.o_head : place;
        *reinterpret_cast<u32x4*>(to + first * 2) = p;
        *reinterpret_cast<u32x4*>(to + second * 2) = q;
    }
}

}  // namespace

int rope_launch(const RopeArgs& a, int dtype, void* stream)
{
    // Tokens per workgroup: up to 16, fewer where the chip would not be full; heads are shared out where there are few tokens.
    const long long all = (long long)a.batches * a.tokens;
    int log_tokens = 4;
    while (log_tokens > 0 && all >> log_tokens < 1024) --log_tokens;
    const long long blocks = ((a.tokens + (1ll << log_tokens) - 1) >> log_tokens) * a.batches;
    int head_step = a.heads;
    while (head_step > 4 && blocks * ((a.heads + head_step - 1) / head_step) < 512) head_step = (head_step + 1) / 2;
    RopeArgs arg = a;
    void* args[] = {&arg, &log_tokens, &head_step};
    const void* kern = dtype == 0 ? reinterpret_cast<const void*>(rope_kernel<0>) : reinterpret_cast<const void*>(rope_kernel<1>);
    const dim3 grid((unsigned)blocks, (unsigned)((a.heads + head_step - 1) / head_step));
    return hipLaunchKernel(kern, grid, dim3(THREADS), args, (a.rot / 2 * sizeof(f32x2)) << log_tokens, (hipStream_t)stream) == hipSuccess ? 0 : -1;
}

int kv_append_launch(const AppendArgs& a, int dtype, int cache_dtype, void* stream)
{
    // Tokens per workgroup: as above, but four times as many workgroups (7800 tokens of 48 heads into an E4M3 cache: 68 / 58 / 55 / 52 / 57 us with 512 / 1024 / 2048 /
    // 4096 / 8192 workgroups; rope, whose rows are the longer streams, 4 x 16 heads, N 4096 28.9 / 28.8 / 25.8 / 27.1 / 27.5, 16 heads, N 16384
    // 28.6 / 28.5 / 31.7 / 32.5 / 32.4).
    int log_tokens = 4;
    while (log_tokens > 0 && a.tokens >> log_tokens < 4096) --log_tokens;
    const int blocks = (a.tokens + (1 << log_tokens) - 1) >> log_tokens;
    // rows that a workgroup takes at a time, and how many workgroups share a block of tokens where the chip would not be full
    const int at_once = THREADS / (a.d / 16), most = (((a.heads + 2 * a.key_heads) << log_tokens) + at_once - 1) / at_once;
    int parts = 1;
    while (parts < most && (long long)blocks * parts < 512) parts *= 2;
    AppendArgs arg = a;
    void* args[] = {&arg, &log_tokens};
    const bool c8 = cache_dtype == KV_E4M3;
    const void* kern = dtype == 0 ? (c8 ? reinterpret_cast<const void*>(kv_append_kernel<0, true>) : reinterpret_cast<const void*>(kv_append_kernel<0, false>))
                                  : (c8 ? reinterpret_cast<const void*>(kv_append_kernel<1, true>) : reinterpret_cast<const void*>(kv_append_kernel<1, false>));
    return hipLaunchKernel(kern, dim3((unsigned)blocks, (unsigned)parts), dim3(THREADS), args, (a.rot / 2 * sizeof(f32x2)) << log_tokens, (hipStream_t)stream) == hipSuccess ? 0 : -1;
}
