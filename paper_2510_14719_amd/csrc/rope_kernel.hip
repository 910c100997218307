// Rotary positions and the writing of new tokens to a paged cache (include/kv_cache.h), for gfx950 (MI355X).
//
// Both are bound by memory: every element is read once and written once.  The angles of a token serve all of its heads, so a workgroup takes a
// few tokens with all their heads, computes the sines and cosines once into the LDS and streams the heads past them.  An
// angle is position x frequency; at position 10^6 a product in 32 bits would be off by 0.06, so it is formed in 64 bits, in turns, and only the
// part of the last turn goes on in 32.  A thread's unit of work is 16 elements of a head, two times 16 bytes: 8 pairs, or 16 elements
// that are not turned.

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

// One unit: u < rot / 16 has the pairs 8 u ... 8 u + 7, the others 16 elements to copy.  `first`, `second`: where its two chunks of 8 elements stand.
__device__ __forceinline__ void unit_place(int u, int rot, int layout, int& first, int& second)
{
    const bool split = layout == KV_HALF && u < rot / 16;
    first = split ? u * 8 : u * 16;
    second = split ? u * 8 + rot / 2 : u * 16 + 8;
}
__device__ __forceinline__ void turn_unit(float (&a)[8], float (&b)[8], const f32x2* cs, int layout)
{
    if (layout == KV_HALF) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x2 t = cs[i];
            const float x = a[i], y = b[i];
            a[i] = x * t[0] - y * t[1];
            b[i] = y * t[0] + x * t[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const f32x2 t = cs[i];
            float& x = i < 4 ? a[2 * i] : b[2 * i - 8];
            float& y = i < 4 ? a[2 * i + 1] : b[2 * i - 7];
            const float x0 = x, y0 = y;
            x = x0 * t[0] - y0 * t[1];
            y = y0 * t[0] + x0 * t[1];
        }
    }
}

template <int DTYPE>
__global__ __launch_bounds__(THREADS)
void rope_kernel(RopeArgs a, int block_tokens, int head_step)
{
    extern __shared__ __attribute__((aligned(16))) char smem[];
    f32x2* const cs = reinterpret_cast<f32x2*>(smem);        // [token][rot / 2]
    const int blocks = (a.tokens + block_tokens - 1) / block_tokens, b = blockIdx.x / blocks, n0 = blockIdx.x % blocks * block_tokens;
    const int h0 = blockIdx.y * head_step, heads = min(head_step, a.heads - h0), count = min(block_tokens, a.tokens - n0);
    const int half = a.rot / 2, units = a.d / 16;
    for (int i = threadIdx.x; i < count * half; i += THREADS) {
        const int n = n0 + i / half;
        cs[i] = turn(a.pos ? a.pos[b * a.pos_stride + n] : n, a.freq[i % half], a.cos_factor, a.sin_factor);
    }
    __syncthreads();
    const char* const x = a.x + b * a.x_batch;
    char* const y = a.y + b * a.y_batch;
    const bool heads_inside = a.x_head < a.x_token;          // whichever of heads and tokens is nearer in memory goes first
    for (int i = threadIdx.x; i < count * heads * units; i += THREADS) {
        const int u = i % units, r = i / units;
        const int h = h0 + (heads_inside ? r % heads : r / count), n = heads_inside ? r / heads : r % count;
        int first, second;
        unit_place(u, a.rot, a.layout, first, second);
        const char* const from = x + h * a.x_head + (n0 + n) * a.x_token;
        char* const to = y + h * a.y_head + (n0 + n) * a.y_token;
        u32x4 w0 = *reinterpret_cast<const u32x4*>(from + first * 2), w1 = *reinterpret_cast<const u32x4*>(from + second * 2);
        if (u < a.rot / 16) {
            float p[8], q[8];
            unpack8<DTYPE>(w0, p);
            unpack8<DTYPE>(w1, q);
            turn_unit(p, q, cs + n * half + u * 8, a.layout);
            w0 = pack8<DTYPE>(p);
            w1 = pack8<DTYPE>(q);
        }
        *reinterpret_cast<u32x4*>(to + first * 2) = w0;
        *reinterpret_cast<u32x4*>(to + second * 2) = w1;
    }
}

// Eight values divided by the scale as E4M3: to nearest even, beyond the largest finite value to that one, NaN stays.
__device__ __forceinline__ u32x2 to_e4m3(const float (&x)[8], float scale)
{
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = x[i] / scale;
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
__global__ __launch_bounds__(THREADS)
void kv_append_kernel(AppendArgs a, int block_tokens)
{
    constexpr int MAX_TOKENS = 16;
    __shared__ int s_pos[MAX_TOKENS];
    __shared__ long long s_place[MAX_TOKENS];                // byte offset of the token in the cache, -1: not stored
    __shared__ int s_real[MAX_TOKENS];
    extern __shared__ __attribute__((aligned(16))) char smem[];
    f32x2* const cs = reinterpret_cast<f32x2*>(smem);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t0 = blockIdx.x * block_tokens, count = min(block_tokens, a.tokens - t0);
    for (int i = wave; i < count; i += THREADS / 64) {
        const int t = t0 + i, s = seq_of_token(a.q_start, a.sequences, t, lane);
        bool real = false;
        int pos = 0;
        long long place = -1;
        if (s >= 0) {
            const SeqRange seq = seq_range(a.q_start, a.kv_len, s, a.tokens, a.max_q, a.max_kv);
            real = t >= seq.q0 && t - seq.q0 < seq.n;
            pos = seq.kv - seq.n + (t - seq.q0);
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
    const int half = a.rot / 2, units = a.d / 16;
    for (int i = threadIdx.x; i < count * half; i += THREADS) cs[i] = turn(s_pos[i / half], a.freq[i % half], a.amplitude, a.amplitude);
    __syncthreads();
    const int rows = a.heads + 2 * a.key_heads;
    for (int i = threadIdx.x + blockIdx.y * THREADS; i < count * rows * units; i += THREADS * gridDim.y) {
        const int u = i % units, row = i / units % rows, n = i / units / rows, t = t0 + n;
        const bool is_q = row < a.heads, is_k = !is_q && row < a.heads + a.key_heads;
        const long long place = s_place[n];
        if (!s_real[n] || (!is_q && place < 0)) continue;
        const int h = is_q ? row : is_k ? row - a.heads : row - a.heads - a.key_heads;
        const char* const from = is_q ? a.q + t * a.q_token + h * a.q_head : is_k ? a.k + t * a.k_token + h * a.k_head : a.v + t * a.v_token + h * a.v_head;
        int first, second;
        unit_place(u, a.rot, a.layout, first, second);
        u32x4 w0 = *reinterpret_cast<const u32x4*>(from + first * 2), w1 = *reinterpret_cast<const u32x4*>(from + second * 2);
        const bool turned = u < a.rot / 16 && (is_q || is_k);
        if (is_q || !C8) {
            if (turned) {
                float p[8], q[8];
                unpack8<DTYPE>(w0, p);
                unpack8<DTYPE>(w1, q);
                turn_unit(p, q, cs + n * half + u * 8, a.layout);
                w0 = pack8<DTYPE>(p);
                w1 = pack8<DTYPE>(q);
            }
            char* const to = is_q ? a.q_out + t * a.o_token + h * a.o_head : (is_k ? a.k_cache : a.v_cache) + place + h * a.head_bytes;
            *reinterpret_cast<u32x4*>(to + first * 2) = w0;
            *reinterpret_cast<u32x4*>(to + second * 2) = w1;
        } else {
            float p[8], q[8];
            unpack8<DTYPE>(w0, p);
            unpack8<DTYPE>(w1, q);
            if (turned) turn_unit(p, q, cs + n * half + u * 8, a.layout);
            const float scale = a.k_scale ? (is_k ? a.k_scale : a.v_scale)[h] : 1.f;
            char* const to = (is_k ? a.k_cache : a.v_cache) + place + h * a.head_bytes;
            *reinterpret_cast<u32x2*>(to + first) = to_e4m3(p, scale);
            *reinterpret_cast<u32x2*>(to + second) = to_e4m3(q, scale);
        }
    }
}

}  // namespace

int rope_launch(const RopeArgs& a, int dtype, void* stream)
{
    // Tokens per workgroup: up to 16, fewer where the chip would not be full; heads are shared out where there are few tokens.
    const long long all = (long long)a.batches * a.tokens;
    int bt = 16;
    while (bt > 1 && all / bt < 1024) bt /= 2;
    const long long blocks = (a.tokens + bt - 1) / bt * (long long)a.batches;
    int head_step = a.heads;
    while (head_step > 4 && blocks * ((a.heads + head_step - 1) / head_step) < 512) head_step = (head_step + 1) / 2;
    RopeArgs arg = a;
    void* args[] = {&arg, &bt, &head_step};
    const void* kern = dtype == 0 ? reinterpret_cast<const void*>(rope_kernel<0>) : reinterpret_cast<const void*>(rope_kernel<1>);
    const dim3 grid((unsigned)blocks, (unsigned)((a.heads + head_step - 1) / head_step));
    return hipLaunchKernel(kern, grid, dim3(THREADS), args, bt * a.rot / 2 * sizeof(f32x2), (hipStream_t)stream) == hipSuccess ? 0 : -1;
}

int kv_append_launch(const AppendArgs& a, int dtype, int cache_dtype, void* stream)
{
    int bt = 16;
    while (bt > 1 && a.tokens / bt < 1024) bt /= 2;
    const int blocks = (a.tokens + bt - 1) / bt;
    const int most = (bt * (a.heads + 2 * a.key_heads) * (a.d / 16) + THREADS - 1) / THREADS;
    int parts = 1;
    while (parts < most && (long long)blocks * parts < 512) parts *= 2;
    AppendArgs arg = a;
    void* args[] = {&arg, &bt};
    const bool c8 = cache_dtype == KV_E4M3;
    const void* kern = dtype == 0 ? (c8 ? reinterpret_cast<const void*>(kv_append_kernel<0, true>) : reinterpret_cast<const void*>(kv_append_kernel<0, false>))
                                  : (c8 ? reinterpret_cast<const void*>(kv_append_kernel<1, true>) : reinterpret_cast<const void*>(kv_append_kernel<1, false>));
    return hipLaunchKernel(kern, dim3((unsigned)blocks, (unsigned)parts), dim3(THREADS), args, bt * a.rot / 2 * sizeof(f32x2), (hipStream_t)stream) == hipSuccess ? 0 : -1;
}
