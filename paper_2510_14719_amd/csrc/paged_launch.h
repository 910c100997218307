// Internal seam between the host side of include/kv_cache.h (kv_api.cpp) and its kernels.
#pragma once

#include "kv_cache.h"

#if defined(__HIPCC__)
#define PAGED_HD __host__ __device__
#else
#define PAGED_HD
#endif

// What the attention kernels of one call share.
struct PagedArgs {
    const char *k, *v;
    const float *k_scale, *v_scale;
    long long page_bytes, head_bytes, token_bytes;          // strides of the cache
    const int *q_start, *kv_len, *table;
    const char* q;
    char* o;
    float* lse;
    long long q_token, q_head, o_token, o_head;              // strides, bytes
    // Partial results of the small tiles, [slot][d] and [slot][4]: reference, sum of the weights, of the rounded ones.  A slot is a row of a piece.
    // Where pieces are numbered from the plan on (few_first), piece i of key head h has the slots (i * key heads + h) * rows ...; else piece p of a row has the slot
    // p * part_rows + its row, counted as token * heads + head, or, where those are fewer (part_most > 0), as the r-th of part_most of its sequence and key head.
    float *part_o, *part_ml;
    long long part_rows;
    int part_most;
    int* few_first;                                          // [sequence][row tile]: number of its first piece
    int sequences, tokens, table_stride, max_q, max_kv, pages, page_shift;
    int heads, group;                                        // query heads, and how many share a key head
    int causal;
    int few_rows;                                            // sequences with more rows (new tokens x group) than this go by chunks of PAGED_CHUNK_ROWS
    int rows, row_tiles, split, splits;                      // the others: rows per workgroup, row tiles of the longest one, most keys of a piece (a multiple of 64), pieces of
                                                             // the longest
    int few_room;                                            // > 0: how long their pieces are is found on the device (few_cut), so that there are at most so many (of every key head)
    int few_fixed;                                           // the shortest length mostly fits
    float few_finest, few_step, few_coarsest;                // 1 / keys: of the shortest, log2 of a step, of the longest
    float* few_inverse;                                      // what was found, for the join
    int chunk_parts;                                         // room for partial results of chunks, in workgroups (0: chunks are not cut along the keys)
    float *chunk_o, *chunk_ml;                               // [workgroup][PAGED_CHUNK_ROWS][d], [..][4]
    int* chunk_what;                                         // [chunk of a key head][4]: sequence, chunk in it, pieces, workgroup of the first; behind the last [..][0] their number
    float scale;
};

constexpr int PAGED_CHUNK_ROWS = 256;                        // query rows (tokens x heads of a group) of a workgroup of attn_paged_chunk

// How a call is laid out (chosen by its sizes alone, so that the workspace is known beforehand).
struct PagedPlan {
    int few_rows, rows, row_tiles, split, splits, few_room, split_max, chunk_parts;      // as in PagedArgs (few_rows 0: all sequences go by chunks)
    long long chunk_tiles;                                   // chunks of all sequences, at most; 0: none does
};
PagedPlan paged_plan(int sequences, int tokens, int max_q, int max_kv, int heads, int key_heads, int d, int cache_bytes);

// Row tiles as they are cut from a sequence: tile t has the rows t * rows ... of the n * group rows (token-major) of its n new tokens, the first of which has position `first`.
// How many of its kv keys the rows of a tile may see.
PAGED_HD inline int paged_tile_keys(int tile, int rows, int n, int group, int first, int kv, int causal)
{
    if (!causal) return kv;
    const int last = (tile + 1) * rows - 1, token = last / group;
    const int end = first + (token < n ? token : n - 1) + 1;
    return end < 0 ? 0 : end;
}

// Enqueue for validated arguments: 0, or -1 if HIP refused a launch.
int attn_paged_chunk_launch(const PagedArgs& a, const PagedPlan& plan, int d, int dtype, int cache_dtype, void* stream);
int attn_paged_launch(const PagedArgs& a, const PagedPlan& plan, int d, int dtype, int cache_dtype, void* stream);

// Keys of a piece where a row of so many keys is cut into as many pieces as it has splits begun, all alike (the last may be shorter, or there are fewer).
PAGED_HD inline int paged_piece_keys(int keys, int split)
{
    if (keys <= split) return split;
    const int n = (keys + split - 1) / split;
    return ((keys + n - 1) / n + 63) / 64 * 64;
}

struct RopeArgs {
    const char* x;
    char* y;
    const int* pos;
    const double* freq;
    long long x_batch, x_head, x_token, y_batch, y_head, y_token, pos_stride;    // bytes (pos: entries)
    int batches, heads, tokens, d, rot, layout;
    float cos_factor, sin_factor;                            // amplitude, and amplitude with the sign of the direction
};
int rope_launch(const RopeArgs& a, int dtype, void* stream);

struct AppendArgs {
    char *k_cache, *v_cache;
    const float *k_scale, *v_scale;
    long long page_bytes, head_bytes, token_bytes;
    const int *q_start, *kv_len, *table;
    const char *k, *v, *q;
    char* q_out;
    const double* freq;
    long long k_token, k_head, v_token, v_head, q_token, q_head, o_token, o_head;
    int sequences, tokens, table_stride, max_q, max_kv, pages, page_shift;
    int heads, key_heads, d, rot, layout;                    // heads 0: no Q
    float amplitude;
};
int kv_append_launch(const AppendArgs& a, int dtype, int cache_dtype, void* stream);

// Contents of pages: rows of row_bytes, [layers][page][heads][tokens] by strides in bytes.
struct PageCopy {
    char *k, *v;
    long long layer, page, head, token;
    int layers, pages, heads, page_size, row_bytes;
    bool solid;                                              // the rows of a page of a layer lie without gaps, in whatever order
};
int kv_reserve_launch(const kv_book& b, const int* list, const int* new_len, int n, int* missing, void* stream);
int kv_free_launch(const kv_book& b, const int* list, int n, void* stream);
int kv_fork_launch(const PageCopy& c, const kv_book& b, const int* src, const int* dst, int n, int* missing, void* stream);
int kv_compact_launch(const PageCopy& c, const kv_book& b, int* workspace, void* stream);
int kv_copy_pages_launch(const PageCopy& c, const int* src, const int* dst, int n, void* stream);
