// Paged K/V: the structures and launchers behind odb_page_tables, odb_rope_table, odb_qk_norm_rope and odb_paged_attention.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/odb.h"
#include "common.h"

namespace odb {

constexpr int kMaxRequests = 4096;

struct PageTables {
    const int32_t *held, *wanted, *first, *count;      // first / count may be null: the rows behind the held positions
    int n, page_shift, columns, n_pages, rows_cap;
    int32_t *tables, *free_pages;
    const int32_t *n_free;
    int32_t *len, *cu_rows, *slots, *positions, *state;
    int row_groups, page_groups;        // workgroups for the rows, and for each of pages given back and pages taken
};
void launch_page_tables(PageTables a, hipStream_t s);

// Angle per position of every pair, in turns: hi + lo (two doubles, so that far positions keep their fraction)
constexpr int kMaxRotPairs = 128;
struct RopeTable {
    float *table;
    int n_pos, pairs;
    double magnitude;
    double hi[kMaxRotPairs], lo[kMaxRotPairs];
};
void launch_rope_angles(const RopeTable &a, hipStream_t s);

struct QkNormRope {
    const void *q, *k, *v;
    int in_dtype;
    long long q_row, k_row, v_row;      // elements from row to row; the heads of a row follow each other
    int rows, heads;
    const float *q_gain, *k_gain;       // null: no norm
    float eps;
    const float *table;
    int n_pos, rot, interleaved;
    const int32_t *positions, *slots;
    void *q_out;
    long long q_out_row;
    odb_pages pages;
    const int32_t *row_end;             // null: all rows count
    unsigned *status;                   // a model's status word: binary16 values saturate and are reported there; null: they become infinite
};
// head_dim / 16 lanes a head; rows times this, 64 threads each, is below 2^32
inline int qk_waves_per_row(int heads, const odb_pages &p) {
    const int per_wave = 64 / (p.head_dim / 16);
    return (heads + 2 * p.n_kv_heads + per_wave - 1) / per_wave;
}
void launch_qk_norm_rope(const QkNormRope &a, hipStream_t s);

struct PagedAttn {
    const void *q;
    void *out;
    long long q_row, out_row;
    int out_mt;                         // > 0: out is in operand tiles [heads * head_dim / 32][out_mt][512] (see common.h)
    // cu_rows null: every request has rows_per_request rows; first null: the rows are the last positions
    const int32_t *cu_rows, *first, *kv_len, *tables;
    int rows_per_request;
    int columns, n, rows, heads, group;
    float sc;                           // scale * log2(e)
    int causal, window, sinks;
    odb_pages pages;
    int page_shift;
    // split > 0: that many workgroups per K/V head share the blocks of all (request, row tile) pairs; the sums of a pair that lies in
    // more than one go to `partial`, [2 split][heads of K/V][tile rows][head_dim], and (reference, sum) to `ml`; `where` tells the
    // joining kernel of each (row, head) the first of them, and their number * 64 + row of the tile (0: the row is done).
    int split;
    long long items;                    // workgroups of the grid per K/V head
    long long stride;                   // many requests, no split: from one workgroup's item to the next one's
    int tile_rows;
    float *partial;
    float2 *ml;
    int2 *where;
    int4 *plan;                         // kManyRows: where each of `split` pieces starts (request, tile, place), then the pieces' size and sum
    int tiles;                          // upper bound of the row tiles
};
// The way of a call: nt 16-row tiles per workgroup whose waves split the keys (1, 2 or 4), or kManyRows, where they split the rows;
// workgroups per K/V head that share the keys (0: no split), and the grid's items per K/V head.
constexpr int kManyRows = 0;
void paged_attn_plan(const odb_pages &p, int n, int rows, int group, int max_rows, long long max_len, long long columns, int *nt, int *split,
                     long long *items);
size_t paged_attn_workspace(const odb_pages &p, int rows, int heads, int nt, int split);
// Checks a call's sizes and fills the fields that follow from them (paged_api.hip); buffers: the pools' addresses are checked too
int plan_paged_attention(const odb_attention *a, const odb_pages *pages, bool buffers, PagedAttn &p, int &nt);
void launch_paged_attention(PagedAttn a, int nt, void *workspace, hipStream_t s);

}  // namespace odb
