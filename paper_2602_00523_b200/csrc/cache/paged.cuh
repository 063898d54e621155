// What the operators around the paged cache share: the tensor maps and settings of the attention entry points
// (tree_attention.cu), and the parameters of the paged kernel.
#pragma once

#include <cuda.h>

#include "sage_common.cuh"

namespace sage {

// tree_attention.cu
bool make_pool_map(CUtensorMap* map, const void* pool, int n_layers, int n_pages, int n_kv_heads, int64_t layer_stride_elems);
bool make_sealed_map(CUtensorMap* map, const void* pool, int n_layers, int n_pages, int n_kv_heads, int64_t layer_stride_bytes);
bool make_q_map(CUtensorMap* map, const void* q, int n_layers, int sum_nodes, int n_kv_heads, int G);
int resident_ctas();
long long attention_wait_cycles();
int attention_producer_off();

namespace paged {

struct Params {
    __nv_bfloat16* out;
    float4* part_o;    // [item behind the whole ones][slice][32 column quads][row_tiles*128 rows]   unnormalised
    float2* part_ml;   // [item behind the whole ones][slice][row_tiles*128 rows]                    (reference in log2 units, sum)
    const int32_t* page_table;
    const int32_t* page_table8;     // of the sealed pages
    const int32_t* sealed;          // sealed pages of each sequence; null: the cache is bf16 throughout
    const uint8_t* k_exp;           // [layer][page][KV head]
    const uint8_t* v_exp;
    const int32_t* seq_len;
    const int32_t* parent;
    const int32_t* node_offsets;
    int32_t* status;
    int n_layers, batch, sum_nodes, n_pages, max_pages, n_pages8, max_pages8;
    int Hq, Hkv, G, g_shift;        // G = 1 << g_shift query heads per KV head
    int n_whole, n_splits;          // items that are not cut, context slices of the others
    int in_cluster;                 // all items are cut, and the slices of a row tile are one cluster
    int row_tiles;                  // 128-row tiles of the largest possible tree
    int window, sink;
    float scale_log2;               // sm_scale * log2(e)
    long long wait_cycles;          // budget of every on-device wait
    int producer_off;               // diagnostics: the copy warp issues nothing
};

}  // namespace paged
}  // namespace sage
