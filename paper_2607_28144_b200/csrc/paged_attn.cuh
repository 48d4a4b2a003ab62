// Parameters of the attention over a paged cache (paged_attn.cu), shared with its entry point (cache_ops.cu).
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace regenvc {

constexpr int kPagedMaxGrid = 160;           // thread blocks of the attention kernel
constexpr int kPagedMaxSequences = 4096;
constexpr int kPagedRows = 256;              // rows of an item

// What a thread block left of an item it did not do alone: slot 0 an item's middle or end, slot 1 its beginning.
struct PagedPiece {
    int valid, ends;                         // ends: the item's last piece
    int seq_row0, first_row, rows, head;     // the item: first token row of its sequence, its rows, its head of the cache
};

struct PagedAttnParams {
    const void* q;
    void* out;
    float* lse;                              // [n_tokens][n_q_heads] or nullptr
    long long q_token, q_head, out_token, out_head;   // strides in elements
    const int* row_starts;                   // [n_sequences + 1]
    const int* lengths;                      // [n_sequences] cached tokens, the new ones among them
    const int* table;                        // [n_sequences][pages_per_sequence]
    long long table_stride;
    int n_tokens, n_sequences, n_q_heads, n_k_heads, share;   // share: query heads per head of the cache
    int page_size, n_pages, pages_per_sequence;
    int group, window;
    float scale_log2;
    int box_rows;                            // rows of the small boxes
    int one_page_box;                        // 1: a tile of keys may lie within one page and comes by one box of 128 rows
    int rounds;                              // 1: whole items in rounds first (several tiles of rows share keys)
    float4* part_o;                          // [slot][head_dim / 4][256 rows]
    float2* part_ml;                         // [slot][256 rows] (reference in log2 units, row sum)
    PagedPiece* pieces;                      // [slot]
    int* status;
};

inline int paged_attn_grid(int sm_count) { return sm_count < kPagedMaxGrid ? sm_count : kPagedMaxGrid; }
size_t paged_attn_workspace_bytes(int head_dim);
cudaError_t configure_paged_attn();
struct PagedMaps {
    CUtensorMap k, v, k_page, v_page;        // small boxes; boxes of 128 rows
};
cudaError_t launch_paged_attn(const PagedMaps& maps, const PagedAttnParams& p, int head_dim, bool f16, int sm_count,
                              int* launches, cudaStream_t stream);

}  // namespace regenvc
