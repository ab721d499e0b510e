// Launch interface of the attention side of a layer (rope.hip, attention.hip), filled in by attention_api.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace patch {

// A batch of sequences whose tokens lie side by side, and the rows of their page table.
struct SeqArgs {
    const int32_t* q_start;   // n_seqs + 1, or null: sequence s has the one token s
    const int32_t* kv_len;
    const int32_t* table;     // n_seqs x table_stride page numbers
    int64_t table_stride;
    int n_seqs, n_tokens;
    int max_q;
    int max_kv;               // no more than table_stride pages hold
};

struct CacheArgs {
    uint8_t *k, *v;           // pages: kv_heads x page x head_dim and kv_heads x head_dim x page cells
    int64_t page_bytes;       // from one page to the next
    const float *k_scale, *v_scale;   // per head, or null: 1
    int n_pages, page_log2, kv_heads, head_dim, e4m3;
};

struct HeadArgs {
    const uint8_t* x;
    int64_t stride;           // bytes from one token to the next
    const float* gamma;       // head_dim factors of the normed head, or null: not normed
    uint8_t* out;
    int64_t out_stride;       // bytes
    int heads;
};

struct RopeArgs {
    HeadArgs q, k, v;         // heads = 0: not there
    const float* table;       // n_pos x 2 x rot / 2
    const int32_t* positions; // null: from the sequences
    SeqArgs seqs;
    CacheArgs cache;          // k null: no cache, K goes to k.out
    int64_t n_tokens, n_pos;
    int head_dim, rot, interleaved, f32;
    int v_tiles;              // filled in by launch_rope
    float eps;
};
void launch_rope(const RopeArgs& a, hipStream_t stream);

struct AttnArgs {
    const uint16_t* Q;
    uint16_t* O;
    float* lse;               // n_tokens x heads, or null
    int64_t q_stride, o_stride;   // elements
    SeqArgs seqs;
    CacheArgs cache;
    int heads, group;         // query heads, and how many of them share a key head
    float scale;              // times log2(e)
    int prefix;               // keys [0, prefix) are the same for all: they take parts of their own
    int own_chunk;            // keys of a sequence's own that one workgroup takes: a multiple of 128, counted from prefix rounded down to 64
    int prefix_chunk, prefix_parts;
    int parts;                // prefix_parts + the most that a sequence's own keys are; 1: workgroups write O, else partial results
    // few rows a sequence: one launch of front_blocks workgroups for the shared front and line_waves wavefronts that have equal stretches (least_steps at least)
    // of all own keys, in steps of 64 keys (heads of 256: 32); 0: a workgroup for each sequence and key head
    int few, front_blocks, line_waves, least_steps;
    float* part_ml;           // parts x n_tokens x heads pairs: running maximum (of scores times log2(e)) and sum
    float* part_o;            // parts x n_tokens x heads x head_dim
    int* unit_parts;          // n_seqs x kv_heads: the parts of its own keys
};
// fills all that from own_chunk on for a workspace of ws_bytes (0: none), prefix too where it does without; returns the bytes used
size_t plan_attention(AttnArgs* a, size_t ws_bytes);
void launch_attention(const AttnArgs& a, hipStream_t stream);

}  // namespace patch
