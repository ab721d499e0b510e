// Device side of a batch of sequences: which tokens a sequence has, where they are in its cache, and page numbers that are checked before use.
#pragma once
#include "attention.h"
#include "epilogue.h"

namespace patch {

template <typename T>
__device__ __forceinline__ const PATCH_EP_GLOBAL T* as_global(const T* p) {
    return reinterpret_cast<const PATCH_EP_GLOBAL T*>(reinterpret_cast<uintptr_t>(p));
}
template <typename T>
__device__ __forceinline__ PATCH_EP_GLOBAL T* as_global_out(T* p) {
    return reinterpret_cast<PATCH_EP_GLOBAL T*>(reinterpret_cast<uintptr_t>(p));
}

struct Seq {
    int first, n;    // its tokens in the batch, inside [0, n_tokens] whatever q_start holds
    int len;         // its tokens in the cache, inside [0, max_kv]
    int pos0;        // position of its first token in the batch: may be negative, that token then has no place
    bool bad;        // kv_len beyond what the caller said or the table holds
};

__host__ __device__ inline int within(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
// from what the device arrays say, whatever that is
__host__ __device__ inline Seq seq_from(int t0, int t1, int len, int n_tokens, int max_kv) {
    Seq q;
    q.first = within(t0, 0, n_tokens);
    q.n = within(t1, q.first, n_tokens) - q.first;
    q.bad = len > max_kv;
    q.len = within(len, 0, max_kv);
    q.pos0 = q.len - q.n;
    return q;
}
// Which of its sequence's tokens row t of the call is; -1: rows in front of the first sequence's, or behind the last one's, are nobody's.
__host__ __device__ inline int place_of(const Seq& q, int t) { return t >= q.first && t - q.first < q.n ? t - q.first : -1; }
// Tile `tile` of kTurn positions (base on) of those that are new: [begin, q.len).  V is turned a tile at a time; none: there is nothing new in it.
constexpr int kTurn = 64;
struct NewTile { int begin, base; bool none; };
__host__ __device__ inline NewTile new_tile(const Seq& q, int tile) {
    NewTile n;
    n.begin = q.pos0 > 0 ? q.pos0 : 0;
    n.base = (n.begin & ~(kTurn - 1)) + tile * kTurn;
    n.none = q.bad || n.begin >= q.len || n.base >= q.len;       // (a sequence without new tokens begins at its end, also inside a tile)
    return n;
}
// The row of the call that position base + i of such a tile is read from: its token's, or another new one's if it is not new itself.
__host__ __device__ inline int row_of_new(const Seq& q, const NewTile& n, int i) { return q.first + (within(n.base + i, n.begin, q.len - 1) - q.pos0); }
__host__ __device__ inline int page_or_none(int id, int n_pages) { return id >= 0 && id < n_pages ? id : -1; }

__device__ __forceinline__ Seq seq_at(const SeqArgs& a, int s) {
    const int len = as_global(a.kv_len)[s];
    if (!a.q_start) return seq_from(s, s + 1, len, a.n_tokens, a.max_kv);
    return seq_from(as_global(a.q_start)[s], as_global(a.q_start)[s + 1], len, a.n_tokens, a.max_kv);
}

// The sequence of token t, if any has it (place_of tells): the last one whose tokens begin at or before t (those without tokens in between are passed over).
__device__ __forceinline__ int seq_of(const SeqArgs& a, int t) {
    const int same = min(t, a.n_seqs - 1);
    if (!a.q_start) return same;
    // where all have one token, sequence t has token t: known after one look
    if (a.n_tokens == a.n_seqs && as_global(a.q_start)[same] <= t && t < as_global(a.q_start)[same + 1]) return same;
    int lo = 0, hi = a.n_seqs - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (as_global(a.q_start)[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

}  // namespace patch
