// Eviction from a paged cache by the weight of its tokens (patch_kv_evict): which tokens stay, and the cells that move.
//
// Of each key head's tokens the `keep` of the largest rank stay; a rank is 32 bits: the weight as an ordered integer, the largest of all for tokens that always
// stay.  The border is found digit by digit (11, 11 and 10 bits) from histograms; of the tokens at the border those in the lowest slots stay.  Whoever
// stays in a slot below `keep` does not move: only the holes there are filled, from behind, so that sources and goals are apart and all cells move at once.
#include <algorithm>

#include "cells.h"

namespace patch {

// Larger: heavier.  NaN: 0; always staying: all ones (a number's is at most 0xFF800000, that of infinity).
__device__ __forceinline__ uint32_t rank_of(float w, bool always) {
    const uint32_t u = __float_as_uint(w);
    if (always) return 0xFFFFFFFFu;
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) return 0u;
    if ((u & 0x7FFFFFFFu) == 0u) return 0x80000000u;             // both zeros
    return u >> 31 ? ~u : u | 0x80000000u;
}

constexpr int kSelect = 1024;          // threads
constexpr int kChunk = 4 * kSelect;    // slots at a time

struct SelectLds {
    int count[2048];
    int wave[16][4];
    int movers[2 * kChunk];            // slots behind the budget whose tokens stay, as a ring
};

// Sums of x over the threads in front of this one, and of all.
__device__ __forceinline__ int before_me(int x, int (*wave)[4], int which, int* total) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int sum = x;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int other = __shfl_up(sum, m);
        if (lane >= m) sum += other;
    }
    if (lane == 63) wave[w][which] = sum;
    __syncthreads();
    int front = 0, all = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int n = wave[i][which];
        front += i < w ? n : 0;
        all += n;
    }
    __syncthreads();
    *total = all;
    return front + sum - x;
}

__global__ __launch_bounds__(kSelect) void evict_select_kernel(const EvictArgs a) {
    __shared__ SelectLds sh;
    const int kh = blockIdx.x % a.cache.kv_heads, s = blockIdx.x / a.cache.kv_heads, tid = threadIdx.x, keep = a.keep;
    const int64_t unit = (int64_t)s * a.cache.kv_heads + kh;
    const Seq q = seq_at(a.seqs, s);
    int32_t* from = a.from + unit * keep;
    const int len = q.bad ? 0 : q.len;
    if (len <= keep) {
        for (int i = tid; i < keep; i += kSelect) as_global_out(from)[i] = i < len ? i : -1;
        return;
    }
    const float* w = a.w + unit * a.w_stride;
    const int32_t* pos = a.positions ? a.positions + unit * a.w_stride : nullptr;
    // the largest position
    int newest = len - 1;
    if (pos) {
        newest = INT32_MIN;
        for (int i = tid; i < len; i += kSelect) newest = max(newest, as_global(pos)[i]);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) newest = max(newest, __shfl_xor(newest, m));
        if ((tid & 63) == 0) sh.wave[tid >> 6][0] = newest;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) newest = max(newest, sh.wave[i][0]);
        __syncthreads();
    }
    const int64_t recent = (int64_t)newest - a.recent;
    const auto rank_at = [&](int i) {
        const int p = pos ? as_global(pos)[i] : i;
        return rank_of(as_global(w)[i], p < a.sinks || p > recent);
    };
    // the border: `border` is the rank of the last that stays, `left` how many of that rank do
    uint32_t border = 0;
    int left = keep;
    for (int digit = 0; digit < 3; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bins = digit == 2 ? 1024 : 2048;
        for (int i = tid; i < bins; i += kSelect) sh.count[i] = 0;
        __syncthreads();
        for (int i = tid; i < len; i += kSelect) {
            const uint32_t r = rank_at(i);
            if (digit == 0 || r >> (shift + (digit == 1 ? 11 : 10)) == border >> (shift + (digit == 1 ? 11 : 10))) atomicAdd(&sh.count[(r >> shift) & (bins - 1)], 1);
        }
        __syncthreads();
        // bins from the largest on, two a thread: the one in which the sum reaches `left`
        const int top = bins - 1 - 2 * tid, n0 = top > 0 ? sh.count[top] : 0, n1 = top > 0 ? sh.count[top - 1] : 0;
        int total;
        const int front = before_me(n0 + n1, sh.wave, 0, &total);
        if (front < left && left <= front + n0 + n1) {
            const bool second = front + n0 < left;
            sh.wave[0][1] = top - (second ? 1 : 0);
            sh.wave[0][2] = left - front - (second ? n0 : 0);
        }
        __syncthreads();
        border |= (uint32_t)sh.wave[0][1] << shift;
        left = sh.wave[0][2];
        __syncthreads();
    }
    // slots in their order: which of the border's stay, the ranks of holes and of movers
    int ties = 0, holes = 0, movers = 0, ahead = keep;           // behind the budget `ahead` slots have been looked at
    int ties_ahead;
    {
        int mine = 0;
        for (int i = tid; i < keep; i += kSelect) mine += rank_at(i) == border;
        before_me(mine, sh.wave, 0, &ties_ahead);
    }
    for (int chunk = 0; chunk < keep; chunk += kChunk) {
        bool stays[4];
        int equal[4], n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = chunk + 4 * tid + e;
            const uint32_t r = i < keep ? rank_at(i) : 0xFFFFFFFFu;
            equal[e] = i < keep && r == border;
            stays[e] = i >= keep || r > border;
            n += equal[e];
        }
        int total;
        int tie = ties + before_me(n, sh.wave, 0, &total);
        ties += total;
        n = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (equal[e]) stays[e] = tie++ < left;
            n += !stays[e];
        }
        int hole = holes + before_me(n, sh.wave, 1, &total);
        holes += total;
        // as many movers as these holes take
        while (movers < holes && ahead < len) {
            int m = 0, eq = 0;
            bool goes[4], same[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = ahead + 4 * tid + e;
                const uint32_t r = i < len ? rank_at(i) : 0u;
                same[e] = i < len && r == border;
                goes[e] = i < len && r > border;
                eq += same[e];
            }
            int tied = ties_ahead + before_me(eq, sh.wave, 2, &total);
            ties_ahead += total;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (same[e]) goes[e] = tied++ < left;
                m += goes[e];
            }
            int at = movers + before_me(m, sh.wave, 3, &total);
            movers += total;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (goes[e]) sh.movers[at++ % (2 * kChunk)] = ahead + 4 * tid + e;
            ahead += kChunk;
            __syncthreads();
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = chunk + 4 * tid + e;
            if (i < keep) as_global_out(from)[i] = stays[e] ? i : sh.movers[hole % (2 * kChunk)];
            hole += !stays[e];
        }
        __syncthreads();
    }
}

// Cells to where `from` says: 64 slots of a sequence's head by a workgroup, lanes beside each other with slots beside each other.
template <int CELL>     // bytes of a cell of V's rows: 2, 1 (e4m3), 0: pairs of 4 bits and powers
__device__ __forceinline__ void move_slots(const EvictArgs& a, int s, int kh, int first) {
    __shared__ int sh_to[64], sh_from[64], sh_n;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, slot = first + lane;
    const int64_t unit = (int64_t)s * a.cache.kv_heads + kh;
    const int came = slot < a.keep ? as_global(a.from)[unit * a.keep + slot] : -1;
    if (wave == 0) {
        if (came >= 0) {
            const int64_t to = unit * a.w_stride + slot, at = unit * a.w_stride + came;
            if (a.w_out) as_global_out(a.w_out)[to] = as_global(a.w)[at];
            if (a.positions_out) as_global_out(a.positions_out)[to] = a.positions ? as_global(a.positions)[at] : came;
        }
        const bool moves = came >= 0 && came != slot;
        const uint64_t all = __ballot(moves);
        if (moves) {
            const int i = __builtin_popcountll(all & ((1ull << lane) - 1));
            sh_to[i] = slot;
            sh_from[i] = came;
        }
        if (lane == 0) sh_n = __builtin_popcountll(all);
    }
    __syncthreads();
    const int n = sh_n, p = a.cache.page_log2, mask = (1 << p) - 1, D = a.cache.head_dim;
    if (lane >= n) return;
    const int to = sh_to[lane], at = sh_from[lane];
    const PATCH_EP_GLOBAL int32_t* table = as_global(a.seqs.table) + s * a.seqs.table_stride;
    const int64_t dst = page_or_none(table[to >> p], a.cache.n_pages), src = page_or_none(table[at >> p], a.cache.n_pages);
    if (dst < 0 || src < 0) return;
    const int64_t head = (int64_t)kh << p;
    const auto copy = [&](auto* base, int64_t stride, int64_t goal, int64_t source) {    // of one element
        typedef typename std::remove_reference<decltype(*base)>::type T;
        const uint8_t* b = reinterpret_cast<const uint8_t*>(base);
        *reinterpret_cast<PATCH_EP_GLOBAL T*>(as_global_out(const_cast<uint8_t*>(b)) + dst * stride + goal) =
            *reinterpret_cast<const PATCH_EP_GLOBAL T*>(as_global(b) + src * stride + source);
    };
    const int bytes = CELL == 0 ? D / 2 : D * CELL;
    const int64_t k_to = (head + (to & mask)) * bytes, k_at = (head + (at & mask)) * bytes;
    for (int c = 16 * wave; c < bytes; c += 64) copy(reinterpret_cast<u32x4_t*>(a.cache.k), a.cache.page_bytes, k_to + c, k_at + c);
    const int features = CELL == 0 ? D / 2 : D;
    const int64_t row = (int64_t)kh * features;
    for (int d = wave; d < features; d += 4) {
        const int64_t f = (row + d) << p;
        if constexpr (CELL == 2) copy(reinterpret_cast<uint16_t*>(a.cache.v), a.cache.page_bytes, 2 * (f + (to & mask)), 2 * (f + (at & mask)));
        else copy(a.cache.v, a.cache.page_bytes, f + (to & mask), f + (at & mask));
    }
    if constexpr (CELL == 0) {
        const int powers = D / 32;
        for (int b = wave; b < powers; b += 4) {
            copy(a.cache.k_power, a.cache.power_bytes, (head + (to & mask)) * powers + b, (head + (at & mask)) * powers + b);
            const int64_t f = ((int64_t)kh * powers + b) << p;
            copy(a.cache.v_power, a.cache.power_bytes, f + (to & mask), f + (at & mask));
        }
    }
}

template <int CELL>
__global__ __launch_bounds__(256) void evict_move_kernel(const EvictArgs a) {
    const int kh = blockIdx.x % a.cache.kv_heads, s = blockIdx.y;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        const int len = as_global(a.seqs.kv_len)[s];
        as_global_out(a.kv_len_out)[s] = len > a.seqs.max_kv ? len : max(min(len, a.keep), 0);
    }
    const int most = min(a.keep, a.seqs.max_kv);                 // (behind that nobody has tokens)
    for (int first = blockIdx.x / a.cache.kv_heads * 64; first < most; first += gridDim.x / a.cache.kv_heads * 64) {
        move_slots<CELL>(a, s, kh, first);
        __syncthreads();
    }
}

void launch_evict(const EvictArgs& a, hipStream_t stream) {
    const unsigned heads = (unsigned)a.cache.kv_heads;
    evict_select_kernel<<<(unsigned)a.seqs.n_seqs * heads, kSelect, 0, stream>>>(a);
    const unsigned chunks = (unsigned)std::min<int64_t>(((int64_t)std::min(a.keep, std::max(a.seqs.max_kv, 1)) + 63) / 64, std::max((1u << 22) / heads, 1u));
    const dim3 grid(chunks * heads, (unsigned)a.seqs.n_seqs);
    if (a.cache.cells == kBf16) evict_move_kernel<2><<<grid, 256, 0, stream>>>(a);
    else if (a.cache.cells == kE4m3) evict_move_kernel<1><<<grid, 256, 0, stream>>>(a);
    else evict_move_kernel<0><<<grid, 256, 0, stream>>>(a);
}

}  // namespace patch
