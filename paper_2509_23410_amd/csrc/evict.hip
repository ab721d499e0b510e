// Eviction from a paged cache by the weight of its tokens (patch_kv_evict): which tokens stay, and the cells that move.
//
// Of each key head's tokens the `keep` of the largest rank stay; a rank is 32 bits: the weight as an ordered integer, the largest of all for tokens that always
// stay.  The border is found digit by digit (11, 11 and 10 bits) from histograms; of the tokens at the border those in the lowest slots stay.  Whoever
// stays in a slot below `keep` does not move: only the holes there are filled, from behind, so that sources and goals are apart and all cells move at once, and a
// budget that is one token too small costs one token's move.
//
// Two launches: who stays (a workgroup for each sequence and key head; `from` is what it says), then the moves.  64 sequences of 4097 tokens to 4096, 8 key heads: 16 + 15
// us, waits of one step for the other; 4 prompts of up to 16000 to 2048, 32 key heads, e4m3: 12 + 75, V's cells, each in a line of the cache of its own; one of 131000
// to 32768, 8 key heads in 4 bits: 61 + 42, eight compute units' instructions.
#include <algorithm>

#include "cells.h"

namespace patch {

// Larger: heavier.  NaN: 0; always staying: all ones (a number's is at most 0xFF800000, that of infinity).
__device__ __forceinline__ uint32_t rank_of(float w, bool always) {
    const int u = __float_as_int(w + 0.f);                       // both zeros are one
    const uint32_t r = w != w ? 0u : (uint32_t)(u ^ (u >> 31 | INT32_MIN));
    return always ? 0xFFFFFFFFu : r;
}
// Positions that always stay: those below `sinks`, and if `any` those from `last` on.
struct Always {
    int sinks, last;
    bool any;
    __device__ __forceinline__ bool operator()(int p) const { return p < sinks || (any && p >= last); }
};

// Sums over the lanes up to this one: of its row of 16, and of all.
__device__ __forceinline__ uint32_t row_sums(uint32_t x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, true);      // lanes 1, 2, 4 and 8 in front
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, true);
    return x;
}
__device__ __forceinline__ uint32_t lane_sums(uint32_t x) {
    x = row_sums(x);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);     // the last lane of rows 0 and 2 to rows 1 and 3, then that of row 1 to rows 2 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
    return x;
}

constexpr int kThreads = 1024, kWaves = kThreads / 64;   // (of 256 threads 64 sequences of 4097 slots, 8 key heads, took 24 us for 20)
constexpr int kStrip = 4 * kThreads;                     // slots that they have four each of, side by side

// The ranks of J strips of slots from `base` on: strip j's slots 4 tid .. 4 tid + 3 in r[j].
template <int J>
struct Ranks {
    uint32_t r[J][4];
    u32x4_t at[J], asked[J];           // positions, and weights as they are loaded (rows of both are a multiple of four apart)
    int base, begin, len;              // there are those in [begin, len)

    __device__ __forceinline__ int slot(int j) const { return base + j * kStrip + 4 * (int)threadIdx.x; }
    __device__ __forceinline__ void ask(const float* w, const int32_t* pos, int first, int length) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int i = first + j * kStrip + 4 * (int)threadIdx.x;
            asked[j] = u32x4_t{0, 0, 0, 0};
            if (i < length) asked[j] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(w) + i);
            if (pos && i < length) at[j] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(pos) + i);
        }
    }
    // the largest position of those asked for
    __device__ __forceinline__ int newest(int length) const {
        int top = INT32_MIN;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j * kStrip + 4 * (int)threadIdx.x + e < length) top = max(top, (int)at[j][e]);
        return top;
    }
    __device__ __forceinline__ void frame(int first, int lowest, int length) {
        base = first;
        begin = lowest;
        len = length;
    }
    // J strips full of slots from all over [0, length): every so many fours of them
    __device__ __forceinline__ void sample(const float* w, const int32_t* pos, int length, const Always& always) {
        const int64_t fours = length / 4;
        int i[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            i[j] = 4 * (int)((j * kThreads + (int)threadIdx.x) * fours / (J * kThreads));
            asked[j] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(w) + i[j]);
            if (pos) at[j] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(pos) + i[j]);
        }
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) r[j][e] = rank_of(__uint_as_float(asked[j][e]), always(pos ? (int)at[j][e] : i[j] + e));
        frame(0, 0, J * kStrip);
    }
    // what was asked for
    __device__ __forceinline__ void take(const int32_t* pos, int first, int lowest, int length, const Always& always) {
        frame(first, lowest, length);
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) r[j][e] = rank_of(__uint_as_float(asked[j][e]), always(pos ? (int)at[j][e] : slot(j) + e));
    }
    // whether strip j is all there, and else a bit for each of the thread's slots that is
    __device__ __forceinline__ bool whole(int j) const { return base + j * kStrip >= begin && base + (j + 1) * kStrip <= len; }
    __device__ __forceinline__ uint32_t bits(int j) const {
        uint32_t b = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) b |= slot(j) + e >= begin && slot(j) + e < len ? 1u << e : 0u;
        return b;
    }
    // f(rank) of those that there are
    template <typename F>
    __device__ __forceinline__ void each(const F& f) const {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            if (whole(j)) {
#pragma unroll
                for (int e = 0; e < 4; ++e) f(r[j][e]);
            } else {
                const uint32_t b = bits(j);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (b >> e & 1) f(r[j][e]);
            }
        }
    }
};

// Histograms are four side by side, of every fourth lane each: an atomic add takes as long as its most frequent address has lanes.
constexpr int kCopies = 4, kBins = 2048;

// Slots whose tokens stay are a bit each where a head has more than registers hold; of so many at most.  Those near the border (between the kMargin-th of the sample in
// front of it and the kMargin-th behind, see near_border) are a list of ranks and slots.  It holds as many as the longest of these heads is expected to have there and
// five standard deviations more (sqrt(2 kMargin) of the sample's): with 8192 the list ran out from 200000 slots on, and 205000, half of which stay, took 276 us for 140.
constexpr int kMaskWords = 6656, kMargin = 320, kNear = 10240;
static_assert(kNear >= 32 * kMaskWords / 16384 * (2 * kMargin + 5 * 26), "the list and the bits are for heads of the same length");

template <int J, int RING, int MASK>
struct SelectLds {
    int count[kBins * kCopies];
    uint32_t strip[J][kWaves];         // counts of a strip's wavefronts
    int wave[kWaves], found[3];
    int movers[MASK > 1 && RING < 2 * kNear ? 2 * kNear : RING];      // a ring of slots behind the budget whose tokens stay, or the list of those near the border
    uint32_t mask[MASK];
};

// front[j] = the sums of x[j] (two counts of 16 bits) over the threads in front of this one in strip j, total[j] = of the whole strip
template <int J>
__device__ __forceinline__ void before_me(const uint32_t (&x)[J], uint32_t (*strip)[kWaves], uint32_t (&front)[J], uint32_t (&total)[J]) {
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const uint32_t sum = lane_sums(x[j]);
        if (lane == 63) strip[j][w] = sum;
        front[j] = sum - x[j];
    }
    __syncthreads();
#pragma unroll
    for (int j0 = 0; j0 < J; j0 += 4) {                          // the wavefronts of four strips at a time, one a lane
        const uint32_t n = j0 + (lane >> 4) < J ? strip[j0 + (lane >> 4)][lane & 15] : 0, sum = row_sums(n);
#pragma unroll
        for (int j = j0; j < J && j < j0 + 4; ++j) {
            front[j] += __builtin_amdgcn_readlane(sum - n, 16 * (j - j0) + w);
            total[j] = __builtin_amdgcn_readlane(sum, 16 * (j - j0) + 15);
        }
    }
    __syncthreads();
}
// The sum of x over all threads, added to by each wavefront.
__device__ __forceinline__ int sum_of_all(int x, int* wave) {
    const uint32_t sum = lane_sums((uint32_t)x);
    if ((threadIdx.x & 63) == 63) wave[threadIdx.x >> 6] = (int)sum;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) all += wave[i];
    __syncthreads();
    return all;
}

// The `left`-th largest of the ranks that each(f) calls f with, to its first `digits` digits of 11, 11 and 10 bits: the rank (those of them), how many ranks that
// are the same there are counted with it, and how many of them there are.
struct Border { uint32_t rank; int left, same; };
template <typename Lds, typename Each>
__device__ __forceinline__ Border select(Lds& sh, int digits, int left, const Each& each) {
    const int tid = threadIdx.x, lane = tid & 63;
    Border b = {0u, left, 0};
    for (int digit = 0; digit < digits; ++digit) {
        const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, bins = digit == 2 ? kBins / 2 : kBins, above = digit == 0 ? 31 : digit == 1 ? 21 : 10;
        for (int i = tid; i < bins; i += kThreads) *reinterpret_cast<u32x4_t*>(&sh.count[kCopies * i]) = u32x4_t{0, 0, 0, 0};
        __syncthreads();
        each([&](uint32_t r) {
            if (digit == 0 || r >> above == b.rank >> above) atomicAdd(&sh.count[kCopies * ((r >> shift) & (bins - 1)) + (lane & (kCopies - 1))], 1);
        });
        __syncthreads();
        // bins from the largest on, kBins / kThreads a thread (the last digit: half of them): the one in which the sum reaches `left`
        const auto in_bin = [&](int i) {
            const u32x4_t n = *reinterpret_cast<const u32x4_t*>(&sh.count[kCopies * i]);
            return (int)(n[0] + n[1] + n[2] + n[3]);
        };
        const int per = bins / kThreads, top = bins - 1 - per * tid;
        int n[kBins / kThreads], sum = 0;
#pragma unroll
        for (int i = 0; i < kBins / kThreads; ++i) {
            n[i] = i < per ? in_bin(top - i) : 0;
            sum += n[i];
        }
        const int upto = (int)lane_sums((uint32_t)sum);
        if (lane == 63) sh.wave[tid >> 6] = upto;
        __syncthreads();
        int front = upto - sum;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) front += i < tid >> 6 ? sh.wave[i] : 0;
        if (front < b.left && b.left <= front + sum) {
#pragma unroll
            for (int i = 0; i < kBins / kThreads; ++i) {
                if (front < b.left && b.left <= front + n[i]) {
                    sh.found[0] = top - i;
                    sh.found[1] = b.left - front;
                }
                front += n[i];
            }
        }
        __syncthreads();
        b.rank |= (uint32_t)sh.found[0] << shift;
        b.left = sh.found[1];
        b.same = in_bin(sh.found[0]);
        __syncthreads();
    }
    return b;
}

// Slots of a block in their order: which stay, and the ranks of holes and of movers among their like.  `left` of the border's stay, the first ones, `ties` of which have
// been seen; some: not all of them do.
template <int J>
struct Block {
    uint32_t stays[J], front[J], total[J];      // a bit each; holes in the low half, movers in the high one: in front in the strip, and in all of it

    __device__ __forceinline__ void look(const Ranks<J>& k, uint32_t (*strip)[kWaves], int keep, uint32_t border, bool some, int left, int* ties) {
        uint32_t there[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            there[j] = k.whole(j) ? 15u : k.bits(j);
            stays[j] = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) stays[j] |= k.r[j][e] >= border ? 1u << e : 0u;
            stays[j] &= there[j];
        }
        if (some) {
            uint32_t n[J];
#pragma unroll
            for (int j = 0; j < J; ++j) {
                n[j] = 0;
#pragma unroll
                for (int e = 0; e < 4; ++e) n[j] += k.r[j][e] == border && (there[j] >> e & 1);
            }
            before_me<J>(n, strip, front, total);
#pragma unroll
            for (int j = 0; j < J; ++j) {
                int tie = *ties + (int)front[j];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (k.r[j][e] == border && (there[j] >> e & 1) && tie++ >= left) stays[j] &= ~(1u << e);
                *ties += (int)total[j];
            }
        }
        sums(k, there, strip, keep);
    }
    __device__ __forceinline__ void sums(const Ranks<J>& k, const uint32_t (&there)[J], uint32_t (*strip)[kWaves], int keep) {
        uint32_t n[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int within = min(max(keep - k.slot(j), 0), 4);             // of the thread's four
            const uint32_t low = (1u << within) - 1;
            n[j] = __builtin_popcount(there[j] & ~stays[j] & low) + (__builtin_popcount(stays[j] & ~low) << 16);
        }
        before_me<J>(n, strip, front, total);
    }
    __device__ __forceinline__ int holes() const {
        int n = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) n += (int)(total[j] & 0xFFFFu);
        return n;
    }
    // the movers' slots into a ring, `movers` of them are in it
    template <int RING>
    __device__ __forceinline__ void collect(const Ranks<J>& k, int keep, int* ring, int* movers) const {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            int at = *movers + (int)(front[j] >> 16);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (k.slot(j) + e >= keep && (stays[j] >> e & 1)) ring[at++ % RING] = k.slot(j) + e;
            *movers += (int)(total[j] >> 16);
        }
    }
    // what is in the slots within the budget afterwards; `holes` were in front
    template <int RING>
    __device__ __forceinline__ void fill(const Ranks<J>& k, int keep, const int* ring, int* holes, int32_t* from) const {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            int hole = *holes + (int)(front[j] & 0xFFFFu);
            typedef int Four32 __attribute__((ext_vector_type(4), aligned(4)));
            const int i = k.slot(j);
            Four32 came = {i, i + 1, i + 2, i + 3};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < keep && !(stays[j] >> e & 1)) came[e] = ring[hole++ % RING];
            if (i + 3 < keep) {
                *reinterpret_cast<PATCH_EP_GLOBAL Four32*>(as_global_out(from) + i) = came;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e < keep) as_global_out(from)[i + e] = came[e];
            }
            *holes += (int)(total[j] & 0xFFFFu);
        }
    }
};

// The bits of those that stay, in one pass over the ranks: 16384 of them say between which two the border lies, those above it stay, and only those in between
// are looked at closely.  A histogram of all takes four times as long, by its atomic adds.  False: the border is not in between, or too many are (or are the same) there.
template <int J, typename Lds, typename Stream>
__device__ __forceinline__ bool near_border(Ranks<J>& ranks, Lds& sh, int keep, int len, const float* w, const int32_t* pos, const Always& always, const Stream& stream) {
    static_assert(J * kStrip == 16384, "a sample");
    // (kMargin is five standard deviations of how many of 16384 are above the border, where that is the median)
    const int tid = threadIdx.x, lane = tid & 63;
    if (len > 32 * kMaskWords) return false;
    ranks.sample(w, pos, len, always);
    const int at = (int)((int64_t)keep * (J * kStrip) / len);
    const auto all = [&](const auto& f) { ranks.each(f); };
    const uint32_t high = at - kMargin < 1 ? 0xFFFFFFFFu : select(sh, 2, at - kMargin, all).rank | 0x3FFu;
    const uint32_t low = at + kMargin > J * kStrip ? 0u : select(sh, 2, at + kMargin, all).rank;
    if (tid == 0) sh.found[2] = 0;
    __syncthreads();
    int sure = 0;
    stream(len, [&] {
        int mine = 0;
        uint32_t near[J];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const uint32_t there = ranks.whole(j) ? 15u : ranks.bits(j);
            uint32_t stay = 0, maybe = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                stay |= ranks.r[j][e] > high ? 1u << e : 0u;
                maybe |= ranks.r[j][e] >= low ? 1u << e : 0u;
            }
            stay &= there;
            near[j] = maybe & there & ~stay;
            sure += __builtin_popcount(stay);
            mine += __builtin_popcount(near[j]);
            const uint32_t next = __builtin_amdgcn_update_dpp(0, stay, 0xB1, 0xF, 0xF, true);      // the neighbour's
            if ((tid & 1) == 0 && ranks.slot(j) < 32 * kMaskWords) reinterpret_cast<uint8_t*>(sh.mask)[ranks.slot(j) >> 3] = (uint8_t)(stay | next << 4);
        }
        const int upto = (int)lane_sums((uint32_t)mine);
        int to = 0;
        if (lane == 63 && upto) to = atomicAdd(&sh.found[2], upto);
        to = __builtin_amdgcn_readlane(to, 63) + upto - mine;
        if (!mine) return;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (near[j] >> e & 1) {
                    if (to < kNear) {
                        sh.movers[2 * to] = (int)ranks.r[j][e];
                        sh.movers[2 * to + 1] = ranks.slot(j) + e;
                    }
                    ++to;
                }
    });
    const int need = keep - sum_of_all(sure, sh.wave), n = sh.found[2];
    if (n > kNear || need < 0 || need > n) return false;
    if (need == 0) return true;
    // (their first digits are much the same: what they are above `low` is spread over all bits)
    const int wide = __builtin_clz((high - low) | 1u);
    Border border = select(sh, 3, need, [&](const auto& f) {
        for (int i = tid; i < n; i += kThreads) f(((uint32_t)sh.movers[2 * i] - low) << wide);
    });
    border.rank = (border.rank >> wide) + low;
    const bool some = border.left < border.same;
    if (some && border.same > kThreads) return false;
    if (tid == 0) sh.found[2] = 0;
    __syncthreads();
    const auto stays = [&](int slot) { atomicOr(&sh.mask[slot >> 5], 1u << (slot & 31)); };
    for (int i = tid; i < n; i += kThreads) {
        const uint32_t r = (uint32_t)sh.movers[2 * i];
        if (r > border.rank || (r == border.rank && !some)) stays(sh.movers[2 * i + 1]);
        else if (r == border.rank) sh.count[atomicAdd(&sh.found[2], 1)] = sh.movers[2 * i + 1];
    }
    __syncthreads();
    if (some && tid < border.same) {                             // those in the lowest slots
        const int slot = sh.count[tid];
        int lower = 0;
        for (int i = 0; i < border.same; ++i) lower += sh.count[i] < slot;
        if (lower < border.left) stays(slot);
    }
    __syncthreads();
    return true;
}

// What is in the slots within the budget, from the bits of those that stay: each thread has words of 32 slots, and the movers of a word's holes follow each other.
template <typename Lds>
__device__ __forceinline__ void fill_from_bits(Lds& sh, int keep, int len, int32_t* from) {
    const int tid = threadIdx.x, lane = tid & 63, words = (len + 31) / 32, per = (words + kThreads - 1) / kThreads, first = min(tid * per, words);
    int sum = 0;
    for (int i = first; i < min(first + per, words); ++i) sum += __builtin_popcount(sh.mask[i]);
    const int upto = (int)lane_sums((uint32_t)sum);
    if (lane == 63) sh.wave[tid >> 6] = upto;
    __syncthreads();                                             // (and the list of candidates is done with)
    int front = upto - sum;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) front += i < tid >> 6 ? sh.wave[i] : 0;
    int* before = sh.movers;                                     // bits in front of each word
    for (int i = first; i < min(first + per, words); ++i) {
        before[i] = front;
        front += __builtin_popcount(sh.mask[i]);
    }
    __syncthreads();
    const int within = before[keep >> 5] + __builtin_popcount(sh.mask[keep >> 5] & ((1u << (keep & 31)) - 1));       // bits of slots within the budget
    for (int w = tid; 32 * w < keep; w += kThreads) {
        const uint32_t stay = sh.mask[w];
        const int bit = within + 32 * w - before[w];             // that of the first hole's mover
        int lo = keep >> 5, hi = words - 1;                      // the word that it is in
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (before[mid] <= bit) lo = mid; else hi = mid - 1;
        }
        uint32_t rest = sh.mask[lo];
        for (int i = before[lo]; i < bit; ++i) rest &= rest - 1;
#pragma unroll 1
        for (int i = 32 * w; i < min(32 * w + 32, keep); i += 4) {
            typedef int Four32 __attribute__((ext_vector_type(4), aligned(4)));
            Four32 came = {i, i + 1, i + 2, i + 3};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (i + e >= keep || (stay >> ((i + e) & 31) & 1)) continue;
                while (rest == 0 && lo + 1 < words) rest = sh.mask[++lo];
                came[e] = 32 * lo + __builtin_ctz(rest | 0x80000000u);
                rest &= rest - 1;
            }
            if (i + 3 < keep) {
                *reinterpret_cast<PATCH_EP_GLOBAL Four32*>(as_global_out(from) + i) = came;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e < keep) as_global_out(from)[i + e] = came[e];
            }
        }
    }
}

// One workgroup for each sequence and key head.  WHOLE: its ranks stay in registers (J strips hold all of them), else they are read again in each pass.
template <int J, bool WHOLE>
__global__ __launch_bounds__(kThreads) void evict_select_kernel(const EvictArgs a) {
    constexpr int B = WHOLE ? J : 2;                            // strips of a block in the last pass
    constexpr int kRing = WHOLE ? J * kStrip / 2 : 2 * B * kStrip;              // of `len` slots at most half move
    __shared__ alignas(16) SelectLds<B, kRing, WHOLE ? 1 : kMaskWords> sh;
    const int kh = blockIdx.x % a.cache.kv_heads, s = blockIdx.x / a.cache.kv_heads, tid = threadIdx.x, lane = tid & 63, keep = a.keep;
    const int64_t unit = (int64_t)s * a.cache.kv_heads + kh;
    const Seq q = seq_at(a.seqs, s);
    int32_t* from = a.from + unit * keep;
    const int len = q.bad ? 0 : q.len;
    if (len <= keep) {
        for (int i = tid; i < keep; i += kThreads) as_global_out(from)[i] = i < len ? i : -1;
        return;
    }
    const float* w = a.w + unit * a.w_stride;
    const int32_t* pos = a.positions ? a.positions + unit * a.w_stride : nullptr;
    Ranks<J> ranks;
    if (WHOLE) ranks.ask(w, pos, 0, len);
    int newest = len - 1;                                        // the largest position
    if (pos) {
        newest = INT32_MIN;
        if (WHOLE) newest = ranks.newest(len);
        else
            for (int i = 4 * tid; i < len; i += 4 * kStrip) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = min(i + j * kStrip, (len - 1) & ~3);
                    const u32x4_t x = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(pos) + at);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (at + e < len) newest = max(newest, (int)x[e]);
                }
            }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) newest = max(newest, __shfl_xor(newest, m));
        if (lane == 0) sh.wave[tid >> 6] = newest;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kWaves; ++i) newest = max(newest, sh.wave[i]);
    }
    const Always always = {a.sinks, (int)max((int64_t)newest - a.recent + 1, (int64_t)INT32_MIN), a.recent > 0};
    if (WHOLE) ranks.take(pos, 0, 0, len, always);
    // f() with the ranks of the slots [0, length), J strips at a time, the next ones on their way
    const auto stream = [&](int length, const auto& f) {
        ranks.ask(w, pos, 0, length);
        for (int first = 0; first < length; first += J * kStrip) {
            ranks.take(pos, first, 0, length, always);
            if (first + J * kStrip < length) ranks.ask(w, pos, first + J * kStrip, length);
            f();
        }
    };
    int holes = 0, movers = 0, ties = 0;
    if constexpr (WHOLE) {
        const Border border = select(sh, 3, keep, [&](const auto& f) { ranks.each(f); });
        Block<J> block;
        block.look(ranks, sh.strip, keep, border.rank, border.left < border.same, border.left, &ties);
        block.template collect<kRing>(ranks, keep, sh.movers, &movers);
        __syncthreads();
        block.template fill<kRing>(ranks, keep, sh.movers, &holes, from);
    } else {
        Ranks<B> here, behind;
        Block<B> block, other;
        int ahead = keep & ~3;
        if (near_border(ranks, sh, keep, len, w, pos, always, stream)) {
            fill_from_bits(sh, keep, len, from);
            return;
        }
        const Border border = select(sh, 3, keep, [&](const auto& f) { stream(len, [&] { ranks.each(f); }); });
        const bool some = border.left < border.same;             // not all of the border's stay: those in the lowest slots
        int ties_behind = 0;                                     // the border's behind the budget come after all of those within it
        if (some) {
            int mine = 0;
            stream(keep, [&] { ranks.each([&](uint32_t r) { mine += r == border.rank; }); });
            ties_behind = sum_of_all(mine, sh.wave);
        }
        // as many movers as the holes so far take
        behind.ask(w, pos, ahead, len);
        here.ask(w, pos, 0, keep);
        for (int first = 0; first < keep; first += B * kStrip) {
            here.take(pos, first, 0, keep, always);
            if (first + B * kStrip < keep) here.ask(w, pos, first + B * kStrip, keep);
            block.look(here, sh.strip, keep, border.rank, some, border.left, &ties);
            while (movers < holes + block.holes() && ahead < len) {
                behind.take(pos, ahead, keep, len, always);
                ahead += B * kStrip;
                if (ahead < len) behind.ask(w, pos, ahead, len);
                other.look(behind, sh.strip, keep, border.rank, some, border.left, &ties_behind);
                other.template collect<kRing>(behind, keep, sh.movers, &movers);
            }
            __syncthreads();
            block.template fill<kRing>(here, keep, sh.movers, &holes, from);
            __syncthreads();
        }
    }
}

// Cells to where `from` says, by workgroups of 256 slots of a sequence's head, and the weights and positions of all its slots.
template <int CELL>     // bytes of a cell of V's rows: 2, 1 (e4m3), 0: pairs of 4 bits and powers
__device__ __forceinline__ void move_slots(const EvictArgs& a, int s, int kh, int first) {
    __shared__ int sh_to[256], sh_from[256], sh_n[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, slot = first + tid;
    const int64_t unit = (int64_t)s * a.cache.kv_heads + kh;
    const int came = slot < a.keep ? as_global(a.from)[unit * a.keep + slot] : -1;
    if (came >= 0) {
        const int64_t to = unit * a.w_stride + slot, at = unit * a.w_stride + came;
        if (a.w_out) as_global_out(a.w_out)[to] = as_global(a.w)[at];
        if (a.positions_out) as_global_out(a.positions_out)[to] = a.positions ? as_global(a.positions)[at] : came;
    }
    const bool moves = came >= 0 && came != slot;
    const uint64_t all = __ballot(moves);
    if (lane == 0) sh_n[wave] = __builtin_popcountll(all);
    __syncthreads();
    int n = 0, mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mine += i < wave ? sh_n[i] : 0;
        n += sh_n[i];
    }
    if (n == 0) return;
    const int p = a.cache.page_log2, mask = (1 << p) - 1, D = a.cache.head_dim;
    if (moves) {
        mine += __builtin_popcountll(all & ((1ull << lane) - 1));
        sh_to[mine] = slot;
        sh_from[mine] = came;
    }
    __syncthreads();
    const PATCH_EP_GLOBAL int32_t* table = as_global(a.seqs.table) + s * a.seqs.table_stride;
    // pages of a move, -1: not to be followed
    const auto page = [&](int slot_of) { return (int64_t)page_or_none(table[slot_of >> p], a.cache.n_pages); };
    constexpr int kBatch = 8;                                    // loads that a thread has on their way: a store may not pass a load that could be of its cell
    // rows of K: 16-byte pieces of a row by neighbouring threads
    const int bytes = CELL == 0 ? D / 2 : D * CELL, pieces = __builtin_ctz(bytes / 16);
    for (int item = tid; item < n << pieces; item += 256 * kBatch) {
        u32x4_t x[kBatch];
        int64_t goal[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int i = item + 256 * b;
            goal[b] = -1;
            if (i >= n << pieces) continue;
            const int to = sh_to[i >> pieces], at = sh_from[i >> pieces], c = 16 * (i & ((1 << pieces) - 1));
            const int64_t dst = page(to), src = page(at);
            if (dst < 0 || src < 0) continue;
            goal[b] = dst * a.cache.page_bytes + (((int64_t)kh << p) + (to & mask)) * bytes + c;
            x[b] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(a.cache.k) + src * a.cache.page_bytes + (((int64_t)kh << p) + (at & mask)) * bytes + c);
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b)
            if (goal[b] >= 0) *reinterpret_cast<PATCH_EP_GLOBAL u32x4_t*>(as_global_out(a.cache.k) + goal[b]) = x[b];
    }
    // V, and powers: a cell of a row for neighbouring moves by neighbouring threads, the rows of a token by others
    // 2^side moves at a time: a row of 32 bytes or less shares its line of the cache with the next ones, which other lanes then have.  4 prompts of up to 16000 tokens
    // (rows of 32 bytes) 93.9 us with 64 moves at a time, 75.1 with 16, 78.2 with 8; 131000 tokens (rows of 64 bytes) 42.4, 32 46.9, 16 61.7.
    const int wide = (CELL == 2 ? 2 : 1) << p <= 32 ? 4 : 6, side = n <= 1 ? 0 : min(wide, 32 - __builtin_clz(n - 1));
    const auto cells = [&](auto* base, int64_t stride, int rows, bool by_token) {
        typedef typename std::remove_reference<decltype(*base)>::type T;
        const uint8_t* buffer = reinterpret_cast<const uint8_t*>(base);
        for (int m0 = 0; m0 < n; m0 += 1 << side) {
            const int m = m0 + (tid & ((1 << side) - 1));
            if (m >= n) continue;
            const int to = sh_to[m], at = sh_from[m];
            const int64_t dst = page(to), src = page(at);
            if (dst < 0 || src < 0) continue;
            // element `r` of a token: rows side by side for a token, or tokens side by side for a row
            const auto place = [&](int64_t id, int of, int r) {
                const int64_t in_page = by_token ? (((int64_t)kh << p) + (of & mask)) * rows + r : (((int64_t)kh * rows + r) << p) + (of & mask);
                return id * stride + in_page * (int64_t)sizeof(T);
            };
            const int step = 256 >> side;
            for (int r0 = tid >> side; r0 < rows; r0 += step * kBatch) {
                T x[kBatch];
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (r0 + b * step < rows) x[b] = *reinterpret_cast<const PATCH_EP_GLOBAL T*>(as_global(buffer) + place(src, at, r0 + b * step));
#pragma unroll
                for (int b = 0; b < kBatch; ++b)
                    if (r0 + b * step < rows) *reinterpret_cast<PATCH_EP_GLOBAL T*>(as_global_out(const_cast<uint8_t*>(buffer)) + place(dst, to, r0 + b * step)) = x[b];
            }
        }
    };
    if constexpr (CELL == 2) cells(reinterpret_cast<uint16_t*>(a.cache.v), a.cache.page_bytes, D, false);
    else cells(a.cache.v, a.cache.page_bytes, CELL == 0 ? D / 2 : D, false);
    if constexpr (CELL == 0) {
        cells(a.cache.k_power, a.cache.power_bytes, D / 32, true);
        cells(a.cache.v_power, a.cache.power_bytes, D / 32, false);
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
    for (int first = blockIdx.x / a.cache.kv_heads * 256; first < most; first += gridDim.x / a.cache.kv_heads * 256) {
        move_slots<CELL>(a, s, kh, first);
        __syncthreads();
    }
}

void launch_evict(const EvictArgs& a, hipStream_t stream) {
    const unsigned heads = (unsigned)a.cache.kv_heads, units = (unsigned)a.seqs.n_seqs * heads;
    if (a.seqs.max_kv <= 2 * kStrip) evict_select_kernel<2, true><<<units, kThreads, 0, stream>>>(a);
    else if (a.seqs.max_kv <= 4 * kStrip) evict_select_kernel<4, true><<<units, kThreads, 0, stream>>>(a);
    else evict_select_kernel<4, false><<<units, kThreads, 0, stream>>>(a);
    const unsigned chunks = (unsigned)std::min<int64_t>(((int64_t)std::min(a.keep, std::max(a.seqs.max_kv, 1)) + 255) / 256, std::max((1u << 22) / heads, 1u));
    // (V's rows over several workgroups, which then share lines of the cache: 4 prompts of up to 16000 tokens 75 us with one, 90 with two, 98 with four)
    const dim3 grid(chunks * heads, (unsigned)a.seqs.n_seqs);
    if (a.cache.cells == kBf16) evict_move_kernel<2><<<grid, 256, 0, stream>>>(a);
    else if (a.cache.cells == kE4m3) evict_move_kernel<1><<<grid, 256, 0, stream>>>(a);
    else evict_move_kernel<0><<<grid, 256, 0, stream>>>(a);
}

}  // namespace patch
