// The append of K and V to a paged cache of 4-bit cells (patch_kv_append4), K normed and rotated first, and Q with it.
//
//   y = x * rsqrt(mean(x^2) + eps) * gamma,  (a, b) -> (a cos - b sin, a sin + b cos)         as patch_kv_append, in fp32
//   power = the smallest 2^k with max |y| <= 7 2^k over 32 features,  cell = y / power to the nearest of 0 .5 1 1.5 2 3 4 6
//
// A head is D / 8 threads with eight features each, so that 32 features are four neighbours and a thread's cells are one word of K.  Where halves of a head are
// rotated against each other a thread loads its features' partners too (they are in the cache, another thread has them as its own) and turns only its own.
//
// Rows may be written where they are read (out is x).  A head's threads are in one wavefront, and each stores what it computed from all of their loads.  A tile of V reads
// rows of its own positions only; what it reads for a position that is not new may have been written already, and goes nowhere.  Rows without a place, which the threads of K's
// heads clear, are in no tile.
#include "cells4.h"

namespace patch {

struct Eight { Four lo, hi; };

__device__ __forceinline__ float largest(const Eight& v) {
    float top = 0.f;
    bool odd = false;                                            // maxima pass NaN over
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        top = fmaxf(top, fmaxf(fabsf(v.lo.x[e]), fabsf(v.hi.x[e])));
        odd |= v.lo.x[e] != v.lo.x[e] || v.hi.x[e] != v.hi.x[e];
    }
    return odd ? __builtin_inff() : top;
}
// The byte of the power that this thread's eight features have with those of its three neighbours.
__device__ __forceinline__ uint32_t shared_power(const Eight& v) {
    float top = largest(v);
    top = fmaxf(top, __shfl_xor(top, 1));
    top = fmaxf(top, __shfl_xor(top, 2));
    return power_byte(top);
}
__device__ __forceinline__ uint32_t stored(const Eight& v, uint32_t byte) { return byte == 255u ? 0u : pack8_e2m1(v.lo, v.hi, power_of(byte)); }
// what the cells stand for, to a row of bf16
__device__ __forceinline__ void show(uint8_t* row, int d, uint32_t cells, uint32_t byte, bool placed) {
    u32x4_t w = widen8_e2m1(cells, power_of(byte));
    if (!placed) w = u32x4_t{0, 0, 0, 0};
    *reinterpret_cast<PATCH_EP_GLOBAL u32x4_t*>(as_global_out(row) + 2 * d) = w;
}

// V of a tile of 64 positions of one sequence and key head, turned in LDS: a pair of features' tokens side by side, as the page holds them.
template <int D>
__device__ __forceinline__ void append_v4_tile(const RopeArgs& a, int tile, int kh, int s) {
    __shared__ alignas(16) uint8_t sh_v[D / 2][kTurn + 16], sh_p[D / 32][kTurn];            // rows of whole 16 bytes
    const Seq q = seq_at(a.seqs, s);
    const NewTile there = new_tile(q, tile);
    if (there.none) return;
    constexpr int kThreads = D / 8, kStep = 256 / kThreads, kLoads = kTurn / kStep;
    const int j = threadIdx.x % kThreads, i0 = threadIdx.x / kThreads;
    Eight x[kLoads];
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {                           // all asked for together; a position that is not new has another's value, which is not stored
        const int64_t t = row_of_new(q, there, i0 + n * kStep);
        const uint8_t* row = a.v.x + t * a.v.stride + (int64_t)kh * D * (a.f32 ? 4 : 2);
        x[n] = Eight{load4(row, 8 * j, a.f32), load4(row, 8 * j + 4, a.f32)};
    }
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
        const int i = i0 + n * kStep;
        const uint32_t byte = shared_power(x[n]), u = stored(x[n], byte);
#pragma unroll
        for (int e = 0; e < 4; ++e) sh_v[4 * j + e][i] = (uint8_t)(u >> (8 * e));
        if (j % 4 == 0) sh_p[j / 4][i] = (uint8_t)byte;
        const int pos = there.base + i;
        if (a.v.out && pos >= there.begin && pos < q.len) show(a.v.out + (int64_t)row_of_new(q, there, i) * a.v.out_stride + (int64_t)kh * D * 2, 8 * j, u, byte, true);
    }
    // sixteen positions of a row at a time: they are in one page, and side by side there
    const int c = (threadIdx.x % (kTurn / 16)) * 16, pos = there.base + c;
    int page = -1;
    if (pos + 16 > there.begin && pos < q.len) page = page_or_none(as_global(a.seqs.table)[s * a.seqs.table_stride + (pos >> a.cache.page_log2)], a.cache.n_pages);
    __syncthreads();
    if (page < 0) return;
    const bool whole = pos >= there.begin && pos + 16 <= q.len;
    const int slot = pos & ((1 << a.cache.page_log2) - 1);
    const auto put = [&](uint8_t* to, const uint8_t* from) {
        if (whole) *reinterpret_cast<PATCH_EP_GLOBAL u32x4_t*>(as_global_out(to)) = *reinterpret_cast<const u32x4_t*>(from);
        else
            for (int e = 0; e < 16; ++e)
                if (pos + e >= there.begin && pos + e < q.len) as_global_out(to)[e] = from[e];
    };
#pragma unroll 1
    for (int r = threadIdx.x / (kTurn / 16); r < D / 2 + D / 32; r += 256 / (kTurn / 16)) {
        if (r < D / 2) put(a.cache.v + page * a.cache.page_bytes + (((int64_t)kh * (D / 2) + r) << a.cache.page_log2) + slot, &sh_v[r][c]);
        else put(a.cache.v_power + page * a.cache.power_bytes + (((int64_t)kh * (D / 32) + r - D / 2) << a.cache.page_log2) + slot, &sh_p[r - D / 2][c]);
    }
}

template <int D>
__global__ __launch_bounds__(256) void append4_kernel(const RopeArgs a) {
    constexpr int kThreads = D / 8, kHeads = 256 / kThreads;    // threads of a head, heads at a time
    // workgroups behind those of the heads have tiles of V (v_tiles of every sequence and key head), numbered along x, then y
    const int heads = a.q.heads + a.k.heads + (a.v_tiles ? 0 : a.v.heads), rows_y = (heads + kHeads - 1) / kHeads;
    if ((int)blockIdx.y >= rows_y) {
        const int64_t i = (int64_t)(blockIdx.y - rows_y) * gridDim.x + blockIdx.x;
        const int s = (int)(i / a.v_tiles / a.v.heads);
        if (s < a.seqs.n_seqs) append_v4_tile<D>(a, (int)(i % a.v_tiles), (int)(i / a.v_tiles % a.v.heads), s);
        return;
    }
    const int head = blockIdx.y * kHeads + threadIdx.x / kThreads, j = threadIdx.x % kThreads;
    if (head >= heads) return;                                   // whole heads: shuffles stay inside one
    const int64_t t = blockIdx.x;
    const int kind = head < a.q.heads ? 0 : head < a.q.heads + a.k.heads ? 1 : 2;
    const int at = kind == 0 ? head : kind == 1 ? head - a.q.heads : head - a.q.heads - a.k.heads;
    const HeadArgs& h = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    const uint8_t* row = h.x + t * h.stride + (int64_t)at * D * (a.f32 ? 4 : 2);
    const bool rotated = kind != 2 && 8 * j < a.rot;
    Eight y = {load4(row, 8 * j, a.f32), load4(row, 8 * j + 4, a.f32)}, other = y;
    // the partners of each run of four (rot / 2 is a multiple of four)
    const int half = a.rot / 2;
    const auto partner = [&](int i) { return i < half ? i + half : i - half; };
    if (rotated && !a.interleaved) other = Eight{load4(row, partner(8 * j), a.f32), load4(row, partner(8 * j + 4), a.f32)};

    const int s = seq_of(a.seqs, (int)t);
    const Seq q = seq_at(a.seqs, s);
    const int i = place_of(q, (int)t);
    const int64_t pos = !q.bad && i >= 0 ? q.pos0 + i : -1;
    const bool placed = pos >= 0;
    int page = -1;
    if (placed) page = page_or_none(as_global(a.seqs.table)[s * a.seqs.table_stride + (pos >> a.cache.page_log2)], a.cache.n_pages);

    const float* gamma = h.gamma;
    if (gamma) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += y.lo.x[e] * y.lo.x[e] + y.hi.x[e] * y.hi.x[e];
#pragma unroll
        for (int m = 1; m < kThreads; m <<= 1) sum += __shfl_xor(sum, m);
        const float r = rsqrtf(sum * (1.f / D) + a.eps);
        const auto scaled = [&](Four& x, int first) {
            const Four g = load4(reinterpret_cast<const uint8_t*>(gamma), first, 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) x.x[e] = x.x[e] * r * g.x[e];
        };
        scaled(y.lo, 8 * j);
        scaled(y.hi, 8 * j + 4);
        if (rotated && !a.interleaved) {
            scaled(other.lo, partner(8 * j));
            scaled(other.hi, partner(8 * j + 4));
        }
    }
    if (rotated && placed) {
        const int64_t angle = a.positions ? as_global(a.positions)[t] : pos;
        const bool known = angle >= 0 && angle < a.n_pos;        // beyond the table: no angle, and to be seen in the result
        const uint8_t* angles = reinterpret_cast<const uint8_t*>(a.table + (known ? angle : 0) * a.rot);
        const auto turn = [&](Four& x, const Four& z, int first) {
            const bool front = first < half;
            const Four c = load4(angles, front ? first : first - half, 1), sn = load4(angles, half + (front ? first : first - half), 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float turned = front ? x.x[e] * c.x[e] - z.x[e] * sn.x[e] : z.x[e] * sn.x[e] + x.x[e] * c.x[e];
                x.x[e] = known ? turned : __builtin_nanf("");
            }
        };
        if (a.interleaved) {                                     // four pairs, next to each other
            const Four c = load4(angles, 4 * j, 1), sn = load4(angles, half + 4 * j, 1);
            const auto pairs = [&](Four& x, int first) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float u = x.x[2 * e], w = x.x[2 * e + 1];
                    x.x[2 * e] = known ? u * c.x[first + e] - w * sn.x[first + e] : __builtin_nanf("");
                    x.x[2 * e + 1] = known ? u * sn.x[first + e] + w * c.x[first + e] : __builtin_nanf("");
                }
            };
            pairs(y.lo, 0);
            pairs(y.hi, 2);
        } else {
            turn(y.lo, other.lo, 8 * j);
            turn(y.hi, other.hi, 8 * j + 4);
        }
    }

    if (kind == 0) {                                             // to a tensor; a token without a place is zero there
        u32x2_t lo = pack_bf16(y.lo), hi = pack_bf16(y.hi);
        u32x4_t w = {lo[0], lo[1], hi[0], hi[1]};
        if (!placed) w = u32x4_t{0, 0, 0, 0};
        *reinterpret_cast<PATCH_EP_GLOBAL u32x4_t*>(as_global_out(a.q.out) + t * a.q.out_stride + ((int64_t)at * D + 8 * j) * 2) = w;
        return;
    }
    // the tiles of V are of positions: they leave out rows that have none
    if (kind == 1 && a.v_tiles && a.v.out && !placed)
        *reinterpret_cast<PATCH_EP_GLOBAL u32x4_t*>(as_global_out(a.v.out) + t * a.v.out_stride + ((int64_t)at * D + 8 * j) * 2) = u32x4_t{0, 0, 0, 0};
    const uint32_t byte = shared_power(y), cells = stored(y, byte);
    if (h.out) show(h.out + t * h.out_stride + (int64_t)at * D * 2, 8 * j, cells, byte, placed);
    if (page < 0) return;
    const int p = a.cache.page_log2, slot = (int)pos & ((1 << p) - 1);
    if (kind == 1) {
        const int64_t token = ((int64_t)at << p) + slot;
        *reinterpret_cast<PATCH_EP_GLOBAL uint32_t*>(as_global_out(a.cache.k) + page * a.cache.page_bytes + token * (D / 2) + 4 * j) = cells;
        if (j % 4 == 0) as_global_out(a.cache.k_power)[page * a.cache.power_bytes + token * (D / 32) + j / 4] = (uint8_t)byte;
    } else {                                                     // V: pairs of features, the token's are a page apart
        PATCH_EP_GLOBAL uint8_t* to = as_global_out(a.cache.v) + page * a.cache.page_bytes + (((int64_t)at * (D / 2) + 4 * j) << p) + slot;
#pragma unroll
        for (int e = 0; e < 4; ++e) to[(int64_t)e << p] = (uint8_t)(cells >> (8 * e));
        if (j % 4 == 0) as_global_out(a.cache.v_power)[page * a.cache.power_bytes + (((int64_t)at * (D / 32) + j / 4) << p) + slot] = (uint8_t)byte;
    }
}

void launch_append4(const RopeArgs& in, hipStream_t stream) {
    RopeArgs a = in;
    // Tiles of V where sequences bring runs of tokens, enough of them to fill the chip, and not so ragged ones that most tiles would be empty, as in the append of
    // wider cells.
    const int64_t tiles = ((int64_t)a.seqs.max_q + 2 * kTurn - 2) / kTurn;
    a.v_tiles = a.seqs.max_q >= 8 && a.n_tokens >= 256 && a.seqs.n_seqs * tiles <= a.n_tokens ? (int)tiles : 0;
    const int heads = a.q.heads + a.k.heads + (a.v_tiles ? 0 : a.v.heads), each = 256 / (a.head_dim / 8);
    const int64_t more = a.v_tiles ? ((int64_t)a.seqs.n_seqs * a.v_tiles * a.v.heads + a.n_tokens - 1) / a.n_tokens : 0;      // at most v.heads
    const dim3 grid((unsigned)a.n_tokens, (unsigned)((heads + each - 1) / each + more));
    if (a.head_dim == 64) append4_kernel<64><<<grid, 256, 0, stream>>>(a);
    else if (a.head_dim == 128) append4_kernel<128><<<grid, 256, 0, stream>>>(a);
    else append4_kernel<256><<<grid, 256, 0, stream>>>(a);
}

}  // namespace patch
