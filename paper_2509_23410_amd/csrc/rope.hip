// Norm and rotation of the heads of Q and K, and the append of K and V to a paged cache (patch_qk_rope, patch_kv_append).
//
//   y = x * rsqrt(mean(x^2) + eps) * gamma          per head, where gamma is given
//   (a, b) -> (a cos - b sin, a sin + b cos)        per pair, angles from the table's row of the token's position
//
// all in fp32, rounded once where a value is stored.  Some ten operations a value: the memory bounds it (4096 tokens of 32 + 8 heads of 128 in fp32 29.5 us,
// 4.3 TB/s), and latency where there are few tokens (64 tokens into their pages 4.6).
#include "cells.h"

namespace patch {

// V of a tile of 64 positions of one sequence and key head, turned in LDS: a feature's tokens side by side, as the page holds them.  By itself each value is a
// store of its own, a page's tokens apart: two prompts of 1100 tokens, 32 key heads of 128, e4m3, 70.3 us, in tiles 37.9 (and
// 33.1 with several heads a thread for Q and K).
template <int D>
__device__ __forceinline__ void append_v_tile(const RopeArgs& a, int tile, int kh, int s) {
    __shared__ uint16_t sh_v[D][kTurn + 2];                      // bf16, or e4m3 in the low byte; rows an odd number of words apart
    const Seq q = seq_at(a.seqs, s);
    const NewTile there = new_tile(q, tile);
    if (there.none) return;
    const int begin = there.begin, base = there.base;
    const float scale = a.cache.v_scale ? as_global(a.cache.v_scale)[kh] : 1.f;
    constexpr int kThreads = D / 4;
    const int d = (threadIdx.x % kThreads) * 4, i0 = threadIdx.x / kThreads;
    constexpr int kLoads = kTurn * kThreads / 256, kStep = 256 / kThreads;
    Four x[kLoads];
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {                           // all asked for together; a position that is not new has another's value, which is not stored
        const int64_t t = row_of_new(q, there, i0 + n * kStep);
        x[n] = load4(a.v.x + t * a.v.stride + (int64_t)kh * D * (a.f32 ? 4 : 2), d, a.f32);
    }
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
        const int i = i0 + n * kStep;
        if (a.cache.e4m3) {
            const uint32_t u = pack_e4m3(x[n], scale);
#pragma unroll
            for (int e = 0; e < 4; ++e) sh_v[d + e][i] = (u >> (8 * e)) & 0xFFu;
        } else {
            const u32x2_t u = pack_bf16(x[n]);
#pragma unroll
            for (int e = 0; e < 4; ++e) sh_v[d + e][i] = (uint16_t)(u[e / 2] >> (16 * (e % 2)));
        }
    }
    // eight positions of a feature at a time: they are in one page, and side by side there
    const int c = (threadIdx.x % (kTurn / 8)) * 8, pos = base + c;
    int page = -1;
    if (pos + 8 > begin && pos < q.len) page = page_or_none(as_global(a.seqs.table)[s * a.seqs.table_stride + (pos >> a.cache.page_log2)], a.cache.n_pages);
    __syncthreads();
    if (page < 0) return;
    const bool whole = pos >= begin && pos + 8 <= q.len;
    uint8_t* to = a.cache.v + page * a.cache.page_bytes;
    const int64_t slot = ((int64_t)kh * D << a.cache.page_log2) + (pos & ((1 << a.cache.page_log2) - 1));
#pragma unroll 4
    for (int f = threadIdx.x / (kTurn / 8); f < D; f += 256 / (kTurn / 8)) {
        const int64_t cell = slot + ((int64_t)f << a.cache.page_log2);
        if (a.cache.e4m3) {
            if (whole) {
                u32x2_t w;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    w[e] = sh_v[f][c + 4 * e] | (uint32_t)sh_v[f][c + 4 * e + 1] << 8 | (uint32_t)sh_v[f][c + 4 * e + 2] << 16 | (uint32_t)sh_v[f][c + 4 * e + 3] << 24;
                *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(to) + cell) = w;
            } else {
                for (int e = 0; e < 8; ++e)
                    if (pos + e >= begin && pos + e < q.len) as_global_out(to)[cell + e] = (uint8_t)sh_v[f][c + e];
            }
        } else if (whole) {
            u32x4_t w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = sh_v[f][c + 2 * e] | (uint32_t)sh_v[f][c + 2 * e + 1] << 16;
            *reinterpret_cast<PATCH_EP_GLOBAL u32x4_t*>(as_global_out(to) + 2 * cell) = w;
        } else {
            for (int e = 0; e < 8; ++e)
                if (pos + e >= begin && pos + e < q.len) reinterpret_cast<PATCH_EP_GLOBAL uint16_t*>(as_global_out(to))[cell + e] = sh_v[f][c + e];
        }
    }
}

// A head is D / 8 threads with two runs of four values each.  Rotated pairs are a run apart in halves (runs 4 j and rot / 2 + 4 j) and next to each
// other in an interleaved head (one run of eight), so that a thread has both values of its pairs, and the same four angles of the row, either way.
// A thread has the same places of U heads of a token, all of them asked for together, and one set of angles for them.
template <int D, int U>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a) {
    constexpr int kThreads = D / 8, kHeads = 256 / kThreads;    // threads of a head, heads at a time
    // workgroups behind those of the heads have tiles of V (v_tiles of every sequence and key head), numbered along x, then y
    const int heads = a.q.heads + a.k.heads + (a.v_tiles ? 0 : a.v.heads), rows_y = (heads + U * kHeads - 1) / (U * kHeads);
    if ((int)blockIdx.y >= rows_y) {
        const int64_t i = (int64_t)(blockIdx.y - rows_y) * gridDim.x + blockIdx.x;
        const int s = (int)(i / a.v_tiles / a.v.heads);
        if (s < a.seqs.n_seqs) append_v_tile<D>(a, (int)(i % a.v_tiles), (int)(i / a.v_tiles % a.v.heads), s);
        return;
    }
    const int first = blockIdx.y * (U * kHeads) + threadIdx.x / kThreads, j = threadIdx.x % kThreads;
    const int64_t t = blockIdx.x;
    const bool rotated = j < a.rot / 8;
    int kind[U], at[U];                                          // 0: Q, 1: K, 2: V, and which head; -1: none (whole heads: shuffles stay inside one)
    Four x0[U], x1[U];
    const auto place = [&](int u, int* i0, int* i1) {
        const bool apart = rotated && kind[u] != 2 && !a.interleaved;
        *i0 = apart ? 4 * j : 8 * j;
        *i1 = apart ? a.rot / 2 + 4 * j : 8 * j + 4;
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int head = first + u * kHeads;
        kind[u] = head < a.q.heads ? 0 : head < a.q.heads + a.k.heads ? 1 : head < heads ? 2 : -1;
        at[u] = kind[u] == 0 ? head : kind[u] == 1 ? head - a.q.heads : head - a.q.heads - a.k.heads;
        int i0, i1;
        place(u, &i0, &i1);
        if (kind[u] >= 0) {
            const uint8_t* x = kind[u] == 0 ? a.q.x : kind[u] == 1 ? a.k.x : a.v.x;
            const int64_t stride = kind[u] == 0 ? a.q.stride : kind[u] == 1 ? a.k.stride : a.v.stride;
            x += t * stride + (int64_t)at[u] * D * (a.f32 ? 4 : 2);
            x0[u] = load4(x, i0, a.f32);
            x1[u] = load4(x, i1, a.f32);
        } else {
            x0[u] = x1[u] = Four{{0.f, 0.f, 0.f, 0.f}};
        }
    }

    // where the token stands: its position, and its cell in the cache
    int64_t pos;
    int page = -1;
    if (a.positions) {
        pos = as_global(a.positions)[t];
    } else {
        const int s = seq_of(a.seqs, (int)t);
        const Seq q = seq_at(a.seqs, s);
        const int i = place_of(q, (int)t);
        pos = !q.bad && i >= 0 ? q.pos0 + i : -1;
        if (pos >= 0) page = page_or_none(as_global(a.seqs.table)[s * a.seqs.table_stride + (pos >> a.cache.page_log2)], a.cache.n_pages);
    }
    const bool placed = pos >= 0;
    Four c = {{1.f, 1.f, 1.f, 1.f}}, s = {{0.f, 0.f, 0.f, 0.f}};
    if (rotated && placed) {
        if (pos < a.n_pos) {
            const uint8_t* angles = reinterpret_cast<const uint8_t*>(a.table + pos * a.rot);
            c = load4(angles, 4 * j, 1);
            s = load4(angles, a.rot / 2 + 4 * j, 1);
        } else {                                                 // beyond the table: no angle, and to be seen in the result
#pragma unroll
            for (int e = 0; e < 4; ++e) c.x[e] = s.x[e] = __builtin_nanf("");
        }
    }

#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (kind[u] < 0) continue;
        int i0, i1;
        place(u, &i0, &i1);
        Four y0 = x0[u], y1 = x1[u];
        const float* gamma = kind[u] == 0 ? a.q.gamma : kind[u] == 1 ? a.k.gamma : nullptr;
        if (gamma) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += y0.x[e] * y0.x[e] + y1.x[e] * y1.x[e];
#pragma unroll
            for (int m = 1; m < kThreads; m <<= 1) sum += __shfl_xor(sum, m);
            const float r = rsqrtf(sum * (1.f / D) + a.eps);
            const Four g0 = load4(reinterpret_cast<const uint8_t*>(gamma), i0, 1), g1 = load4(reinterpret_cast<const uint8_t*>(gamma), i1, 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y0.x[e] = y0.x[e] * r * g0.x[e];
                y1.x[e] = y1.x[e] * r * g1.x[e];
            }
        }
        if (rotated && placed && kind[u] != 2) {
            const Four z0 = y0, z1 = y1;
            if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    y0.x[2 * e] = z0.x[2 * e] * c.x[e] - z0.x[2 * e + 1] * s.x[e];
                    y0.x[2 * e + 1] = z0.x[2 * e] * s.x[e] + z0.x[2 * e + 1] * c.x[e];
                    y1.x[2 * e] = z1.x[2 * e] * c.x[e + 2] - z1.x[2 * e + 1] * s.x[e + 2];
                    y1.x[2 * e + 1] = z1.x[2 * e] * s.x[e + 2] + z1.x[2 * e + 1] * c.x[e + 2];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    y0.x[e] = z0.x[e] * c.x[e] - z1.x[e] * s.x[e];
                    y1.x[e] = z0.x[e] * s.x[e] + z1.x[e] * c.x[e];
                }
            }
        }

        if (kind[u] == 0 || !a.cache.k) {                        // to a tensor; a token without a place is zero there
            if (!placed) y0 = y1 = Four{{0.f, 0.f, 0.f, 0.f}};
            uint8_t* out = (kind[u] == 0 ? a.q.out + t * a.q.out_stride : a.k.out + t * a.k.out_stride) + (int64_t)at[u] * D * 2;
            *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(out) + 2 * i0) = pack_bf16(y0);
            *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(out) + 2 * i1) = pack_bf16(y1);
            continue;
        }
        if (page < 0) continue;
        const int slot = (int)pos & ((1 << a.cache.page_log2) - 1);
        const int64_t cells = (int64_t)at[u] << a.cache.page_log2;       // those of the heads in front, over D
        if (kind[u] == 1) {
            uint8_t* base = a.cache.k + page * a.cache.page_bytes;
            if (a.cache.e4m3) {
                const float scale = a.cache.k_scale ? as_global(a.cache.k_scale)[at[u]] : 1.f;
                base += (cells + slot) * D;
                *reinterpret_cast<PATCH_EP_GLOBAL uint32_t*>(as_global_out(base) + i0) = pack_e4m3(y0, scale);
                *reinterpret_cast<PATCH_EP_GLOBAL uint32_t*>(as_global_out(base) + i1) = pack_e4m3(y1, scale);
            } else {
                base += (cells + slot) * (2 * D);
                *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(base) + 2 * i0) = pack_bf16(y0);
                *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(base) + 2 * i1) = pack_bf16(y1);
            }
        } else {                                                 // V: feature-major, the token's values are a page apart
            uint8_t* base = a.cache.v + page * a.cache.page_bytes;
            const int p = a.cache.page_log2;
            if (a.cache.e4m3) {
                const float scale = a.cache.v_scale ? as_global(a.cache.v_scale)[at[u]] : 1.f;
                const uint32_t u0 = pack_e4m3(y0, scale), u1 = pack_e4m3(y1, scale);
                base += cells * D + slot;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    as_global_out(base)[(int64_t)(i0 + e) << p] = (uint8_t)(u0 >> (8 * e));
                    as_global_out(base)[(int64_t)(i1 + e) << p] = (uint8_t)(u1 >> (8 * e));
                }
            } else {
                const u32x2_t u0 = pack_bf16(y0), u1 = pack_bf16(y1);
                PATCH_EP_GLOBAL uint16_t* o = reinterpret_cast<PATCH_EP_GLOBAL uint16_t*>(as_global_out(base)) + cells * D + slot;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[(int64_t)(i0 + e) << p] = (uint16_t)(u0[e / 2] >> (16 * (e % 2)));
                    o[(int64_t)(i1 + e) << p] = (uint16_t)(u1[e / 2] >> (16 * (e % 2)));
                }
            }
        }
    }
}

template <int U>
static void launch_rope_of(const RopeArgs& a, hipStream_t stream) {
    const int heads = a.q.heads + a.k.heads + (a.v_tiles ? 0 : a.v.heads), each = U * 256 / (a.head_dim / 8);
    const int64_t more = a.v_tiles ? ((int64_t)a.seqs.n_seqs * a.v_tiles * a.v.heads + a.n_tokens - 1) / a.n_tokens : 0;      // at most v.heads
    const dim3 grid((unsigned)a.n_tokens, (unsigned)((heads + each - 1) / each + more));
    if (a.head_dim == 64) rope_kernel<64, U><<<grid, 256, 0, stream>>>(a);
    else if (a.head_dim == 128) rope_kernel<128, U><<<grid, 256, 0, stream>>>(a);
    else rope_kernel<256, U><<<grid, 256, 0, stream>>>(a);
}

void launch_rope(const RopeArgs& in, hipStream_t stream) {
    RopeArgs a = in;
    // Tiles of V where sequences bring runs of tokens, enough of them to fill the chip, and not so ragged ones that most tiles would be empty: 32 sequences of 8
    // tokens, 8 key heads of 128, 8.7 us by itself and 7.0 in tiles, 64 of 16 17.3 and 14.4, but 64 of one 6.5 and 6.8, and one of 50 (a head of 256) 6.0 and 8.2.
    const int64_t tiles = ((int64_t)a.seqs.max_q + 2 * kTurn - 2) / kTurn;
    a.v_tiles = a.cache.k && a.seqs.max_q >= 8 && a.n_tokens >= 256 && a.seqs.n_seqs * tiles <= a.n_tokens ? (int)tiles : 0;
    const int heads = a.q.heads + a.k.heads + (a.v_tiles ? 0 : a.v.heads), each = 256 / (a.head_dim / 8);
    // Four heads a thread where a token has enough of them and the workgroups fill the chip all the same: 4096 tokens, 32 + 8 + 8 heads of 128, appended in bf16
    // 40.8 -> 35.6 us; 4000 tokens of 14 + 2 + 2 heads of 64 would go from 10.5 to 12.5.
    if (heads > 2 * each && a.n_tokens >= 1024) launch_rope_of<4>(a, stream);
    else launch_rope_of<1>(a, stream);
}

}  // namespace patch
