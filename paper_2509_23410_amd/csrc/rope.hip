// Norm and rotation of the heads of Q and K, and the append of K and V to a paged cache (patch_qk_rope, patch_kv_append).
//
//   y = x * rsqrt(mean(x^2) + eps) * gamma          per head, where gamma is given
//   (a, b) -> (a cos - b sin, a sin + b cos)        per pair, angles from the table's row of the token's position
//
// all in fp32, rounded once where a value is stored.  Some ten operations a value: the memory bounds it, and latency where there are few tokens.
#include "cells.h"

namespace patch {

// A head is D / 8 threads with two runs of four values each.  Rotated pairs are a run apart in halves (runs 4 j and rot / 2 + 4 j) and next to each
// other in an interleaved head (one run of eight), so that a thread has both values of its pairs, and the same four angles of the row, either way.
template <int D>
__global__ __launch_bounds__(256) void rope_kernel(const RopeArgs a) {
    constexpr int kThreads = D / 8;                    // of a head
    const int heads = a.q.heads + a.k.heads + a.v.heads;
    const int head = blockIdx.y * (256 / kThreads) + threadIdx.x / kThreads;
    const int64_t t = blockIdx.x;
    if (head >= heads) return;                          // whole heads: the shuffles below stay inside one
    const int j = threadIdx.x % kThreads;
    const int kind = head < a.q.heads ? 0 : head < a.q.heads + a.k.heads ? 1 : 2;
    const HeadArgs& h = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    const int at = kind == 0 ? head : kind == 1 ? head - a.q.heads : head - a.q.heads - a.k.heads;

    const bool turns = kind != 2 && j < a.rot / 8;
    int i0, i1;
    if (turns && !a.interleaved) {
        i0 = 4 * j;
        i1 = a.rot / 2 + 4 * j;
    } else {
        i0 = 8 * j;
        i1 = 8 * j + 4;
    }
    const uint8_t* row = h.x + t * h.stride + (int64_t)at * D * (a.f32 ? 4 : 2);
    Four x0 = load4(row, i0, a.f32), x1 = load4(row, i1, a.f32);

    // where the token stands: its position, and its cell in the cache
    int64_t pos;
    int page = -1;
    if (a.positions) {
        pos = as_global(a.positions)[t];
    } else {
        const int s = seq_of(a.seqs, (int)t);
        const Seq q = seq_at(a.seqs, s);
        const int i = (int)t - q.first;
        pos = !q.bad && i < q.n ? q.pos0 + i : -1;
        if (pos >= 0 && kind != 0) {
            page = page_or_none(as_global(a.seqs.table)[s * a.seqs.table_stride + (pos >> a.cache.page_log2)], a.cache.n_pages);
        }
    }
    const bool placed = pos >= 0;

    if (h.gamma) {
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += x0.x[e] * x0.x[e] + x1.x[e] * x1.x[e];
#pragma unroll
        for (int m = 1; m < kThreads; m <<= 1) sum += __shfl_xor(sum, m);
        const float r = rsqrtf(sum * (1.f / D) + a.eps);
        const Four g0 = load4(reinterpret_cast<const uint8_t*>(h.gamma), i0, 1), g1 = load4(reinterpret_cast<const uint8_t*>(h.gamma), i1, 1);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x0.x[e] = x0.x[e] * r * g0.x[e];
            x1.x[e] = x1.x[e] * r * g1.x[e];
        }
    }
    if (turns && placed) {
        Four c, s;
        if (pos < a.n_pos) {
            const uint8_t* angles = reinterpret_cast<const uint8_t*>(a.table + pos * a.rot);
            c = load4(angles, 4 * j, 1);
            s = load4(angles, a.rot / 2 + 4 * j, 1);
        } else {                                        // beyond the table: no angle, and to be seen in the result
#pragma unroll
            for (int e = 0; e < 4; ++e) c.x[e] = s.x[e] = __builtin_nanf("");
        }
        if (a.interleaved) {
            const Four y0 = x0, y1 = x1;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                x0.x[2 * e] = y0.x[2 * e] * c.x[e] - y0.x[2 * e + 1] * s.x[e];
                x0.x[2 * e + 1] = y0.x[2 * e] * s.x[e] + y0.x[2 * e + 1] * c.x[e];
                x1.x[2 * e] = y1.x[2 * e] * c.x[e + 2] - y1.x[2 * e + 1] * s.x[e + 2];
                x1.x[2 * e + 1] = y1.x[2 * e] * s.x[e + 2] + y1.x[2 * e + 1] * c.x[e + 2];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float y = x0.x[e];
                x0.x[e] = y * c.x[e] - x1.x[e] * s.x[e];
                x1.x[e] = y * s.x[e] + x1.x[e] * c.x[e];
            }
        }
    }

    if (kind == 0 || !a.cache.k) {                      // to a tensor; a token without a place is zero there
        if (!placed) x0 = x1 = Four{{0.f, 0.f, 0.f, 0.f}};
        uint8_t* out = h.out + t * h.out_stride + (int64_t)at * D * 2;
        *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(out) + 2 * i0) = pack_bf16(x0);
        *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(out) + 2 * i1) = pack_bf16(x1);
        return;
    }
    if (page < 0) return;
    const int slot = (int)pos & ((1 << a.cache.page_log2) - 1);
    const int64_t cells = (int64_t)at << (a.cache.page_log2);      // heads in front, in cells of D
    if (kind == 1) {
        uint8_t* base = a.cache.k + page * a.cache.page_bytes;
        if (a.cache.e4m3) {
            const float scale = a.cache.k_scale ? as_global(a.cache.k_scale)[at] : 1.f;
            base += (cells + slot) * D;
            *reinterpret_cast<PATCH_EP_GLOBAL uint32_t*>(as_global_out(base) + i0) = pack_e4m3(x0, scale);
            *reinterpret_cast<PATCH_EP_GLOBAL uint32_t*>(as_global_out(base) + i1) = pack_e4m3(x1, scale);
        } else {
            base += (cells + slot) * (2 * D);
            *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(base) + 2 * i0) = pack_bf16(x0);
            *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(base) + 2 * i1) = pack_bf16(x1);
        }
    } else {                                            // V: feature-major, the token's values are a page apart
        uint8_t* base = a.cache.v + page * a.cache.page_bytes;
        const int p = a.cache.page_log2;
        if (a.cache.e4m3) {
            const float scale = a.cache.v_scale ? as_global(a.cache.v_scale)[at] : 1.f;
            const uint32_t u0 = pack_e4m3(x0, scale), u1 = pack_e4m3(x1, scale);
            base += cells * D + slot;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                as_global_out(base)[(int64_t)(i0 + e) << p] = (uint8_t)(u0 >> (8 * e));
                as_global_out(base)[(int64_t)(i1 + e) << p] = (uint8_t)(u1 >> (8 * e));
            }
        } else {
            const u32x2_t u0 = pack_bf16(x0), u1 = pack_bf16(x1);
            PATCH_EP_GLOBAL uint16_t* o = reinterpret_cast<PATCH_EP_GLOBAL uint16_t*>(as_global_out(base)) + cells * D + slot;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                o[(int64_t)(i0 + e) << p] = (uint16_t)(u0[e / 2] >> (16 * (e % 2)));
                o[(int64_t)(i1 + e) << p] = (uint16_t)(u1[e / 2] >> (16 * (e % 2)));
            }
        }
    }
}

void launch_rope(const RopeArgs& a, hipStream_t stream) {
    const int heads = a.q.heads + a.k.heads + a.v.heads, each = 256 / (a.head_dim / 8);
    const dim3 grid((unsigned)a.n_tokens, (unsigned)((heads + each - 1) / each));
    if (a.head_dim == 64) rope_kernel<64><<<grid, 256, 0, stream>>>(a);
    else if (a.head_dim == 128) rope_kernel<128><<<grid, 256, 0, stream>>>(a);
    else rope_kernel<256><<<grid, 256, 0, stream>>>(a);
}

}  // namespace patch
