// Causal attention of a batch's new tokens over a paged cache (patch_attention).
//
//   o_r = sum_j p_rj v_j / sum_j p_rj,   p_rj = exp(q_r . k_j scale - m_r),   over the keys j <= position of row r,
//
// in one pass over the keys: m_r is the running maximum; where it rises, what was summed so far is scaled down by exp(old - new).  Scores, maxima and
// sums are fp32; p is rounded to bf16 as an operand of the second product (its sum is taken before that), which puts 2^-9 of each p into o at most.
//
// A key head's rows are (token, query head of its group) side by side, so that a group shares every K and V that is read.  Both products have the
// keys' side as the matrix instruction's A operand: S^T = K Q^T and O^T = V^T P^T.  A column is then a row of the attention, one column per lane in
// both, and the second product's B operand is what the lane already holds of the first's result, if the keys of a step are given out to the rows of A
// in the right order: no value of P crosses lanes.  V lies feature-major in its pages, so V^T's operand is a plain 16-byte load too.
#include <algorithm>

#include "cells.h"

namespace patch {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4_t v) { return *reinterpret_cast<bf16x8_t*>(&v); }

// eight e4m3 cells as bf16 (every one of them is exact there)
__device__ __forceinline__ u32x4_t widen8(uint32_t lo, uint32_t hi) {
    const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.f, true);
    const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.f, true);
    return u32x4_t{*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b), *reinterpret_cast<const uint32_t*>(&c), *reinterpret_cast<const uint32_t*>(&d)};
}

constexpr float kNone = -__builtin_inff();
// The maximum that scores are held against follows the true one only where that is more than this above it (in powers of two): a p is then at most 2^8, which
// costs neither bf16's relative step nor the fp32 sums anything, and after a row's first keys the sums hardly ever have to be scaled down.
constexpr float kRise = 8.f;
// exp2(x - m) where m may be the maximum of nothing
__device__ __forceinline__ float exp2_off(float x, float m) { return __builtin_amdgcn_exp2f(x - (m == kNone ? 0.f : m)); }

// Which rows and keys a workgroup has.  The shared front is one batch of all tokens against the first sequence's pages.
struct Span {
    int t0, rows;        // first token, rows (tokens times group)
    int pos0;            // position of token t0; in the shared front each row looks up its own
    int key0, key1;      // keys [key0, key1) are there to be read
    int begin, end;      // and those this workgroup takes, begin a multiple of 32
    int part;            // its partial result, -1: it writes the result itself
    int64_t table;       // its row of the page table
    bool front, bad;
};

__device__ __forceinline__ Span front_span(const AttnArgs& a, int part) {
    Span p;
    p.front = true;
    p.t0 = 0;
    p.rows = a.seqs.n_tokens * a.group;
    p.pos0 = 0;
    p.key0 = 0;
    p.key1 = a.prefix;
    p.begin = part * a.prefix_chunk;
    p.end = min(a.prefix, p.begin + a.prefix_chunk);
    p.part = part;
    p.table = 0;
    p.bad = false;
    return p;
}

__device__ __forceinline__ int own_parts(const AttnArgs& a, int len) {
    const int base = a.prefix & ~31;
    return len > a.prefix ? (len - base + a.own_chunk - 1) / a.own_chunk : 0;
}

__device__ __forceinline__ Span own_span(const AttnArgs& a, int s, int chunk) {
    const Seq q = seq_at(a.seqs, s);
    Span p;
    p.front = false;
    p.t0 = q.first;
    p.rows = q.n * a.group;
    p.pos0 = q.pos0;
    p.key0 = a.prefix;
    p.key1 = max(q.len, a.prefix);
    p.begin = (a.prefix & ~31) + chunk * a.own_chunk;
    p.end = min(q.len, p.begin + a.own_chunk);
    p.part = a.parts == 1 || (a.prefix_parts == 0 && q.len - p.begin <= a.own_chunk && chunk == 0) ? -1 : a.prefix_parts + chunk;
    p.table = s * a.seqs.table_stride;
    p.bad = q.bad;
    return p;
}

// Keys [0, result) are those that row r (of a span, not counted from a workgroup's first) sees, if it has any of the span's.
__device__ __forceinline__ int row_limit(const AttnArgs& a, const Span& p, int r) {
    if (r >= p.rows) return 0;
    const int t = p.t0 + r / a.group;
    if (!p.front) return p.pos0 + r / a.group + 1;
    const Seq q = seq_at(a.seqs, seq_of(a.seqs, t));
    return t - q.first < q.n ? min(a.prefix, q.pos0 + t - q.first + 1) : 0;
}

// Of a lane's eight keys from `key` on, zero where they are not in [lo, hi).
__device__ __forceinline__ void keep_keys(u32x4_t& v, int key, int lo, int hi) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (key + e < lo || key + e >= hi) v[e / 2] &= e % 2 ? 0x0000FFFFu : 0xFFFF0000u;
}
__device__ __forceinline__ bool any_infinite(const u32x4_t& v) {      // or NaN
    bool any = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) any |= (v[e] & 0x7F80u) == 0x7F80u || (v[e] & 0x7F800000u) == 0x7F800000u;
    return any;
}

// Few rows: each wavefront takes steps of 32 keys of its own, K and V straight from memory into the operands' registers, RB blocks of 16 rows against
// them; the four wavefronts' results meet in LDS.
constexpr int kTableKeys = 4096;   // page numbers of so many keys are in LDS at a time

template <int D, bool E4M3>
struct KeyRegs {
    u32x4_t k[2][E4M3 ? D / 64 : D / 32];
    u32x4_t v[E4M3 ? D / 32 : D / 16];
};

template <int D, bool E4M3>
__device__ __forceinline__ void load_keys(KeyRegs<D, E4M3>& r, const AttnArgs& a, const int* pages, int step, int kh, int lane) {
    constexpr int kCell = E4M3 ? 1 : 2;
    const int g = lane >> 4, row = lane & 15, mask = (1 << a.cache.page_log2) - 1;
    // row i of A's tile b is key 8 (i / 4) + 4 b + i % 4: a lane then holds, of both tiles, the keys 8 g .. 8 g + 7 of its column
    const int key = 8 * (row >> 2) + (row & 3);
    {
        const int at = step + key;
        const int page = max(pages[at >> a.cache.page_log2], 0);
        const PATCH_EP_GLOBAL uint8_t* base = as_global(a.cache.k) + page * a.cache.page_bytes + (((int64_t)kh << a.cache.page_log2) + (at & mask)) * (D * kCell) + 16 * g;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < (E4M3 ? D / 64 : D / 32); ++i)
                r.k[b][i] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(base + b * (4 * D * kCell) + 64 * i);
    }
    {
        const int at = step + 8 * g;
        const int page = max(pages[at >> a.cache.page_log2], 0);
        const PATCH_EP_GLOBAL uint8_t* base = as_global(a.cache.v) + page * a.cache.page_bytes + ((((int64_t)kh * D + row) << a.cache.page_log2) + (at & mask)) * kCell;
        const int64_t next = (int64_t)(16 * kCell) << a.cache.page_log2;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            if constexpr (E4M3) {
                const u32x2_t v = *reinterpret_cast<const PATCH_EP_GLOBAL u32x2_t*>(base + i * next);
                r.v[i / 2][2 * (i % 2)] = v[0];
                r.v[i / 2][2 * (i % 2) + 1] = v[1];
            } else {
                r.v[i] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(base + i * next);
            }
        }
    }
}

// the operand of 32 of a head's values (i counts them) for keys of tile b; in e4m3 a 16-byte load is the operands of two products, and Q's follow it
template <int D, bool E4M3>
__device__ __forceinline__ bf16x8_t key_operand(const KeyRegs<D, E4M3>& r, int b, int i) {
    if constexpr (E4M3) return as_bf16x8(widen8(r.k[b][i / 2][2 * (i % 2)], r.k[b][i / 2][2 * (i % 2) + 1]));
    else return as_bf16x8(r.k[b][i]);
}
template <bool E4M3>
__device__ __forceinline__ int query_offset(int i, int g) { return E4M3 ? 64 * (i / 2) + 16 * g + 8 * (i % 2) : 32 * i + 8 * g; }

template <int D, int RB, bool E4M3>
__global__ __launch_bounds__(256, D * RB <= 128 ? 2 : 1) void attend_rows_kernel(const AttnArgs a, const int front) {
    constexpr int kPitch = D + 4;
    __shared__ float sh_o[4][16][kPitch];
    __shared__ float sh_m[4][RB * 16], sh_l[4][RB * 16];
    __shared__ int sh_pages[kTableKeys / 16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    const int kh = blockIdx.y, groups = ((front ? a.seqs.n_tokens : a.seqs.max_q) * a.group + 16 * RB - 1) / (16 * RB);
    const int first_row = (blockIdx.x % groups) * (16 * RB), chunk = blockIdx.x / groups;
    const Span p = front ? front_span(a, chunk) : own_span(a, blockIdx.z, chunk);
    if (first_row >= p.rows) return;
    if (p.begin >= p.end && (p.part >= 0 || chunk > 0)) return;     // no keys here; the first workgroup of rows that see none writes that

    int limit[RB], fewest = 0x7FFFFFFF, most = 0;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = first_row + 16 * b + col;
        limit[b] = row_limit(a, p, r);
        if (r < p.rows) fewest = min(fewest, limit[b]);
        most = max(most, limit[b]);
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) {
        fewest = min(fewest, __shfl_xor(fewest, m));
        most = max(most, __shfl_xor(most, m));
    }
    fewest = __builtin_amdgcn_readfirstlane(fewest);
    const int end = __builtin_amdgcn_readfirstlane(min(p.end, most));

    bf16x8_t q[RB][D / 32];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = first_row + 16 * b + col;
        const bool there = r < p.rows;
        const int64_t at = there ? (int64_t)(p.t0 + r / a.group) * a.q_stride + (int64_t)(kh * a.group + r % a.group) * D : 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            u32x4_t v = {0, 0, 0, 0};
            if (there) v = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(a.Q) + at + query_offset<E4M3>(i, g));
            q[b][i] = as_bf16x8(v);
        }
    }
    float scale = a.scale;
    if (E4M3 && a.cache.k_scale) scale *= as_global(a.cache.k_scale)[kh];

    f32x4_t o[RB][D / 16];
    float m[RB], l[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        m[b] = kNone;
        l[b] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[b][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }

    for (int window = p.begin; window < end; window += kTableKeys) {
        const int stop = min(end, window + kTableKeys);
        // page numbers, as steps of 32 keys may touch them: -1 where there is none or it is out of range
        if (window != p.begin) __syncthreads();
        {
            const int page0 = window >> a.cache.page_log2, last = window + ((stop - window + 31) & ~31) - 1;
            if ((int)threadIdx.x <= (last >> a.cache.page_log2) - page0) {     // at most kTableKeys / 16 of them: window is a multiple of 32
                const int64_t i = page0 + (int)threadIdx.x;
                int id = -1;
                if (i * (1 << a.cache.page_log2) < p.key1 && i < a.seqs.table_stride) id = as_global(a.seqs.table)[p.table + i];
                sh_pages[threadIdx.x] = page_or_none(id, a.cache.n_pages);
            }
        }
        __syncthreads();
        const int* pages = sh_pages - (window >> a.cache.page_log2);
        // the keys of a wavefront's next step are on their way while it works on one; behind its last it asks for that one again
        KeyRegs<D, E4M3> next;
        const int first_step = window + 32 * wave, last_step = first_step + (max(stop - 1 - first_step, 0) & ~127);
        if (first_step < stop) load_keys<D, E4M3>(next, a, pages, first_step, kh, lane);
        for (int step = first_step; step < stop; step += 128) {
            const KeyRegs<D, E4M3> kv = next;
            load_keys<D, E4M3>(next, a, pages, min(step + 128, last_step), kh, lane);
            f32x4_t s[RB][2];
#pragma unroll
            for (int b = 0; b < RB; ++b) s[b][0] = s[b][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bf16x8_t k = key_operand<D, E4M3>(kv, h, i);
#pragma unroll
                    for (int b = 0; b < RB; ++b) s[b][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[b][i], s[b][h], 0, 0, 0);
                }
            const bool ragged = step < p.key0 || step + 32 > fewest || step + 32 > p.key1 || p.bad ||
                                (pages[step >> a.cache.page_log2] | pages[(step + 16) >> a.cache.page_log2]) < 0;
            const int key = step + 8 * g;                       // the lane's eight keys
            bf16x8_t pr[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                float x[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = s[b][e / 4][e % 4] * scale;
                if (ragged) {
                    const bool bad = p.bad || pages[key >> a.cache.page_log2] < 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        x[e] = key + e >= p.key0 && key + e < limit[b] ? (bad ? __builtin_nanf("") : x[e]) : kNone;
                }
                float top = x[0];
#pragma unroll
                for (int e = 1; e < 8; ++e) top = fmaxf(top, x[e]);
                if (__any(top > m[b] + kRise)) {
                    top = fmaxf(top, __shfl_xor(top, 16));
                    top = fmaxf(top, __shfl_xor(top, 32));
                    const float m_new = fmaxf(m[b], top), down = exp2_off(m[b], m_new);
                    m[b] = m_new;
                    l[b] *= down;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) o[b][i] = o[b][i] * down;
                }
                float sum = 0.f, y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = exp2_off(x[e], m[b]);
                    sum += y[e];
                }
                l[b] += sum;
                pr[b] = as_bf16x8(u32x4_t{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7])});
            }
            u32x4_t v[D / 16];
            bool infinite = false;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                if constexpr (E4M3) v[i] = widen8(kv.v[i / 2][2 * (i % 2)], kv.v[i / 2][2 * (i % 2) + 1]);
                else v[i] = kv.v[i];
                if (ragged) {                                    // cells that no key is in may hold anything, and 0 times a NaN is one
                    keep_keys(v[i], key, p.key0, p.key1);
                    infinite |= any_infinite(v[i]);
                }
            }
            // ... and so may keys that only some of the rows see: those are then taken one by one, for the rows that see them
            if (ragged && fewest < min(step + 32, p.key1) && __any(infinite)) {
#pragma unroll 1
                for (int one = step; one < step + 32; ++one)
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        __builtin_amdgcn_sched_barrier(0);       // one operand at a time: this is rare, and registers are not
                        u32x4_t w = v[i];
                        keep_keys(w, key, one, one + 1);
#pragma unroll
                        for (int b = 0; b < RB; ++b) {
                            const f32x4_t add = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(w), pr[b], f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                            if (one < limit[b]) o[b][i] = o[b][i] + add;
                        }
                    }
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int b = 0; b < RB; ++b) o[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v[i]), pr[b], o[b][i], 0, 0, 0);
            }
        }
    }

    // the four wavefronts' results: rows of a block of 16 at a time, 16 threads a row
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
        if (g == 0) {
            sh_m[wave][16 * b + col] = m[b];
            sh_l[wave][16 * b + col] = l[b];
        }
    }
    float v_scale = 1.f;
    if (E4M3 && a.cache.v_scale) v_scale = as_global(a.cache.v_scale)[kh];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        __syncthreads();
        float top = kNone;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sh_m[w][16 * b + col]);
        const float down = exp2_off(m[b], top);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4_t*>(&sh_o[wave][col][16 * i + 4 * g]) = o[b][i] * down;
        __syncthreads();
        const int c = threadIdx.x / 16, d0 = (threadIdx.x % 16) * (D / 16), r = first_row + 16 * b + c;
        if (r < p.rows) {
            float mc = kNone, lc = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) mc = fmaxf(mc, sh_m[w][16 * b + c]);
#pragma unroll
            for (int w = 0; w < 4; ++w) lc += sh_l[w][16 * b + c] * exp2_off(sh_m[w][16 * b + c], mc);
            const int64_t row = (int64_t)(p.t0 + r / a.group) * a.heads + kh * a.group + r % a.group;
            // p.part < 0: the result itself, over its sum (0 where the row sees nothing)
            const float over = (p.part < 0 ? (lc == 0.f ? 0.f : 1.f / lc) : 1.f) * v_scale;
            f32x4_t out[D / 64];
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                out[i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; ++w) out[i] += *reinterpret_cast<const f32x4_t*>(&sh_o[w][c][d0 + 4 * i]);
                out[i] *= over;
            }
            if (p.part < 0) {
                const int64_t at = (int64_t)(p.t0 + r / a.group) * a.o_stride + (int64_t)(kh * a.group + r % a.group) * D + d0;
#pragma unroll
                for (int i = 0; i < D / 64; ++i)
                    *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(a.O) + at + 4 * i) =
                        u32x2_t{bf16_pair(out[i][0], out[i][1]), bf16_pair(out[i][2], out[i][3])};
                if (a.lse && d0 == 0) as_global_out(a.lse)[row] = 0.6931471805599453f * (mc + __builtin_log2f(lc));
            } else {
                const int64_t at = ((int64_t)p.part * a.seqs.n_tokens * a.heads + row);
#pragma unroll
                for (int i = 0; i < D / 64; ++i) *reinterpret_cast<PATCH_EP_GLOBAL f32x4_t*>(as_global_out(a.part_o) + at * D + d0 + 4 * i) = out[i];
                if (d0 == 0) {
                    as_global_out(a.part_ml)[2 * at] = mc;
                    as_global_out(a.part_ml)[2 * at + 1] = lc;
                }
            }
        }
    }
}

// The parts of a row: D / 4 threads hold a part's row, so that a workgroup's other threads take other parts; every load is there before one is needed.  Each
// group of threads adds its parts in their order, then the groups' sums are added in theirs.
template <int D>
__global__ __launch_bounds__(256) void attend_merge_kernel(const AttnArgs a) {
    constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
    __shared__ float sh_top[4], sh_sum[kGroups];
    __shared__ f32x4_t sh_acc[kGroups][kLanes];
    const int64_t rows = (int64_t)a.seqs.n_tokens * a.heads, row = (int64_t)blockIdx.x * a.heads + blockIdx.y;
    const int t = blockIdx.x, head = blockIdx.y;
    const Seq q = seq_at(a.seqs, seq_of(a.seqs, t));
    if (t - q.first >= q.n) return;                           // no sequence has this token
    const int own = own_parts(a, q.len);
    if (a.prefix_parts == 0 && own <= 1) return;              // written by the workgroup itself
    // own parts behind the row's position are left out: nothing in them is seen
    const int pos = q.pos0 + t - q.first, base = a.prefix & ~31;
    const int parts = a.prefix_parts + (pos < base ? 0 : min(own, (pos - base) / a.own_chunk + 1));
    float top = kNone;
    for (int i = threadIdx.x; i < parts; i += 256) top = fmaxf(top, as_global(a.part_ml)[2 * (i * rows + row)]);
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    if ((threadIdx.x & 63) == 0) sh_top[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(sh_top[0], sh_top[1]), fmaxf(sh_top[2], sh_top[3]));
    const int group = threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll 4
    for (int i = group; i < parts; i += kGroups) {
        const int64_t at = i * rows + row;
        const float up = exp2_off(as_global(a.part_ml)[2 * at], top);
        sum += as_global(a.part_ml)[2 * at + 1] * up;
        acc += *reinterpret_cast<const PATCH_EP_GLOBAL f32x4_t*>(as_global(a.part_o) + at * D + 4 * lane) * up;
    }
    sh_acc[group][lane] = acc;
    if (lane == 0) sh_sum[group] = sum;
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int i = 1; i < kGroups; ++i) {
        acc += sh_acc[i][lane];
        sum += sh_sum[i];
    }
    acc *= q.bad ? __builtin_nanf("") : sum == 0.f ? 0.f : 1.f / sum;
    *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(a.O) + t * a.o_stride + (int64_t)head * D + 4 * lane) =
        u32x2_t{bf16_pair(acc[0], acc[1]), bf16_pair(acc[2], acc[3])};
    if (a.lse && lane == 0) as_global_out(a.lse)[row] = 0.6931471805599453f * (top + __builtin_log2f(sum));
}

// Workgroups that a launch over keys is split into: two on each compute unit, all of them there at once.  One sequence of 65000 keys, 8 key heads of 128:
// 512 workgroups 56.5 us, 1024 62.2; 64 rows behind 8192 shared keys 109 and 154; 29 ragged sequences of up to 8000 64.6 and 65.3.
constexpr int64_t kWanted = 512;
constexpr int64_t kMostGroups = (int64_t)1 << 22;

static inline int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

size_t plan_attention(AttnArgs* a, size_t ws_bytes) {
    const int64_t rows = (int64_t)a->seqs.n_tokens * a->heads;
    const size_t per_part = (size_t)rows * (a->cache.head_dim + 2) * 4;
    const int64_t most = ws_bytes < 16 ? 0 : (int64_t)((ws_bytes - 16) / per_part);      // parts that the workspace holds
    a->prefix_parts = 0;
    a->parts = 1;
    if (a->prefix > a->seqs.max_kv) a->prefix = a->seqs.max_kv;
    if (most < 2 || a->seqs.n_seqs < 2) a->prefix = 0;        // every sequence reads the shared keys as its own
    const int base = a->prefix & ~31;
    const int own = a->seqs.max_kv - base;
    int64_t units = (int64_t)a->seqs.n_seqs * a->cache.kv_heads * ((a->seqs.max_q * a->group + 63) / 64);
    int64_t chunk = up_to((own * units + kWanted - 1) / kWanted, 128);
    if (chunk < 256) chunk = 256;
    if (chunk > 4096) chunk = 4096;
    const int64_t groups = ((int64_t)a->seqs.max_q * a->group + 15) / 16;
    if (own / chunk * groups > kMostGroups) chunk = up_to(own / (kMostGroups / groups), 128);
    int64_t prefix_parts = 0;
    if (a->prefix) {
        units = (int64_t)a->cache.kv_heads * (((int64_t)a->seqs.n_tokens * a->group + 63) / 64);
        a->prefix_chunk = (int)up_to(std::min<int64_t>((a->prefix * units + kWanted - 1) / kWanted, a->prefix), 128);
        if (a->prefix_chunk < 256) a->prefix_chunk = 256;
        prefix_parts = (a->prefix + a->prefix_chunk - 1) / a->prefix_chunk;
        if (prefix_parts > most / 2) {
            a->prefix_chunk = (int)up_to((a->prefix + most / 2 - 1) / (most / 2), 128);
            prefix_parts = (a->prefix + a->prefix_chunk - 1) / a->prefix_chunk;
        }
    }
    const int64_t left = most - prefix_parts;
    if (left < 2 && !a->prefix) chunk = up_to(own > 0 ? own : 1, 128);
    else if ((own + chunk - 1) / chunk > left) chunk = up_to((own + left - 1) / left, 128);
    a->own_chunk = (int)chunk;
    const int64_t own_most = own > 0 ? (own + chunk - 1) / chunk : 1;
    a->prefix_parts = (int)prefix_parts;
    a->parts = (int)(prefix_parts + own_most);
    if (a->parts == 1) return 0;
    a->part_o = a->part_ml + 2 * up_to(a->parts * rows, 2);
    return (size_t)(2 * up_to(a->parts * rows, 2) + (int64_t)a->parts * rows * a->cache.head_dim) * 4;
}

template <int D, int RB, bool E4M3>
static void launch_rows(const AttnArgs& a, int front, hipStream_t stream) {
    const int tokens = front ? a.seqs.n_tokens : a.seqs.max_q, parts = front ? a.prefix_parts : a.parts - a.prefix_parts;
    const unsigned groups = (unsigned)(((int64_t)tokens * a.group + 16 * RB - 1) / (16 * RB));
    attend_rows_kernel<D, RB, E4M3><<<dim3(parts * groups, (unsigned)a.cache.kv_heads, front ? 1u : (unsigned)a.seqs.n_seqs), 256, 0, stream>>>(a, front);
}

template <int D, bool E4M3>
static void launch_rows_of(const AttnArgs& a, hipStream_t stream) {
    for (int front = a.prefix_parts ? 1 : 0; front >= 0; --front) {
        const int64_t rows = (int64_t)(front ? a.seqs.n_tokens : a.seqs.max_q) * a.group;
        if (rows <= 16 || D == 256) launch_rows<D, 1, E4M3>(a, front, stream);
        else launch_rows<D, D == 256 ? 1 : 2, E4M3>(a, front, stream);
    }
}

template <int D>
static void launch_d(const AttnArgs& a, hipStream_t stream) {
    if (a.cache.e4m3) launch_rows_of<D, true>(a, stream);
    else launch_rows_of<D, false>(a, stream);
    if (a.parts > 1) {
        attend_merge_kernel<D><<<dim3((unsigned)a.seqs.n_tokens, (unsigned)a.heads), 256, 0, stream>>>(a);
    }
}

void launch_attention(const AttnArgs& a, hipStream_t stream) {
    if (a.cache.head_dim == 64) launch_d<64>(a, stream);
    else if (a.cache.head_dim == 128) launch_d<128>(a, stream);
    else launch_d<256>(a, stream);
}

}  // namespace patch
