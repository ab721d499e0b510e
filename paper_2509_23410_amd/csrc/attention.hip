// Causal attention of a batch's new tokens over a paged cache (patch_attention).
//
//   o_r = sum_j p_rj v_j / sum_j p_rj,   p_rj = exp(q_r . k_j scale - m_r),   over the keys j <= position of row r,
//
// in one pass over the keys: m_r is the running maximum; where it rises, what was summed so far is scaled down by exp(old - new).  Scores, maxima and
// sums are fp32; p is rounded to bf16 as an operand of the second product (its sum is taken before that), which puts 2^-8 of each p into o at most.
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

// Which rows and keys a workgroup has.  The shared front is one batch of all tokens against the pages of one sequence.
struct Span {
    int t0, rows;        // first token, rows (tokens times group)
    int pos0;            // position of token t0; in the shared front each row looks up its own
    int key0, key1;      // keys [key0, key1) are there to be read
    int begin, end;      // and those this workgroup takes, begin a multiple of 64
    int part;            // its partial result, -1: it writes the result itself
    int64_t table;       // its row of the page table
    bool front, bad;
};

// What a row's sum is taken for where the result is written: a NaN in a sequence whose length cannot be, also where the row sees nothing of what is there.
__device__ __forceinline__ float sum_of_row(bool bad, float l) { return bad ? __builtin_nanf("") : l; }

__device__ __forceinline__ Span front_span(const AttnArgs& a, int part) {
    Span p;
    p.front = true;
    p.t0 = 0;
    p.rows = a.seqs.n_tokens * a.group;
    p.pos0 = 0;
    p.key0 = 0;
    p.begin = part * a.prefix_chunk;
    p.end = min(a.prefix, p.begin + a.prefix_chunk);
    p.part = part;
    p.bad = false;
    // The pages are those in the row of the first sequence that has all of the front, or of the longest where none has (no row sees more than that one has).
    // Only sequences with tokens in the call count: one that is idle may not have its pages any more.
    int s = 0, longest = 0;
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < a.seqs.n_seqs; s0 += 64) {
        const Seq q = seq_at(a.seqs, min(s0 + lane, a.seqs.n_seqs - 1));
        const int len = s0 + lane < a.seqs.n_seqs && q.n > 0 && !q.bad ? min(q.len, a.prefix) : 0;
        const uint64_t there = __ballot(len == a.prefix);
        if (there) {
            longest = a.prefix;
            s = s0 + __builtin_ctzll(there);
            break;
        }
        int top = len;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = max(top, __shfl_xor(top, m));
        top = __builtin_amdgcn_readfirstlane(top);
        if (top > longest) {
            longest = top;
            s = s0 + __builtin_ctzll(__ballot(len == top));
        }
    }
    p.key1 = longest;
    p.table = __builtin_amdgcn_readfirstlane(s) * a.seqs.table_stride;
    return p;
}

__device__ __forceinline__ int own_parts(const AttnArgs& a, int len) {
    const int base = a.prefix & ~63;
    return len > a.prefix ? (len - base + a.own_chunk - 1) / a.own_chunk : 0;
}

__device__ __forceinline__ Span own_span(const AttnArgs& a, int s, const Seq& q, int chunk) {
    Span p;
    p.front = false;
    p.t0 = q.first;
    p.rows = q.n * a.group;
    p.pos0 = q.pos0;
    p.key0 = a.prefix;
    p.key1 = max(q.len, a.prefix);
    p.begin = (a.prefix & ~63) + chunk * a.own_chunk;
    p.end = a.line_waves ? q.len : min(q.len, p.begin + a.own_chunk);
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
    const int i = place_of(q, t);
    return i >= 0 ? min(a.prefix, q.pos0 + i + 1) : 0;
}

// Bits of eight keys' cells from `key` on: ones for those that are in [lo, hi).
__device__ __forceinline__ u32x4_t keys_in(int key, int lo, int hi) {
    u32x4_t bits;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int at = key + 2 * e;
        bits[e] = (at >= lo && at < hi ? 0x0000FFFFu : 0u) | (at + 1 >= lo && at + 1 < hi ? 0xFFFF0000u : 0u);
    }
    return bits;
}
__device__ __forceinline__ bool any_infinite(const u32x4_t& v) {      // or NaN
    bool any = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) any |= (v[e] & 0x7F80u) == 0x7F80u || (v[e] & 0x7F800000u) == 0x7F800000u;
    return any;
}

__device__ __forceinline__ float cell_value(const uint8_t* base, int64_t i, bool e4m3) {
    if (e4m3) return __builtin_amdgcn_cvt_f32_fp8((int)as_global(base)[i], 0);
    return __uint_as_float((uint32_t)reinterpret_cast<const PATCH_EP_GLOBAL uint16_t*>(as_global(base))[i] << 16);
}

// One row by one wavefront, key by key and with no key that the row does not see.  In the products of the kernels below a row has 0 times the values of the
// keys behind it, which is a NaN where those are not finite: workgroups that come across such values do their rows again here.  Slow, and hardly ever run: a
// prompt of 1024 over 32 heads of 128 takes 68 us, and 7.5 ms with an infinity in its last key.
// It writes `features` of the head from `first` on, its sums held against *against (null: against the row's maximum), so that another workgroup's others fit.
template <int D, bool E4M3>
__device__ __forceinline__ void attend_row_alone(const AttnArgs& a, const Span& p, int kh, int r, int lane, const float* against, int first, int features) {
    constexpr int E = D / 64;
    const int limit = row_limit(a, p, r), mask = (1 << a.cache.page_log2) - 1;
    const int64_t token = p.t0 + r / a.group;
    const int head = kh * a.group + r % a.group;
    float q[E], acc[E], m = kNone, l = 0.f, scale = a.scale, v_scale = 1.f;
    if (E4M3 && a.cache.k_scale) scale *= as_global(a.cache.k_scale)[kh];
    if (E4M3 && a.cache.v_scale) v_scale = as_global(a.cache.v_scale)[kh];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        q[e] = cell_value(reinterpret_cast<const uint8_t*>(a.Q), token * a.q_stride + (int64_t)head * D + lane * E + e, false);
        acc[e] = 0.f;
    }
#pragma unroll 1
    for (int key = max(p.begin, p.key0); key < min(p.end, limit); ++key) {
        const int id = p.bad ? -1 : page_or_none(as_global(a.seqs.table)[p.table + (key >> a.cache.page_log2)], a.cache.n_pages);
        float s = 0.f, v[E];
        const int64_t cells = (int64_t)kh << a.cache.page_log2;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int d = lane * E + e;
            s += q[e] * cell_value(a.cache.k + max(id, 0) * a.cache.page_bytes, (cells + (key & mask)) * D + d, E4M3);
            v[e] = cell_value(a.cache.v + max(id, 0) * a.cache.page_bytes, cells * D + ((int64_t)d << a.cache.page_log2) + (key & mask), E4M3);
        }
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) s += __shfl_xor(s, x);
        s = id < 0 ? __builtin_nanf("") : s * scale;
        const float m_new = fmaxf(m, s), down = exp2_off(m, m_new), up = exp2_off(s, m_new);
        m = m_new;
        l = l * down + up;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = acc[e] * down + v[e] * up;
    }
    if (against) {
        const float held = *against, move = exp2_off(m, held);
        m = held;
        l *= move;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= move;
    }
    l = sum_of_row(p.bad, l);
    const int64_t row = token * a.heads + head, part = (int64_t)p.part * a.seqs.n_tokens * a.heads + row;
    if (lane * E < first || lane * E >= first + features) return;
    const float over = (p.part < 0 ? (l == 0.f ? 0.f : 1.f / l) : 1.f) * v_scale;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if (p.part < 0) as_global_out(a.O)[token * a.o_stride + (int64_t)head * D + lane * E + e] = (uint16_t)bf16_rne_bits(acc[e] * over);
        else as_global_out(a.part_o)[part * D + lane * E + e] = acc[e] * over;
    }
    if (lane == 0) {
        if (p.part >= 0) {
            as_global_out(a.part_ml)[2 * part] = m;
            as_global_out(a.part_ml)[2 * part + 1] = l;
        } else if (a.lse) {
            as_global_out(a.lse)[row] = 0.6931471805599453f * (m + __builtin_log2f(l));
        }
    }
}

// Few rows: each wavefront takes steps of keys of its own, K and V straight from memory into the operands' registers, RB blocks of 16 rows against them.
// Memory bounds it: a row's work is 4 operations a cell, and the matrix instructions are busy 3 - 5 % of the time (0.26 - 0.38 M of 16 cycles over 1024 SIMDs).
constexpr int kTableKeys = 4096;   // page numbers of so many keys are in LDS at a time

// Page numbers of the keys [window, stop) and on to a multiple of 64 of them, -1 where there is none or it is out of range; window is a multiple of 64 and
// stop at most kTableKeys behind it.  Whether a key of the span is without a page.
__device__ __forceinline__ bool load_pages(const AttnArgs& a, const Span& p, int* to, int window, int stop) {
    const int page0 = window >> a.cache.page_log2, last = window + ((stop - window + 63) & ~63) - 1, count = (last >> a.cache.page_log2) - page0 + 1;
    bool none = false;
    if ((int)threadIdx.x < count) {                              // at most kTableKeys / 16, of 256 threads or more
        const int64_t i = page0 + (int)threadIdx.x;
        const bool there = (i << a.cache.page_log2) < p.key1 && i < a.seqs.table_stride;
        int id = -1;
        if (there && !p.bad) id = page_or_none(as_global(a.seqs.table)[p.table + i], a.cache.n_pages);
        to[threadIdx.x] = id;
        none = there && id < 0;
    }
    return none;
}

// Keys of a step, and workgroups of four wavefronts on a compute unit: with wider heads or more rows a wavefront has its SIMD, and all of its registers, to
// itself.  32 sequences of 2000 keys and 5 tokens of 4 query heads (blocks of 32 rows): 64 keys with a SIMD to itself 67.7 us, 32 72.2, 32 by two 77.3; of 8000
// keys with one head of 256: 91.7 (spilled registers), 58.4, 92.3.
constexpr int step_keys(int head_dim) { return head_dim == 256 ? 32 : 64; }
constexpr int rows_resident(int head_dim, int blocks) { return head_dim * blocks <= 128 ? 2 : 1; }

// The cells of a step, as they are loaded.  Rows of A are given out so that what a lane holds of the first product's result
// is eight keys side by side for each 32, and the 16 (8) of both in one run: V's loads of a step then are whole rows of 64 tokens, 128 bytes together.  With
// steps of 32 keys one sequence of 65000 keys took 59 us in pages of 32 tokens and 71 in pages of 64, whose rows were asked for in halves at different times.
template <int D, int RB, bool E4M3>
struct StepKeys {
    static constexpr int kKeys = step_keys(D), HB = kKeys / 32, kRun = 8 * HB;
    static constexpr int kCell = E4M3 ? 1 : 2;
    u32x4_t k[HB][2][E4M3 ? D / 64 : D / 32];
    u32x4_t v[E4M3 ? HB * D / 32 : HB * D / 16];

    // the first key of the run that a lane's page numbers are of, in K and in V
    static __device__ __forceinline__ int k_key(int lane) { return kRun * ((lane & 15) >> 2); }
    static __device__ __forceinline__ int v_key(int lane) { return kRun * (lane >> 4); }

    // page: that of the lane's run, in range
    __device__ __forceinline__ void load_k(const AttnArgs& a, int page, int step, int kh, int lane) {
        const int at = (step + k_key(lane) + (lane & 3)) & ((1 << a.cache.page_log2) - 1);
        const PATCH_EP_GLOBAL uint8_t* base = as_global(a.cache.k) + page * a.cache.page_bytes + (((int64_t)kh << a.cache.page_log2) + at) * (D * kCell) + 16 * (lane >> 4);
#pragma unroll
        for (int h = 0; h < HB; ++h)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < (E4M3 ? D / 64 : D / 32); ++i)
                    k[h][b][i] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(base + (8 * h + 4 * b) * (D * kCell) + 64 * i);
    }
    __device__ __forceinline__ void load_v(const AttnArgs& a, int page, int step, int kh, int lane) {
        const int at = (step + v_key(lane)) & ((1 << a.cache.page_log2) - 1);
        const PATCH_EP_GLOBAL uint8_t* base = as_global(a.cache.v) + page * a.cache.page_bytes + ((((int64_t)kh * D + (lane & 15)) << a.cache.page_log2) + at) * kCell;
        const int64_t next = (int64_t)(16 * kCell) << a.cache.page_log2;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            if constexpr (E4M3 && HB == 2) {
                v[i] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(base + i * next);
            } else if constexpr (E4M3) {
                const u32x2_t w = *reinterpret_cast<const PATCH_EP_GLOBAL u32x2_t*>(base + i * next);
                v[i / 2][2 * (i % 2)] = w[0];
                v[i / 2][2 * (i % 2) + 1] = w[1];
            } else {
#pragma unroll
                for (int h = 0; h < HB; ++h) v[HB * i + h] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(base + i * next + 16 * h);
            }
        }
    }
    // operands: 32 of a head's values (i counts them) of keys of tile b of half h; eight keys of feature 16 i + column of half h
    __device__ __forceinline__ bf16x8_t k_operand(int h, int b, int i) const {
        if constexpr (E4M3) return as_bf16x8(widen8(k[h][b][i / 2][2 * (i % 2)], k[h][b][i / 2][2 * (i % 2) + 1]));
        else return as_bf16x8(k[h][b][i]);
    }
    __device__ __forceinline__ u32x4_t v_operand(int h, int i) const {
        if constexpr (E4M3 && HB == 2) return widen8(v[i][2 * h], v[i][2 * h + 1]);
        else if constexpr (E4M3) return widen8(v[i / 2][2 * (i % 2)], v[i / 2][2 * (i % 2) + 1]);
        else return v[HB * i + h];
    }
};
// in e4m3 a 16-byte load of K is the operands of two products, and Q's follow it
template <bool E4M3>
__device__ __forceinline__ int query_offset(int i, int g) { return E4M3 ? 64 * (i / 2) + 16 * g + 8 * (i % 2) : 32 * i + 8 * g; }

// What a wavefront has of its rows: running maxima (the same in all lanes of a column), sums (each lane its own keys'), and O^T.
template <int D, int RB, bool E4M3>
struct RowState {
    typedef StepKeys<D, RB, E4M3> Keys;
    static constexpr int HB = Keys::HB;
    f32x4_t o[RB][D / 16];
    float m[RB], l[RB];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            m[b] = kNone;
            l[b] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[b][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }

    static __device__ __forceinline__ void scores(f32x4_t (&s)[RB][HB][2], const bf16x8_t (&q)[RB][D / 32], const Keys& keys) {
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int h = 0; h < HB; ++h) s[b][h][0] = s[b][h][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const bf16x8_t k = keys.k_operand(h, c, i);
#pragma unroll
                    for (int b = 0; b < RB; ++b) s[b][h][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[b][i], s[b][h][c], 0, 0, 0);
                }
    }

    // P of the scores, and what that does to maxima and sums.  ragged: not every row sees all the step's keys; none: the lane's have no page
    __device__ __forceinline__ void soften(bf16x8_t (&pr)[RB][HB], const f32x4_t (&s)[RB][HB][2], const Span& p, int step, bool ragged, bool none, const int (&limit)[RB],
                                           float scale, int lane) {
        const int key = step + Keys::v_key(lane);
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            float x[HB][8], top = kNone;
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    x[h][e] = s[b][h][e / 4][e % 4] * scale;
                    const int at = key + 8 * h + e;
                    if (ragged) x[h][e] = at >= p.key0 && at < limit[b] ? (none ? __builtin_nanf("") : x[h][e]) : kNone;
                    top = fmaxf(top, x[h][e]);
                }
            if (__any(top > m[b] + kRise)) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float m_new = fmaxf(m[b], top), down = exp2_off(m[b], m_new);
                m[b] = m_new;
                l[b] *= down;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) o[b][i] = o[b][i] * down;
            }
            float sum = 0.f;
#pragma unroll
            for (int h = 0; h < HB; ++h) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = exp2_off(x[h][e], m[b]);
                    sum += y[e];
                }
                pr[b][h] = as_bf16x8(u32x4_t{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7])});
            }
            l[b] += sum;
        }
    }

    // Returns whether values that are not finite and that not every row sees went into O.
    __device__ __forceinline__ bool values(const bf16x8_t (&pr)[RB][HB], const Keys& keys, const Span& p, int step, bool ragged, int fewest, int lane) {
        const int key = step + Keys::v_key(lane);
        // cells that no key is in may hold anything, and 0 times a NaN is one; and so may keys that only some of the rows see
        const bool some = fewest < min(step + Keys::kKeys, p.key1);
        bool infinite = false;
        u32x4_t bits[HB];
        if (ragged)
#pragma unroll
            for (int h = 0; h < HB; ++h) bits[h] = keys_in(key + 8 * h, p.key0, p.key1);
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int h = 0; h < HB; ++h) {
                u32x4_t v = keys.v_operand(h, i);
                if (ragged) v &= bits[h];
                if (some) infinite |= any_infinite(v);
#pragma unroll
                for (int b = 0; b < RB; ++b) o[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(v), pr[b][h], o[b][i], 0, 0, 0);
            }
        return infinite;
    }
};

// The queries of rows 0 .. 16 RB - 1 of a span, as the first product's operand.
template <int D, int RB, bool E4M3>
__device__ __forceinline__ void load_queries(bf16x8_t (&q)[RB][D / 32], const AttnArgs& a, const Span& p, int kh, int lane) {
    const int g = lane >> 4, col = lane & 15;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = 16 * b + col;
        const bool there = r < p.rows;
        const int64_t at = there ? (int64_t)(p.t0 + r / a.group) * a.q_stride + (int64_t)(kh * a.group + r % a.group) * D : 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            u32x4_t v = {0, 0, 0, 0};
            if (there) v = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(a.Q) + at + query_offset<E4M3>(i, g));
            q[b][i] = as_bf16x8(v);
        }
    }
}

// The keys that the rows see: of each lane's columns, the fewest of any row, the most.
template <int RB>
__device__ __forceinline__ void row_limits(const AttnArgs& a, const Span& p, int lane, int (&limit)[RB], int* fewest, int* most) {
    int few = 0x7FFFFFFF, many = 0;
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = 16 * b + (lane & 15);
        limit[b] = row_limit(a, p, r);
        if (r < p.rows) few = min(few, limit[b]);
        many = max(many, limit[b]);
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) {
        few = min(few, __shfl_xor(few, m));
        many = max(many, __shfl_xor(many, m));
    }
    *fewest = __builtin_amdgcn_readfirstlane(few);
    *most = __builtin_amdgcn_readfirstlane(many);
}

template <int D, int RB>
struct RowsLds {
    float o[4][16][D + 4], m[4][RB * 16], l[4][RB * 16];
    int pages[kTableKeys / 16];
};

// All rows of a sequence's span (16 RB at most), by a workgroup of four wavefronts that take its steps in turn; their results meet in LDS and are written there.
template <int D, int RB, bool E4M3>
__device__ __forceinline__ void attend_rows(const AttnArgs& a, const Span& p, int kh, RowsLds<D, RB>& sh) {
    typedef StepKeys<D, RB, E4M3> Keys;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, col = lane & 15;
    int limit[RB], fewest, most;
    row_limits<RB>(a, p, lane, limit, &fewest, &most);
    const int end = min(p.end, most);
    bf16x8_t q[RB][D / 32];
    load_queries<D, RB, E4M3>(q, a, p, kh, lane);
    float scale = a.scale;
    if (E4M3 && a.cache.k_scale) scale *= as_global(a.cache.k_scale)[kh];
    RowState<D, RB, E4M3> st;
    st.clear();
    bool redo = false;
    for (int window = p.begin; window < end; window += kTableKeys) {
        const int stop = min(end, window + kTableKeys);
        // page numbers, as steps may touch them: -1 where there is none or it is out of range
        if (window != p.begin) __syncthreads();
        load_pages(a, p, sh.pages, window, stop);
        __syncthreads();
        const int* pages = sh.pages - (window >> a.cache.page_log2);
        const auto page_at = [&](int key) { return pages[key >> a.cache.page_log2]; };
        Keys keys;
        int step = window + Keys::kKeys * wave;
        if (step < stop) {
            keys.load_k(a, max(page_at(step + Keys::k_key(lane)), 0), step, kh, lane);
            keys.load_v(a, max(page_at(step + Keys::v_key(lane)), 0), step, kh, lane);
        }
        for (; step < stop; step += 4 * Keys::kKeys) {           // the next K is on its way once this one is done with, and so the next V
            const int next = step + 4 * Keys::kKeys;
            const bool none = page_at(step + Keys::v_key(lane)) < 0, ragged = step < p.key0 || step + Keys::kKeys > fewest || step + Keys::kKeys > p.key1 || __any(none);
            f32x4_t s[RB][Keys::HB][2];
            bf16x8_t pr[RB][Keys::HB];
            st.scores(s, q, keys);
            if (next < stop) keys.load_k(a, max(page_at(next + Keys::k_key(lane)), 0), next, kh, lane);
            st.soften(pr, s, p, step, ragged, none, limit, scale, lane);
            redo |= st.values(pr, keys, p, step, ragged, fewest, lane);
            if (next < stop) keys.load_v(a, max(page_at(next + Keys::v_key(lane)), 0), next, kh, lane);
        }
    }
    if (__syncthreads_or(redo)) {
        for (int r = wave; r < min(16 * RB, p.rows); r += 4) attend_row_alone<D, E4M3>(a, p, kh, r, lane, nullptr, 0, D);
        return;
    }

    // the four wavefronts' results: rows of a block of 16 at a time, 16 threads a row
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        st.l[b] += __shfl_xor(st.l[b], 16);
        st.l[b] += __shfl_xor(st.l[b], 32);
        if (g == 0) {
            sh.m[wave][16 * b + col] = st.m[b];
            sh.l[wave][16 * b + col] = st.l[b];
        }
    }
    float v_scale = 1.f;
    if (E4M3 && a.cache.v_scale) v_scale = as_global(a.cache.v_scale)[kh];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        __syncthreads();
        float top = kNone;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = fmaxf(top, sh.m[w][16 * b + col]);
        const float down = exp2_off(st.m[b], top);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) *reinterpret_cast<f32x4_t*>(&sh.o[wave][col][16 * i + 4 * g]) = st.o[b][i] * down;
        __syncthreads();
        const int c = threadIdx.x / 16, d0 = (threadIdx.x % 16) * (D / 16), r = 16 * b + c;
        if (r < p.rows) {
            float mc = kNone, lc = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) mc = fmaxf(mc, sh.m[w][16 * b + c]);
#pragma unroll
            for (int w = 0; w < 4; ++w) lc += sh.l[w][16 * b + c] * exp2_off(sh.m[w][16 * b + c], mc);
            lc = sum_of_row(p.bad, lc);
            const int64_t row = (int64_t)(p.t0 + r / a.group) * a.heads + kh * a.group + r % a.group;
            const float over = (lc == 0.f ? 0.f : 1.f / lc) * v_scale;                   // (0 where the row sees nothing)
            const int64_t at = (int64_t)(p.t0 + r / a.group) * a.o_stride + (int64_t)(kh * a.group + r % a.group) * D + d0;
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                f32x4_t out = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < 4; ++w) out += *reinterpret_cast<const f32x4_t*>(&sh.o[w][c][d0 + 4 * i]);
                out *= over;
                *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(a.O) + at + 4 * i) = u32x2_t{bf16_pair(out[0], out[1]), bf16_pair(out[2], out[3])};
            }
            if (a.lse && d0 == 0) as_global_out(a.lse)[row] = 0.6931471805599453f * (mc + __builtin_log2f(lc));
        }
    }
}

// Many rows: a workgroup's wavefronts have 32 rows each, and the keys come through LDS for all of them, kTile at a time, the next ones on their way through
// registers meanwhile.  The products are the ones above on 32 x 32 x 16 instructions.  A prompt of 4096 over 32 heads of 128: 167 - 178 us on different cards,
// 825 - 770 TFLOP/s; with operands from registers alone it would be 116, with the reads from LDS (all of K and V for each wavefront) and no softmax 160: those
// two bound it.  27 % of the LDS' busy cycles are bank conflicts; which of its reads and writes have them has not been found out.
typedef float f32x16_t __attribute__((ext_vector_type(16)));

// Where 16-byte chunk c of a row lies in LDS: the same chunk of 8 rows side by side is in 8 different places of 128 bytes, of 16 rows in 16 of 256
template <int CHUNKS>
__device__ __forceinline__ int chunk_at(int row, int c) {
    return row * CHUNKS + (CHUNKS == 4 ? c ^ (((row >> 1) ^ (row >> 3)) & 3) : CHUNKS == 8 ? c ^ ((row + (row >> 3)) & 7) : c ^ (row & 15));
}
// The row of the K tile that key i of 32 is in: a lane's eight values of P in the order of the second product's operand (bits 2 and 3 change places)
__device__ __forceinline__ int key_row(int i) { return (i & ~12) | ((i & 4) << 1) | ((i & 8) >> 1); }

// Heads of 256 are two workgroups, of 128 of V's features each: with the sums of all 256 in registers a wavefront has its SIMD to itself, and the compiler
// moves them about (6 pieces of up to 700 tokens, 4 key heads of 2: 244 us, and 127 so, though the first product is made twice).
template <int D, int NW>
struct TilesLds {
    static constexpr int kTile = D == 256 ? 32 : 64, DV = D == 256 ? 128 : D;
    u32x4_t k[2][kTile * D / 8], v[2][kTile * DV / 8];
    int infinite[2][NW], fewest[NW], pages[kTableKeys / 16];
    float m[32 * NW];
};

// 32 NW rows of a span from first_row on, by a workgroup of NW wavefronts.
template <int D, int NW, bool E4M3>
__device__ __forceinline__ void attend_tiles(const AttnArgs& a, const Span& p, int kh, int half, int first_row, TilesLds<D, NW>& sh) {
    constexpr int kTile = TilesLds<D, NW>::kTile, kBlocks = kTile / 32;        // keys at a time, as 32 to an instruction
    constexpr int DV = TilesLds<D, NW>::DV;
    constexpr int kThreads = 64 * NW, kCells = E4M3 ? 16 : 8;                  // of a 16-byte load
    constexpr int kLoadsK = kTile * D / kCells, kEachK = (kLoadsK + kThreads - 1) / kThreads;
    constexpr int kLoadsV = kTile * DV / kCells, kEachV = (kLoadsV + kThreads - 1) / kThreads;
    constexpr int kRowLoads = D / kCells, kKeyLoads = kTile / kCells;          // of a key, of a feature
    static_assert(kThreads % kRowLoads == 0 && kThreads % kKeyLoads == 0 && (kLoadsK % kThreads == 0 || kLoadsK < kThreads) &&
                  (kLoadsV % kThreads == 0 || kLoadsV < kThreads), "staging");
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5, col = lane & 31;
    const int r = first_row + 32 * wave + col;
    const bool there = r < p.rows;
    const int limit = row_limit(a, p, r);
    int fewest = there ? limit : 0x7FFFFFFF, most = limit;
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) {
        fewest = min(fewest, __shfl_xor(fewest, m));
        most = max(most, __shfl_xor(most, m));
    }
    fewest = __builtin_amdgcn_readfirstlane(fewest);
    most = __builtin_amdgcn_readfirstlane(most);
    // keys up to the last one that any row of the workgroup sees
    const int end = p.front ? p.end : min(p.end, p.pos0 + min(first_row + 32 * NW - 1, p.rows - 1) / a.group + 1);

    const int64_t q_at = there ? (int64_t)(p.t0 + r / a.group) * a.q_stride + (int64_t)(kh * a.group + r % a.group) * D : 0;
    float scale = a.scale;
    if (E4M3 && a.cache.k_scale) scale *= as_global(a.cache.k_scale)[kh];
    bf16x8_t q[D / 16];
    const uint32_t turn = scale < 0.f ? 0x80008000u : 0u;                      // so that the largest product is the largest score
    if (scale < 0.f) scale = -scale;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        u32x4_t v = {0, 0, 0, 0};
        if (there) v = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(a.Q) + q_at + 16 * i + 8 * h) ^ turn;
        q[i] = as_bf16x8(v);
    }
    if (scale == 0.f) scale = 1.17549435e-38f;                                 // (a masked score, minus infinity, has to stay that)

    f32x16_t o[DV / 32];
#pragma unroll
    for (int i = 0; i < DV / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.f;
    float m = kNone, l = 0.f;
    bool redo = false;

    // staging: each thread's key rows of K (one a load), and keys of V (the same ones for all its loads, of different features)
    const int page_mask = (1 << a.cache.page_log2) - 1;
    const int k_row = tid / kRowLoads, v_row = tid / kKeyLoads, v_key = (tid % kKeyLoads) * kCells;
    constexpr int kRowStep = kThreads / kRowLoads, kFeatureStep = kThreads / kKeyLoads, kBytes = 16 / kCells;
    const uint32_t page_bytes = (uint32_t)a.cache.page_bytes;
    const uint8_t* k_base = a.cache.k + ((((int64_t)kh * D) << a.cache.page_log2) + (tid % kRowLoads) * kCells) * kBytes;
    const uint8_t* v_base = a.cache.v + (((int64_t)kh * D + half * DV + v_row) << a.cache.page_log2) * kBytes;
    const uint32_t v_step = (uint32_t)(kFeatureStep * kBytes) << a.cache.page_log2;
    u32x4_t k_regs[kEachK], v_regs[kEachV];
    bool k_none[kEachK], v_none, any_none = false;                              // keys without a page
    int window = p.begin, fewest_of_all = 0;
    const auto ask_keys = [&](int tile) {
        const int* pages = sh.pages - (window >> a.cache.page_log2);
        if (kLoadsK >= kThreads || tid < kLoadsK) {
#pragma unroll
            for (int i = 0; i < kEachK; ++i) {
                const int key = tile + k_row + i * kRowStep, page = pages[key >> a.cache.page_log2];
                k_none[i] = page < 0;
                k_regs[i] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(k_base) + ((uint64_t)(uint32_t)max(page, 0) * page_bytes + (uint32_t)((key & page_mask) * (D * kBytes))));
            }
        }
        if (kLoadsV >= kThreads || tid < kLoadsV) {
            const int key = tile + v_key, page = pages[key >> a.cache.page_log2];
            v_none = page < 0;
            const PATCH_EP_GLOBAL uint8_t* at = as_global(v_base) + ((uint64_t)(uint32_t)max(page, 0) * page_bytes + (uint32_t)((key & page_mask) * kBytes));
#pragma unroll
            for (int i = 0; i < kEachV; ++i) v_regs[i] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(at + i * v_step);
        }
    };
    const auto put_keys = [&](int tile, int buffer) {
        constexpr int kParts = kCells / 8;
        const bool edge = tile < p.key0 || tile + kTile > p.key1, seen_by_all = tile + kTile <= fewest_of_all;
        bool infinite = false;
        if (kLoadsK >= kThreads || tid < kLoadsK) {
#pragma unroll
            for (int i = 0; i < kEachK; ++i) {
                const int at = k_row + i * kRowStep, row = (at & ~31) | key_row(at & 31);
#pragma unroll
                for (int b = 0; b < kParts; ++b) {
                    u32x4_t k = k_regs[i];
                    if constexpr (E4M3) k = widen8(k_regs[i][2 * b], k_regs[i][2 * b + 1]);
                    if (any_none && k_none[i]) k = u32x4_t{0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u, 0x7FC07FC0u};     // a page that is not there: NaN scores
                    sh.k[buffer][chunk_at<D / 8>(row, (tid % kRowLoads) * kParts + b)] = k;
                }
            }
        }
        if (kLoadsV >= kThreads || tid < kLoadsV) {
#pragma unroll
            for (int i = 0; i < kEachV; ++i) {
#pragma unroll
                for (int b = 0; b < kParts; ++b) {
                    u32x4_t v = v_regs[i];
                    if constexpr (E4M3) v = widen8(v_regs[i][2 * b], v_regs[i][2 * b + 1]);
                    if (any_none && v_none) v = u32x4_t{0, 0, 0, 0};
                    if (edge) v &= keys_in(tile + v_key + 8 * b, p.key0, p.key1);        // cells that no key is in
                    if (!seen_by_all) infinite |= any_infinite(v);
                    sh.v[buffer][chunk_at<kTile / 8>(v_row + i * kFeatureStep, v_key / 8 + b)] = v;
                }
            }
        }
        if (!seen_by_all) {
            infinite = __any(infinite);
            if (lane == 0) sh.infinite[buffer][wave] = infinite;
        }
    };

    if (lane == 0) sh.fewest[wave] = fewest;
    if (p.begin < end) any_none = __syncthreads_or(load_pages(a, p, sh.pages, window, min(end, window + kTableKeys)));
    else __syncthreads();
    fewest_of_all = sh.fewest[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) fewest_of_all = min(fewest_of_all, sh.fewest[w]);
    fewest_of_all = __builtin_amdgcn_readfirstlane(fewest_of_all);
    if (p.begin < end) {
        ask_keys(p.begin);
        put_keys(p.begin, 0);
        __syncthreads();
    }
    int buffer = 0;
    for (int tile = p.begin; tile < end; tile += kTile, buffer ^= 1) {
        const bool more = tile + kTile < end;
        if (more) {
            if (tile + kTile == window + kTableKeys) {                         // (nobody looks into the table between here and the last barrier)
                window += kTableKeys;
                any_none = __syncthreads_or(load_pages(a, p, sh.pages, window, min(end, window + kTableKeys)));
            }
            ask_keys(tile + kTile);
        }
        if (tile < most) {
            // ahead of a wavefront that is in its softmax: the matrix instructions of one then lie under the rest of the other.  A prompt of 4096 over 32 heads of
            // 128, both on one card: 185.8 us, and 175.2 so.
            __builtin_amdgcn_s_setprio(1);
            f32x16_t s[kBlocks];
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[b][e] = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
                    s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(sh.k[buffer][chunk_at<D / 8>(32 * b + col, 2 * i + h)]), q[i], s[b], 0, 0, 0);
            // the operands of the next few products are on their way out of LDS while one runs
            __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
            for (int i = 0; i < kBlocks * D / 16 - 6; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            }
            __builtin_amdgcn_sched_group_barrier(0x008, 6, 0);
            __builtin_amdgcn_s_setprio(0);
            const bool ragged = tile < p.key0 || tile + kTile > fewest;
            if (ragged) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int key = tile + 32 * b + 16 * (e / 8) + 8 * h + e % 8;
                        if (key < p.key0 || key >= limit) s[b][e] = kNone;
                    }
            }
            float top = s[0][0];
#pragma unroll
            for (int e = 1; e < kTile / 2; ++e) top = fmaxf(top, s[e / 16][e % 16]);
            top *= scale;
            if (__any(top > m + kRise)) {
                top = fmaxf(top, __shfl_xor(top, 32));
                const float m_new = fmaxf(m, top), down = exp2_off(m, m_new);
                m = m_new;
                l *= down;
#pragma unroll
                for (int i = 0; i < DV / 32; ++i) o[i] = o[i] * down;
            }
            const float off = m == kNone ? 0.f : m;
            bf16x8_t pr[kTile / 16];
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k) {
                float y[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    y[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k / 2][8 * (k % 2) + e], scale, -off));
                    sum[k % 2] += y[e];
                }
                pr[k] = as_bf16x8(u32x4_t{bf16_pair(y[0], y[1]), bf16_pair(y[2], y[3]), bf16_pair(y[4], y[5]), bf16_pair(y[6], y[7])});
            }
            l += sum[0] + sum[1];
            if (fewest < min(tile + kTile, p.key1)) {                          // keys that only some of the rows see, and not finite?
#pragma unroll
                for (int w = 0; w < NW; ++w) redo |= sh.infinite[buffer][w] != 0;
            }
#pragma unroll
            for (int k = 0; k < kTile / 16; ++k)
#pragma unroll
                for (int i = 0; i < DV / 32; ++i)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(sh.v[buffer][chunk_at<kTile / 8>(32 * i + col, 2 * k + h)]), pr[k], o[i], 0, 0, 0);
        }
        if (more) put_keys(tile + kTile, buffer ^ 1);
        __syncthreads();
    }

    if (__syncthreads_or(redo)) {
        if (h == 0) sh.m[32 * wave + col] = m;
        __syncthreads();
        for (int i = wave; i < min(32 * NW, p.rows - first_row); i += NW) attend_row_alone<D, E4M3>(a, p, kh, first_row + i, lane, &sh.m[i], half * DV, DV);
        return;
    }
    l = sum_of_row(p.bad, l + __shfl_xor(l, 32));
    if (!there) return;
    float v_scale = 1.f;
    if (E4M3 && a.cache.v_scale) v_scale = as_global(a.cache.v_scale)[kh];
    const int64_t token = p.t0 + r / a.group;
    const int head = kh * a.group + r % a.group;
    const int64_t row = token * a.heads + head;
    if (p.part < 0) {
        const float over = (l == 0.f ? 0.f : 1.f / l) * v_scale;
        const int64_t at = token * a.o_stride + (int64_t)head * D + half * DV + 4 * h;
#pragma unroll
        for (int i = 0; i < DV / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(a.O) + at + 32 * i + 2 * e) =
                    u32x2_t{bf16_pair(o[i][e] * over, o[i][e + 1] * over), bf16_pair(o[i][e + 2] * over, o[i][e + 3] * over)};
        if (a.lse && h == 0 && half == 0) as_global_out(a.lse)[row] = 0.6931471805599453f * (m + __builtin_log2f(l));
    } else {
        const int64_t at = (int64_t)p.part * a.seqs.n_tokens * a.heads + row;
#pragma unroll
        for (int i = 0; i < DV / 32; ++i)
#pragma unroll
            for (int e = 0; e < 16; e += 4)
                *reinterpret_cast<PATCH_EP_GLOBAL f32x4_t*>(as_global_out(a.part_o) + at * D + half * DV + 4 * h + 32 * i + 2 * e) =
                    f32x4_t{o[i][e] * v_scale, o[i][e + 1] * v_scale, o[i][e + 2] * v_scale, o[i][e + 3] * v_scale};
        if (h == 0 && half == 0) {
            as_global_out(a.part_ml)[2 * at] = m;
            as_global_out(a.part_ml)[2 * at + 1] = l;
        }
    }
}

template <int D, int NW, bool E4M3>
__global__ __launch_bounds__(64 * NW, 2) void attend_tiles_kernel(const AttnArgs a, const int front) {
    __shared__ TilesLds<D, NW> sh;
    constexpr int kHalves = D / TilesLds<D, NW>::DV;
    // key heads are the fastest index: with 8 of them, or 16 and so on, each die has heads of its own, and those in its L2
    const int kh = blockIdx.x % a.cache.kv_heads, rest = blockIdx.x / a.cache.kv_heads / kHalves, half = blockIdx.x / a.cache.kv_heads % kHalves;
    const int groups = ((front ? a.seqs.n_tokens : a.seqs.max_q) * a.group + 32 * NW - 1) / (32 * NW);
    const int chunk = rest / groups, first_row = (groups - 1 - rest % groups) * (32 * NW);       // the rows that see most first
    const Span p = front ? front_span(a, chunk) : own_span(a, blockIdx.y, seq_at(a.seqs, blockIdx.y), chunk);
    if (first_row >= p.rows) return;
    if (p.begin >= p.end && (p.part >= 0 || chunk > 0)) return;                // no keys here; the first workgroup of rows that see none writes that
    attend_tiles<D, NW, E4M3>(a, p, kh, half, first_row, sh);
}

// Few rows a sequence and nowhere to put parts: a workgroup for each sequence and key head.
template <int D, int RB, bool E4M3>
__global__ __launch_bounds__(256, rows_resident(D, RB)) void attend_rows_kernel(const AttnArgs a) {
    __shared__ RowsLds<D, RB> sh;
    const int s = blockIdx.x / a.cache.kv_heads;
    const Span p = own_span(a, s, seq_at(a.seqs, s), 0);
    if (p.rows > 0) attend_rows<D, RB, E4M3>(a, p, blockIdx.x % a.cache.kv_heads, sh);
}

// A step of the line of all sequences' own keys: sequence by sequence, in it head by head, in that so many keys at a time.
struct Place {
    Seq q;
    int s, kh, n, i, unit;      // sequence, key head, steps of a head of it, which of them this is, and the line's number of the head's first
};

// The steps [me * stretch, + stretch) of the line, by one wavefront by itself: the keys of its next step, of whatever head, and the page numbers of the one
// behind that are on their way while it works on one, and what it has of a head's rows it writes when that head or its stretch ends.  One sequence of 65000
// keys, 8 key heads of 128: 50.6 us, 5.3 TB/s; 29 ragged ones of up to 8000 in e4m3 54.7 us, 4.7 TB/s (a copy of 2 GB: 4.9).
template <int D, int RB, bool E4M3>
__device__ __forceinline__ void attend_line(const AttnArgs& a, int me) {
    typedef StepKeys<D, RB, E4M3> Keys;
    constexpr int kKeys = Keys::kKeys;
    const int lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15, KH = a.cache.kv_heads, base = a.prefix & ~63;
    const auto steps_in = [&](const Seq& q) { return q.n > 0 && q.len > a.prefix ? (q.len - base + kKeys - 1) / kKeys : 0; };
    // steps of 64 sequences from s0 on, one a lane, and their sums up to each
    const auto sums_of = [&](int s0, Seq* q, int* upto) {
        *q = seq_at(a.seqs, min(s0 + lane, a.seqs.n_seqs - 1));
        const int n = s0 + lane < a.seqs.n_seqs ? steps_in(*q) : 0;
        int sum = n;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int other = __shfl_up(sum, m);
            if (lane >= m) sum += other;
        }
        *upto = sum;
        return n;
    };
    Place c;
    c.s = c.unit = 0;
    if (a.seqs.n_seqs == 1) c.q = seq_at(a.seqs, 0);
    else c.q = Seq{};
    int total, n0 = 0, upto0 = 0;
    Seq q0 = c.q;
    if (a.seqs.n_seqs == 1) {
        total = steps_in(c.q) * KH;
    } else {
        n0 = sums_of(0, &q0, &upto0);
        total = __builtin_amdgcn_readlane(upto0, 63);
        for (int s0 = 64; s0 < a.seqs.n_seqs; s0 += 64) {
            Seq unused;
            int upto;
            sums_of(s0, &unused, &upto);
            total += __builtin_amdgcn_readlane(upto, 63);
        }
        total *= KH;
    }
    const int stretch = max((total + a.line_waves - 1) / a.line_waves, a.least_steps);
    if (total == 0 || me > (total - 1) / stretch) return;
    const int at = me * stretch, count = min(stretch, total - at);
    if (a.seqs.n_seqs > 1) {
        for (int s0 = 0, before = 0; s0 < a.seqs.n_seqs; s0 += 64) {
            const uint64_t there = __ballot(before + KH * upto0 > at);
            if (there) {
                const int which = __builtin_ctzll(there);
                c.s = s0 + which;
                c.unit = before + KH * (__builtin_amdgcn_readlane(upto0, which) - __builtin_amdgcn_readlane(n0, which));
                c.q.first = __builtin_amdgcn_readlane(q0.first, which);
                c.q.n = __builtin_amdgcn_readlane(q0.n, which);
                c.q.len = __builtin_amdgcn_readlane(q0.len, which);
                c.q.pos0 = c.q.len - c.q.n;
                c.q.bad = __builtin_amdgcn_readlane((int)q0.bad, which);
                break;
            }
            before += KH * __builtin_amdgcn_readlane(upto0, 63);
            n0 = sums_of(s0 + 64, &q0, &upto0);
        }
    }
    c.n = steps_in(c.q);
    if (c.n == 0) return;                                         // (there is one: total is not 0)
    c.kh = (at - c.unit) / c.n;
    c.unit += c.kh * c.n;
    c.i = at - c.unit;

    // goes to the step behind p, which there is
    const auto go_on = [&](Place& p) {
        if (++p.i < p.n) return;
        p.i = 0;
        p.unit += p.n;
        if (++p.kh < KH) return;
        p.kh = 0;
        do {
            p.s = min(p.s + 1, a.seqs.n_seqs - 1);
            p.q = seq_at(a.seqs, p.s);
            p.n = steps_in(p.q);
        } while (p.n == 0 && p.s < a.seqs.n_seqs - 1);
    };
    // pages of the lane's runs of keys in K and in V: -1 where there is none
    const auto ask_pages = [&](const Place& p, int* k_page, int* v_page) {
        const int k_key = base + kKeys * p.i + Keys::k_key(lane), v_key = base + kKeys * p.i + Keys::v_key(lane);
        const PATCH_EP_GLOBAL int32_t* row = as_global(a.seqs.table) + p.s * a.seqs.table_stride;
        *k_page = *v_page = -1;
        if (k_key < p.q.len) *k_page = row[k_key >> a.cache.page_log2];
        if (v_key < p.q.len) *v_page = row[v_key >> a.cache.page_log2];
    };
    const auto checked = [&](const Place& p, int id) { return p.q.bad ? -1 : page_or_none(id, a.cache.n_pages); };

    int token_of[RB], head_of[RB];                                // of the lane's columns
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        token_of[b] = (16 * b + col) / a.group;
        head_of[b] = (16 * b + col) % a.group;
    }
    bf16x8_t q[RB][D / 32];
    int limit[RB];
    float scale = 0.f;
    RowState<D, RB, E4M3> st;
    Span p;
    bool redo = false;
    // Loads come back in the order in which they were asked for: the page numbers of a step are asked for in front of the cells of the step before it, so that
    // the wait for them is none for those.
    Keys keys;
    Place f = c;
    if (count > 1) go_on(f);
    int k_now, v_now, k_id, v_id;
    ask_pages(c, &k_now, &v_now);
    ask_pages(f, &k_id, &v_id);
    k_now = checked(c, k_now);
    v_now = checked(c, v_now);
    keys.load_k(a, max(k_now, 0), base + kKeys * c.i, c.kh, lane);
    keys.load_v(a, max(v_now, 0), base + kKeys * c.i, c.kh, lane);
    for (int t = 0; t < count; ++t) {
        const int step = base + kKeys * c.i;
        if (t == 0 || c.i == 0) {                                 // a head's rows
            p = own_span(a, c.s, c.q, 0);
            p.begin = step;
            scale = a.scale;
            if (E4M3 && a.cache.k_scale) scale *= as_global(a.cache.k_scale)[c.kh];
            load_queries<D, RB, E4M3>(q, a, p, c.kh, lane);
#pragma unroll
            for (int b = 0; b < RB; ++b) limit[b] = 16 * b + col < p.rows ? p.pos0 + token_of[b] + 1 : 0;
            st.clear();
            redo = false;
        }
        const bool none = v_now < 0, more = t + 1 < count;
        const int fewest = p.pos0 + 1;
        const bool ragged = step < p.key0 || step + kKeys > fewest || __any(none);       // (a row sees nothing that is not there)
        f32x4_t s[RB][Keys::HB][2];
        bf16x8_t pr[RB][Keys::HB];
        st.scores(s, q, keys);
        k_now = checked(f, k_id);
        v_now = checked(f, v_id);
        Place ff = f;
        if (t + 2 < count) go_on(ff);
        ask_pages(ff, &k_id, &v_id);
        if (more) keys.load_k(a, max(k_now, 0), base + kKeys * f.i, f.kh, lane);
        st.soften(pr, s, p, step, ragged, none, limit, scale, lane);
        redo |= st.values(pr, keys, p, step, ragged, fewest, lane);
        if (more) keys.load_v(a, max(v_now, 0), base + kKeys * f.i, f.kh, lane);

        const bool ends = c.i == c.n - 1;
        if (ends || t == count - 1) {
            const int part = me - c.unit / stretch;
            p.end = min(p.end, step + kKeys);
            p.part = a.prefix_parts == 0 && ends && c.i <= t ? -1 : a.prefix_parts + part;      // all of the head's keys: the result itself
            if (ends && lane == 0) as_global_out(a.unit_parts)[c.s * KH + c.kh] = part + 1;
            if (__any(redo)) {
                for (int r = 0; r < min(16 * RB, p.rows); ++r) attend_row_alone<D, E4M3>(a, p, c.kh, r, lane, nullptr, 0, D);
            } else {
                float v_scale = 1.f;
                if (E4M3 && a.cache.v_scale) v_scale = as_global(a.cache.v_scale)[c.kh];
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    float l = st.l[b];
                    l += __shfl_xor(l, 16);
                    l += __shfl_xor(l, 32);
                    l = sum_of_row(p.bad, l);
                    if (16 * b + col >= p.rows) continue;
                    const int64_t token = p.t0 + token_of[b];
                    const int head = c.kh * a.group + head_of[b];
                    const int64_t row = token * a.heads + head, to = (int64_t)p.part * a.seqs.n_tokens * a.heads + row;
                    const float over = (p.part < 0 ? (l == 0.f ? 0.f : 1.f / l) : 1.f) * v_scale;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const f32x4_t o = st.o[b][i] * over;
                        if (p.part < 0)
                            *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(a.O) + token * a.o_stride + (int64_t)head * D + 16 * i + 4 * g) =
                                u32x2_t{bf16_pair(o[0], o[1]), bf16_pair(o[2], o[3])};
                        else
                            *reinterpret_cast<PATCH_EP_GLOBAL f32x4_t*>(as_global_out(a.part_o) + to * D + 16 * i + 4 * g) = o;
                    }
                    if (g == 0) {
                        if (p.part >= 0) {
                            as_global_out(a.part_ml)[2 * to] = st.m[b];
                            as_global_out(a.part_ml)[2 * to + 1] = l;
                        } else if (a.lse) {
                            as_global_out(a.lse)[row] = 0.6931471805599453f * (st.m[b] + __builtin_log2f(l));
                        }
                    }
                }
            }
        }
        c = f;
        f = ff;
    }
}

// Few rows a sequence: the first front_blocks workgroups have the shared front, for all rows (in blocks of 128); beside them, on the same compute units, the
// others have the sequences' own keys.  Those are one line of steps, and each wavefront has an equal stretch of it, whatever lengths it falls on: it ends
// with the others, and the work of a compute unit is bounded by nothing but what its memory can bring.  A sequence's head that lies in several stretches is
// as many parts; who has its last step notes how many.
template <int D, int RB, bool E4M3, bool FRONT>
__global__ __launch_bounds__(256, rows_resident(D, RB)) void attend_few_kernel(const AttnArgs a) {
    if constexpr (FRONT) {
        __shared__ TilesLds<D, 4> sh;
        constexpr int kHalves = D / TilesLds<D, 4>::DV;
        if ((int)blockIdx.x < a.front_blocks) {
            const int kh = blockIdx.x % a.cache.kv_heads, rest = blockIdx.x / a.cache.kv_heads / kHalves, half = blockIdx.x / a.cache.kv_heads % kHalves;
            const int groups = (a.seqs.n_tokens * a.group + 127) / 128;
            attend_tiles<D, 4, E4M3>(a, front_span(a, rest / groups), kh, half, rest % groups * 128, sh);
            return;
        }
    }
    attend_line<D, RB, E4M3>(a, __builtin_amdgcn_readfirstlane((blockIdx.x - a.front_blocks) * 4 + (threadIdx.x >> 6)));
}

// The parts of a row: D / 4 threads hold a part's row, so that a workgroup's other threads take other parts; every load is there before one is needed.  Each
// group of threads adds its parts in their order, then the groups' sums are added in theirs.  64 x 32 rows of 11 parts and more: 5.6 us; 32 rows of 250 parts 7.
template <int D>
__global__ __launch_bounds__(256) void attend_merge_kernel(const AttnArgs a) {
    constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
    __shared__ float sh_top[4], sh_sum[kGroups];
    __shared__ f32x4_t sh_acc[kGroups][kLanes];
    const int64_t rows = (int64_t)a.seqs.n_tokens * a.heads, row = (int64_t)blockIdx.x * a.heads + blockIdx.y;
    const int t = blockIdx.x, head = blockIdx.y;
    const int seq = seq_of(a.seqs, t);
    const Seq q = seq_at(a.seqs, seq);
    const int place = place_of(q, t);
    if (place < 0 || place >= a.seqs.max_q) return;     // no sequence has this token, or it is one too many
    const int own = !a.line_waves ? own_parts(a, q.len) : q.len <= a.prefix ? 0 : as_global(a.unit_parts)[seq * a.cache.kv_heads + head / a.group];
    if (a.prefix_parts == 0 && (own == 1 || (own == 0 && !a.line_waves))) return;     // written by the workgroup itself
    const int parts = a.prefix_parts + own;
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
    sum = sum_of_row(q.bad, sum);
    acc *= sum == 0.f ? 0.f : 1.f / sum;
    *reinterpret_cast<PATCH_EP_GLOBAL u32x2_t*>(as_global_out(a.O) + t * a.o_stride + (int64_t)head * D + 4 * lane) =
        u32x2_t{bf16_pair(acc[0], acc[1]), bf16_pair(acc[2], acc[3])};
    if (a.lse && lane == 0) as_global_out(a.lse)[row] = 0.6931471805599453f * (top + __builtin_log2f(sum));
}

// Which kernel takes so many rows of a key head (those of a sequence, or of all in the shared front), as the rows of a workgroup.
static int rows_of_block(int64_t rows, int head_dim) {
    if (rows <= 16) return 16;
    if (rows <= 32 && head_dim <= 128) return 32;
    return rows <= 128 ? 128 : 256;
}

static inline int64_t up_to(int64_t x, int64_t m) { return (x + m - 1) / m * m; }
static inline int64_t over(int64_t x, int64_t m) { return (x + m - 1) / m; }

// Workgroups of four wavefronts that are there at once: two on each compute unit.  With twice as many, which take turns, one sequence of 65000 keys took 62.2 us
// for 56.5 (workgroups that share a chunk of keys), and a batch of 64 behind 8192 shared keys 154 for 109.
constexpr int64_t kResident = 512;
constexpr int64_t kMostGroups = (int64_t)1 << 22;             // workgroups in x: far from the 2^32 threads that one launch may have there

// Keys that a workgroup takes, so that a launch over `keys` of them for `units` sequences, key heads and blocks of 128 rows or more fills the chip once.
static int64_t chunk_of(int64_t keys, int64_t units, int block, int64_t grid_units) {
    int64_t chunk = std::max(std::min(over(keys * units, block == 256 ? kResident / 2 : kResident), keys), (int64_t)256);
    if (keys / chunk > kMostGroups / grid_units) chunk = keys / std::max<int64_t>(kMostGroups / grid_units, 1) + 1;
    return up_to(chunk, 128);
}

size_t plan_attention(AttnArgs* a, size_t ws_bytes) {
    const int D = a->cache.head_dim, heads = a->cache.kv_heads;
    const int64_t rows = (int64_t)a->seqs.n_tokens * a->heads, notes = (int64_t)a->seqs.n_seqs * heads;
    const int64_t gap = rows % 2 ? 8 : 0;                     // after the maxima and sums, so that what follows is aligned
    const int64_t per_part = rows * (D + 2) * 4, room = (int64_t)std::min<size_t>(ws_bytes, (size_t)1 << 60) - 4 * up_to(notes, 4) - gap;
    const int64_t most = room > 0 ? room / per_part : 0;      // parts that the workspace holds
    const auto blocks = [&](int64_t tokens, int block) { return over(tokens * a->group, block); };
    const auto halves = [&](int block) { return D == 256 && block >= 128 ? 2 : 1; };      // workgroups of such a block
    const int block = rows_of_block((int64_t)a->seqs.max_q * a->group, D);
    const int64_t units = blocks(a->seqs.max_q, block) * heads * halves(block);
    a->few = block <= 32;
    a->prefix_parts = a->front_blocks = a->line_waves = 0;
    if (a->prefix > a->seqs.max_kv) a->prefix = a->seqs.max_kv;
    // Every sequence reads the shared keys as its own where it has to, and where blocks of 128 rows and more, for which reading keys is little of the work, fill
    // the chip without being cut: 32 pieces of 64 tokens, 8 key heads of 4 query heads, behind 2048 shared keys 100 us so, 211 in parts; 6 pieces of 200
    // tokens (192 workgroups) 130 and 109, 8 of 70 behind 8192 (128) 176 and 133.
    if (most < (a->few ? 3 : 2) || a->seqs.n_seqs < 2 || (!a->few && units * a->seqs.n_seqs >= 256)) a->prefix = 0;
    const bool line = a->few && (over(a->seqs.max_kv, 32) + 1) * notes < (int64_t)1 << 29;    // its steps are counted in 32 bits
    if (a->few && !line) a->prefix = 0;
    const int64_t own = a->seqs.max_kv - (a->prefix & ~63);
    const int front = a->few ? 128 : rows_of_block((int64_t)a->seqs.n_tokens * a->group, D);
    const int64_t front_units = blocks(a->seqs.n_tokens, front) * heads * halves(front);
    int64_t own_parts = 1;
    if (a->few) {
        const int64_t resident = kResident / 2 * rows_resident(D, block / 16);
        int64_t own_blocks = resident;
        if (a->prefix) {
            // What both cost in workgroups' time where all share the memory, in us: 64 keys for 128 rows of the front 3, 128 keys of a sequence 7, in e4m3 half of
            // that.  Taken at heads of 128 in bf16 and used for the other sizes too, as a ratio.  The longest sequence is all that the host knows, and the
            // others are taken to be half as long on the whole: right within a factor of two or so where max_kv is close to the lengths, and if it is far
            // beyond them the front has too few workgroups (64 sequences of up to 9000 tokens, 8192 shared, the same inputs each time: 47 us, and 238 with max_kv = 65536).
            const double f = 3.0 * front_units * over(a->prefix, 64), o = (a->cache.e4m3 ? 3.5 : 7.0) * 0.5 * notes * over(std::max<int64_t>(own, 1), 128);
            const int64_t share = (int64_t)(resident * f / (f + o));
            int64_t parts = std::max<int64_t>(over(share, front_units), 1);
            parts = std::min(std::min(parts, over(a->prefix, 128)), std::min(most - 2, std::max<int64_t>(kMostGroups / front_units, 1)));
            a->prefix_chunk = (int)up_to(over(a->prefix, parts), 128);
            a->prefix_parts = (int)over(a->prefix, a->prefix_chunk);
            a->front_blocks = (int)(a->prefix_parts * front_units);
            own_blocks = std::max<int64_t>(resident - a->front_blocks, resident / 4);
        }
        const int64_t longest = over(own, step_keys(D)), waves = 4 * own_blocks, wanted = std::max<int64_t>(waves / heads + 2, 4);
        // as many parts as one sequence of nearly all keys would be, if that is not beyond the workspace or 128 MB
        own_parts = std::min(std::min(most - a->prefix_parts, wanted), std::max<int64_t>(((int64_t)128 << 20) / per_part, 4));
        if (line && own_parts >= 2) {
            a->line_waves = (int)waves;
            a->least_steps = (int)std::max<int64_t>(over(longest, own_parts - 1), 1);      // a head in own_parts - 1 stretches' length is in own_parts of them at most
        } else {
            own_parts = 1;
        }
        a->own_chunk = (int)up_to(std::max<int64_t>(own, 1), 128);
    } else {
        int64_t chunk = chunk_of(own, units * a->seqs.n_seqs, block, units);
        if (a->prefix) {
            // what the sequences' own keys leave of the workspace, or half of it
            const int64_t share = std::max(most / 2, most - std::max<int64_t>(over(own, chunk), 1));
            int64_t shared_chunk = chunk_of(a->prefix, front_units, front, front_units);
            if (over(a->prefix, shared_chunk) > share) shared_chunk = up_to(over(a->prefix, share), 128);
            a->prefix_chunk = (int)shared_chunk;
            a->prefix_parts = (int)over(a->prefix, shared_chunk);
        }
        const int64_t left = most - a->prefix_parts;
        if (left < 2 && !a->prefix) chunk = up_to(std::max<int64_t>(own, 1), 128);
        else if (over(own, chunk) > left) chunk = up_to(over(own, left), 128);
        a->own_chunk = (int)chunk;
        own_parts = std::max<int64_t>(over(own, chunk), 1);
    }
    a->parts = (int)(a->prefix_parts + own_parts);
    if (a->parts == 1) return 0;
    float* at = a->part_ml + 2 * up_to(a->parts * rows, 2);
    a->part_o = at;
    a->unit_parts = reinterpret_cast<int*>(at + (int64_t)a->parts * rows * D);
    return (size_t)(a->parts * per_part + gap + 4 * up_to(notes, 4));
}

template <int D, int RB, bool E4M3>
static void launch_few(const AttnArgs& a, hipStream_t stream) {
    if (a.front_blocks) attend_few_kernel<D, RB, E4M3, true><<<(unsigned)(a.front_blocks + a.line_waves / 4), 256, 0, stream>>>(a);
    else if (a.line_waves) attend_few_kernel<D, RB, E4M3, false><<<(unsigned)(a.line_waves / 4), 256, 0, stream>>>(a);
    else attend_rows_kernel<D, RB, E4M3><<<(unsigned)(a.seqs.n_seqs * a.cache.kv_heads), 256, 0, stream>>>(a);
}

template <int D, int NW, bool E4M3>
static void launch_tiles(const AttnArgs& a, int front, hipStream_t stream) {
    const int tokens = front ? a.seqs.n_tokens : a.seqs.max_q, parts = front ? a.prefix_parts : a.parts - a.prefix_parts;
    const unsigned groups = (unsigned)(((int64_t)tokens * a.group + 32 * NW - 1) / (32 * NW));
    attend_tiles_kernel<D, NW, E4M3><<<dim3(parts * groups * (unsigned)a.cache.kv_heads * (D == 256 ? 2u : 1u), front ? 1u : (unsigned)a.seqs.n_seqs), 64 * NW, 0, stream>>>(a, front);
}

template <int D, bool E4M3>
static void launch_rows_of(const AttnArgs& a, hipStream_t stream) {
    if (a.few) {
        if (a.seqs.max_q * (int64_t)a.group <= 16) launch_few<D, 1, E4M3>(a, stream);
        else launch_few<D, D == 256 ? 1 : 2, E4M3>(a, stream);
        return;
    }
    for (int front = a.prefix_parts ? 1 : 0; front >= 0; --front) {
        const int block = rows_of_block((int64_t)(front ? a.seqs.n_tokens : a.seqs.max_q) * a.group, D);
        if (block <= 128) launch_tiles<D, 4, E4M3>(a, front, stream);
        else launch_tiles<D, 8, E4M3>(a, front, stream);
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
