// How much each cached token has been attended to (patch_attention_weights):
//
//   w_j' = decay w_j + sum_r exp(q_r . k_j scale - lse_r)        over a key head's rows r of the call that see key j
//
// lse is the attention's own, so a probability needs no pass over the keys before it, and every key's sum is one workgroup's: no order but that of the sizes.  The
// product is S = Q K^T with the rows on the matrix instruction's A side: a column, and so a lane, is a key, and the sum over rows stays in the lane but for its last step.
//
// A row whose lse is minus infinity is as one that is not there: it sees no key (its limit is 0), since its scores may be NaN, which no lse makes nothing of.
#include <algorithm>

#include "attention_kernels.h"

namespace patch {

constexpr int64_t kMostGroups = (int64_t)1 << 22;             // workgroups in x: far from the 2^32 threads that one launch may have there
constexpr float kLog2e = 1.4426950408889634f;

// what is written for key j of a sequence, whose head's weights begin at `weights`: `sum` is of the call's rows, `old` what was there for a key that is not new
__device__ __forceinline__ void put_weight(const WeighArgs& a, const Seq& q, int64_t weights, int j, float sum, float old) {
    if (j >= q.len) return;
    if (j < q.pos0) sum += a.decay * old;
    else if (a.slot_positions) as_global_out(a.slot_positions)[weights + j] = as_global(a.positions)[q.first + (j - q.pos0)];
    as_global_out(a.w_out)[weights + j] = sum;
}
__device__ __forceinline__ float key_scale(const WeighArgs& a, int cells, int kh) {
    return cells == kE4m3 && a.cache.k_scale ? a.scale * as_global(a.cache.k_scale)[kh] : a.scale;
}
__device__ __forceinline__ int page_of(const WeighArgs& a, int s, int key) {      // key: one that the sequence has
    return page_or_none(as_global(a.seqs.table)[s * a.seqs.table_stride + (key >> a.cache.page_log2)], a.cache.n_pages);
}

// Sixteen keys of a page as the second operand of D / 32 products of 16 x 16 x 32: lane: key, eight features (in the order of query_offset).
template <int D, int CELLS>
struct KeyTile {
    static constexpr int kLoads = CELLS == kBf16 ? D / 32 : CELLS == kE4m3 ? D / 64 : D < 128 ? 1 : D / 128;
    typedef typename std::conditional<CELLS == kE2m1 && D == 64, u32x2_t, u32x4_t>::type Load;
    Load k[kLoads];
    uint8_t power[kLoads];

    __device__ __forceinline__ void load(const CacheArgs& c, int page, int slot, int kh, int lane) {
        const int64_t token = ((int64_t)kh << c.page_log2) + slot + (lane & 15);
        constexpr int kBytes = CELLS == kBf16 ? 2 * D : CELLS == kE4m3 ? D : D / 2;
        const PATCH_EP_GLOBAL uint8_t* at = as_global(c.k) + page * c.page_bytes + token * kBytes + sizeof(Load) * (lane >> 4);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) k[i] = *reinterpret_cast<const PATCH_EP_GLOBAL Load*>(at + 64 * i);
        if constexpr (CELLS == kE2m1) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) power[i] = as_global(c.k_power)[page * c.power_bytes + token * (D / 32) + 4 * i + (D == 64 ? lane >> 5 : lane >> 4)];
        }
    }
    __device__ __forceinline__ bf16x8_t operand(int i) const {
        if constexpr (CELLS == kE2m1) return as_bf16x8(widen8_e2m1(k[i / 4][i % 4], power_of(power[i / 4])));
        else if constexpr (CELLS == kE4m3) return as_bf16x8(widen8(k[i / 2][2 * (i % 2)], k[i / 2][2 * (i % 2) + 1]));
        else return as_bf16x8(k[i]);
    }
};

// Few rows (16 RB at most): each wavefront has `steps` steps of 64 keys, straight from memory into the operands' registers, the next step's on their way.  Memory
// bounds it: 32 sequences of up to 8000 tokens, 8 key heads of 128 in 4 bits, 26.3 us, 3.9 TB/s (a large copy: 5.0); with a step's page numbers looked up when it is
// asked for 38, with branches around the loads of lse 27.6.
template <int D, int RB, int CELLS>
__global__ __launch_bounds__(256, 2) void weigh_few_kernel(const WeighArgs a, const int steps) {
    const int s = blockIdx.y, kh = blockIdx.x % a.cache.kv_heads, lane = threadIdx.x & 63, g = lane >> 4, col = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int begin = (blockIdx.x / a.cache.kv_heads * 4 + wave) * (steps * 64);
    const Seq q = seq_at(a.seqs, s);
    if (q.bad || q.n == 0 || begin >= q.len) return;
    const int end = min(q.len, begin + steps * 64), rows = min(q.n, a.seqs.max_q) * a.group, mask = (1 << a.cache.page_log2) - 1;
    const float scale = key_scale(a, CELLS, kh);
    bf16x8_t query[RB][D / 32];
    float lse[RB][4];
    int limit[RB][4];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        const int r = 16 * b + col;
        const int64_t at = r < rows ? (int64_t)(q.first + r / a.group) * a.q_stride + (int64_t)(kh * a.group + r % a.group) * D : 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            u32x4_t v = {0, 0, 0, 0};
            if (r < rows) v = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(a.Q) + at + query_offset<D, CELLS>(i, g));
            query[b][i] = as_bf16x8(v);
        }
        int token = (16 * b + 4 * g) / a.group, head = (16 * b + 4 * g) % a.group;
#pragma unroll
        for (int e = 0; e < 4; ++e) {                            // no branch: all of them on their way together
            const bool there = 16 * b + 4 * g + e < rows;
            const float l = as_global(a.lse)[(int64_t)(q.first + (there ? token : 0)) * a.heads + kh * a.group + head];
            lse[b][e] = l * kLog2e;
            limit[b][e] = there && l != kNone ? q.pos0 + token + 1 : 0;
            if (++head == a.group) {
                head = 0;
                ++token;
            }
        }
    }
    typedef KeyTile<D, CELLS> Tile;
    const int64_t weights = ((int64_t)s * a.cache.kv_heads + kh) * a.w_stride;
    // Pages of 64 times 16 keys, one a lane: a step's are known before it is asked for.
    for (int window = begin; window < end; window += 1024) {
        int ids = -1;
        if (window + 16 * lane < end) ids = page_of(a, s, window + 16 * lane);
        Tile keys[4];
        float old = 0.f;
        const auto ask = [&](int step) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int key = step + 16 * t;
                keys[t].load(a.cache, max(__builtin_amdgcn_readlane(ids, (key - window) >> 4), 0), key & mask, kh, lane);
            }
            if (step + lane < q.pos0) old = as_global(a.w)[weights + step + lane];
        };
        ask(window);
        const int stop = min(end, window + 1024);
        for (int step = window; step < stop; step += 64) {
            f32x4_t x[RB][4];
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int t = 0; t < 4; ++t) x[b][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const bf16x8_t k = keys[t].operand(i);
#pragma unroll
                    for (int b = 0; b < RB; ++b) x[b][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(query[b][i], k, x[b][t], 0, 0, 0);
                }
            const float was = old;
            if (step + 64 < stop) ask(step + 64);
            float mine = 0.f;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int key = step + 16 * t + col;
                float sum = 0.f;
                const float by = __builtin_amdgcn_readlane(ids, (step + 16 * t - window) >> 4) < 0 ? __builtin_nanf("") : scale;       // no page: NaN for whichever row sees the key
#pragma unroll
                for (int b = 0; b < RB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][t][e], by, -lse[b][e]));
                        sum += key < limit[b][e] ? p : 0.f;
                    }
                sum += __shfl_xor(sum, 16);
                sum += __shfl_xor(sum, 32);
                if (g == t) mine = sum;
            }
            put_weight(a, q, weights, step + lane, mine, was);
        }
    }
}

// 32 keys as the second operand of D / 16 products of 32 x 32 x 16, a key a lane; returns whether the lane's has a page.
template <int D, int CELLS>
__device__ __forceinline__ bool load_keys(bf16x8_t (&k)[D / 16], const WeighArgs& a, const Seq& q, int s, int kh, int key0) {
    const int lane = threadIdx.x & 63, h = lane >> 5, key = key0 + (lane & 31);
    int page = -1;
    if (key < q.len) page = page_of(a, s, key);
    const int64_t token = ((int64_t)kh << a.cache.page_log2) + (key & ((1 << a.cache.page_log2) - 1));
    const PATCH_EP_GLOBAL uint8_t* at = as_global(a.cache.k) + max(page, 0) * a.cache.page_bytes;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        const int64_t cell = token * D + 16 * i + 8 * h;
        if constexpr (CELLS == kBf16) {
            k[i] = as_bf16x8(*reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(at + 2 * cell));
        } else if constexpr (CELLS == kE4m3) {
            const u32x2_t w = *reinterpret_cast<const PATCH_EP_GLOBAL u32x2_t*>(at + cell);
            k[i] = as_bf16x8(widen8(w[0], w[1]));
        } else {
            const uint32_t w = *reinterpret_cast<const PATCH_EP_GLOBAL uint32_t*>(at + cell / 2);
            const uint32_t power = as_global(a.cache.k_power)[max(page, 0) * a.cache.power_bytes + cell / 32];
            k[i] = as_bf16x8(widen8_e2m1(w, power_of(power)));
        }
    }
    return page >= 0;
}

// In front of it a wavefront's lanes have written to LDS what its others read behind it, or read what the others write: the wavefront's operations there stay in
// this order by themselves, the compiler, for which a lane is a thread of its own, has to be told.
__device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Many rows and few keys: a workgroup has 32 keys, and its wavefronts take the rows 32 at a time in turn, straight from memory; their sums meet in LDS.
constexpr int wide_waves(int head_dim) { return head_dim == 256 ? 8 : 16; }       // as many as have registers for it

template <int D, int CELLS>
__device__ __forceinline__ void weigh_wide(const WeighArgs& a, int s, int kh, int key0) {
    constexpr int NW = wide_waves(D), kStep = 32 * NW;
    __shared__ alignas(16) float sh_lse[NW][32], sh_sum[NW][32];
    __shared__ alignas(16) int sh_limit[NW][32];
    const Seq q = seq_at(a.seqs, s);
    if (q.bad || q.n == 0 || key0 >= q.len) return;
    const int rows = min(q.n, a.seqs.max_q) * a.group, lane = threadIdx.x & 63, h = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    bf16x8_t k[D / 16];
    float scale = key_scale(a, CELLS, kh);
    if (!load_keys<D, CELLS>(k, a, q, s, kh, key0)) scale = __builtin_nanf("");       // for whichever row sees the key
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};
    // rows in front see none of the keys; a lane's row follows from the one kStep in front of it
    const int64_t first = ((int64_t)max(key0 - q.pos0, 0) * a.group & ~(int64_t)31) + 32 * wave;
    int token = (int)((first + col) / a.group), head = (int)((first + col) % a.group);
    bf16x8_t query[D / 16];
    float lse = 0.f;
    int limit = 0;
    const auto ask = [&](int r) {
        const bool there = r + col < rows;
        const int64_t at = (int64_t)(q.first + (there ? token : 0)) * a.q_stride + (int64_t)(kh * a.group + head) * D + 8 * h;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) query[i] = as_bf16x8(*reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(as_global(a.Q) + at + 16 * i));
        lse = as_global(a.lse)[(int64_t)(q.first + (there ? token : 0)) * a.heads + kh * a.group + head];
        limit = there ? q.pos0 + token + 1 : 0;
        head += kStep % a.group;
        token += kStep / a.group + (head >= a.group);
        head -= head >= a.group ? a.group : 0;
    };
    if (first < rows) ask((int)first);
    for (int r = (int)first; r < rows; r += kStep) {
        const int sees = lse == kNone ? 0 : limit;               // 0 also for rows that are not there
        lanes_meet();
        if (h == 0) {                                            // (of this wavefront's own)
            sh_lse[wave][col] = lse * kLog2e;
            sh_limit[wave][col] = sees;
        }
        lanes_meet();
        const bool ragged = __any(key0 + 32 > sees);
        f32x16_t x;
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(query[i], k[i], x, 0, 0, 0);
        if (r + kStep < rows) ask(r + kStep);
        const auto add = [&](auto masked) {
#pragma unroll
            for (int e4 = 0; e4 < 4; ++e4) {
                const f32x4_t l = *reinterpret_cast<const f32x4_t*>(&sh_lse[wave][8 * e4 + 4 * h]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[4 * e4 + e], scale, -l[e]));
                    if constexpr (decltype(masked)::value) p = key0 + col < sh_limit[wave][8 * e4 + 4 * h + e] ? p : 0.f;
                    sum[e] += p;
                }
            }
        };
        if (ragged) add(std::true_type{});
        else add(std::false_type{});
    }
    float w = sum[0] + sum[1] + (sum[2] + sum[3]);
    w += __shfl_xor(w, 32);
    if (h == 0) sh_sum[wave][col] = w;
    __syncthreads();
    if (threadIdx.x < 32) {
        w = 0.f;
#pragma unroll
        for (int i = 0; i < NW; ++i) w += sh_sum[i][col];
        const int64_t weights = ((int64_t)s * a.cache.kv_heads + kh) * a.w_stride;
        put_weight(a, q, weights, key0 + col, w, key0 + col < q.pos0 ? as_global(a.w)[weights + key0 + col] : 0.f);
    }
    __syncthreads();
}

template <int D, int CELLS>
__global__ __launch_bounds__(64 * wide_waves(D)) void weigh_wide_kernel(const WeighArgs a) {
    for (int64_t key = blockIdx.x / a.cache.kv_heads * 32; key < a.seqs.max_kv; key += gridDim.x / a.cache.kv_heads * 32)
        weigh_wide<D, CELLS>(a, blockIdx.y, blockIdx.x % a.cache.kv_heads, (int)key);
}

// Many rows: a workgroup's wavefronts have 32 keys each, in registers as operands, and the rows come through LDS for all of them, 64 at a time, the next ones
// on their way through registers meanwhile.  A prompt of 4096, 32 heads of 128: 96 us, 715 TFLOP/s; 101 with the products of 32 rows after those of the other 32 and
// operands left to the compiler.  Of those 101, 84 without its loads, 95 without exp2, 75 with a quarter of its products: no one of them bounds it, but the wait of
// all wavefronts for each other at each 64 rows.
template <int D>
struct RowTilesLds {
    u32x4_t q[2][64 * D / 8];
    float lse[2][64];
    int limit[2][64], out[2];             // the first key that a row does not see, 0 for one that adds nothing or is not there; whether there are such
};

template <int D, int NW, int CELLS>
__device__ __forceinline__ void weigh_tiles(const WeighArgs& a, int s, int kh, int block, RowTilesLds<D>& sh) {
    constexpr int kThreads = 64 * NW, kRowLoads = D / 8, kRowStep = kThreads / kRowLoads, kEach = 64 / kRowStep, kKeys = 32;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Seq q = seq_at(a.seqs, s);
    if (q.bad || q.n == 0 || block >= q.len) return;
    const int rows = min(q.n, a.seqs.max_q) * a.group, key0 = block + wave * kKeys;
    bf16x8_t k[D / 16];
    float scale = key_scale(a, CELLS, kh);
    if (!load_keys<D, CELLS>(k, a, q, s, kh, key0)) scale = __builtin_nanf("");       // for whichever row sees the key
    f32x4_t sum = {0.f, 0.f, 0.f, 0.f};

    const int row = tid / kRowLoads, chunk = tid % kRowLoads;
    // rows in front see none of the keys
    const int first = (int)((int64_t)max(block - q.pos0, 0) * a.group & ~(int64_t)63);
    // A row's place follows from that of the row 64 in front of it: so many elements, and if it is not in the same token's heads any more so many more.
    const int heads64 = 64 % a.group;
    const int64_t step = 64 / a.group * a.q_stride + heads64 * D, wrap = a.q_stride - (int64_t)a.group * D;
    int64_t at[kEach];
    int head[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int r = first + row + i * kRowStep;
        head[i] = r % a.group;
        at[i] = r / a.group * a.q_stride + head[i] * D;
    }
    const PATCH_EP_GLOBAL uint16_t* queries = as_global(a.Q) + (int64_t)q.first * a.q_stride + (int64_t)kh * a.group * D + 8 * chunk;
    // the first wavefront has their lse, too
    int lse_token = (first + lane) / a.group, lse_head = (first + lane) % a.group;
    // tokens of a tile's first row and of its 64th
    int low = __builtin_amdgcn_readlane(lse_token, 0), low_head = __builtin_amdgcn_readlane(lse_head, 0);
    int high = __builtin_amdgcn_readlane(lse_token, 63), high_head = __builtin_amdgcn_readlane(lse_head, 63);
    const int last = min(q.n, a.seqs.max_q) - 1;
    u32x4_t regs[kEach];
    float lse_reg = 0.f;
    int limit_reg = 0;
    const auto ask = [&](int tile) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            regs[i] = *reinterpret_cast<const PATCH_EP_GLOBAL u32x4_t*>(queries + (tile + row + i * kRowStep < rows ? at[i] : 0));     // (no row: any, its limit is 0)
            head[i] += heads64;
            at[i] += step + (head[i] >= a.group ? wrap : 0);
            head[i] -= head[i] >= a.group ? a.group : 0;
        }
        if (wave == 0) {
            const bool there = tile + lane < rows;
            lse_reg = as_global(a.lse)[(int64_t)(q.first + (there ? lse_token : 0)) * a.heads + kh * a.group + lse_head];
            limit_reg = there ? q.pos0 + lse_token + 1 : 0;
            lse_head += heads64;
            lse_token += 64 / a.group + (lse_head >= a.group);
            lse_head -= lse_head >= a.group ? a.group : 0;
        }
    };
    const auto put = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) sh.q[buffer][chunk_at<D / 8>(row + i * kRowStep, chunk)] = regs[i];
        if (wave == 0) {
            sh.lse[buffer][lane] = lse_reg * kLog2e;
            sh.limit[buffer][lane] = lse_reg == kNone ? 0 : limit_reg;
            sh.out[buffer] = __any(lse_reg == kNone || limit_reg == 0);
        }
    };
    if (first < rows) {
        ask(first);
        put(0);
    }
    // the keys are there before the loop: else the first products of each step wait for them, and so for the rows that were asked for since
    __builtin_amdgcn_s_waitcnt(0x0F70);
    __syncthreads();
    int buffer = 0;
    const auto forward = [&](int& token, int& head) {
        head += heads64;
        token += 64 / a.group + (head >= a.group);
        head -= head >= a.group ? a.group : 0;
    };
    for (int tile = first; tile < rows; tile += 64, buffer ^= 1) {
        const bool more = tile + 64 < rows;
        const int lowest = q.pos0 + low + 1, highest = q.pos0 + min(high, last) + 1;       // limits never fall from row to row, but for rows that are out
        forward(low, low_head);
        forward(high, high_head);
        if (more) ask(tile + 64);
        if (key0 < highest) {
            const int out = sh.out[buffer];
            f32x16_t both[2];
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int e = 0; e < 16; ++e) both[half][e] = 0.f;
            in_order<D / 8>([&](int j) { return as_bf16x8(sh.q[buffer][chunk_at<D / 8>(32 * (j % 2) + col, 2 * (j / 2) + h)]); },
                            [&](int j, bf16x8_t row) { both[j % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(row, k[j / 2], both[j % 2], 0, 0, 0); });
            const bool ragged = key0 + kKeys > lowest || __builtin_amdgcn_readfirstlane(out);       // not every row adds something and sees all of the keys
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const f32x16_t& x = both[half];
                const auto add = [&](auto masked) {
#pragma unroll
                    for (int e4 = 0; e4 < 4; ++e4) {
                        const int r = 32 * half + 8 * e4 + 4 * h;
                        const f32x4_t l = *reinterpret_cast<const f32x4_t*>(&sh.lse[buffer][r]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[4 * e4 + e], scale, -l[e]));
                            if constexpr (decltype(masked)::value) p = key0 + col < sh.limit[buffer][r + e] ? p : 0.f;
                            sum[e] += p;
                        }
                    }
                };
                if (ragged) add(std::true_type{});
                else add(std::false_type{});
            }
        }
        if (more) put(buffer ^ 1);
        __syncthreads();
    }
    float w = sum[0] + sum[1] + (sum[2] + sum[3]);
    w += __shfl_xor(w, 32);
    if (h != 0) return;
    const int64_t weights = ((int64_t)s * a.cache.kv_heads + kh) * a.w_stride;
    put_weight(a, q, weights, key0 + col, w, key0 + col < q.pos0 ? as_global(a.w)[weights + key0 + col] : 0.f);
}

template <int D, int NW, int CELLS>
__global__ __launch_bounds__(64 * NW, 2) void weigh_tiles_kernel(const WeighArgs a) {
    __shared__ RowTilesLds<D> sh;
    // the keys that most rows see come first
    for (int64_t block = blockIdx.x / a.cache.kv_heads * (32 * NW); block < a.seqs.max_kv; block += gridDim.x / a.cache.kv_heads * (32 * NW))
        weigh_tiles<D, NW, CELLS>(a, blockIdx.y, blockIdx.x % a.cache.kv_heads, (int)block, sh);
}

template <int D, int CELLS>
static void launch_weigh_of(const WeighArgs& a, hipStream_t stream) {
    const int64_t rows = (int64_t)a.seqs.max_q * a.group, units = (int64_t)a.seqs.n_seqs * a.cache.kv_heads;
    const unsigned heads = (unsigned)a.cache.kv_heads, seqs = (unsigned)a.seqs.n_seqs;
    // Heads of 256 have no registers for a second block of rows beside the keys.
    if (rows <= (D == 256 ? 16 : 32)) {
        const int64_t all = (a.seqs.max_kv + 63) / 64;
        const int64_t most = std::max<int64_t>(kMostGroups / heads, 1);             // workgroups of a head
        const int steps = (int)std::max(std::min<int64_t>(std::max<int64_t>(all * units / 2048, 1), 8), (all + 4 * most - 1) / (4 * most));
        const dim3 grid((unsigned)((all + 4 * steps - 1) / (4 * steps)) * heads, seqs);
        if (rows <= 16) weigh_few_kernel<D, 1, CELLS><<<grid, 256, 0, stream>>>(a, steps);
        else if constexpr (D != 256) weigh_few_kernel<D, 2, CELLS><<<grid, 256, 0, stream>>>(a, steps);
        return;
    }
    const auto blocks = [&](int keys) { return (unsigned)std::min<int64_t>((a.seqs.max_kv + keys - 1) / keys, std::max<int64_t>(kMostGroups / heads, 1)) * heads; };
    constexpr int NW = 4;
    // Where blocks of 128 keys do not fill the chip, or leave it to the first keys' (which all rows see) for half of the time: one prompt of 2048 tokens, 16 query heads
    // over 1 of 128, 621 us so and 230 with the rows dealt to wavefronts, 32 over 8 160 and 74; of 4096 tokens, 32 over 8 (256 blocks, 16384 rows), 318 and 261, but
    // of 1000 tokens, 32 over 32 (256 blocks, 1000 rows), 23.5 and 38.
    const int64_t groups = (int64_t)blocks(32 * NW) * seqs;
    if (groups < 128 || (groups <= 256 && rows >= 4096))
        weigh_wide_kernel<D, CELLS><<<dim3(blocks(32), seqs), 64 * wide_waves(D), 0, stream>>>(a);
    else
        weigh_tiles_kernel<D, NW, CELLS><<<dim3(blocks(32 * NW), seqs), 64 * NW, 0, stream>>>(a);
}
template <int CELLS>
static void launch_weigh_cells(const WeighArgs& a, hipStream_t stream) {
    if (a.cache.head_dim == 64) launch_weigh_of<64, CELLS>(a, stream);
    else if (a.cache.head_dim == 128) launch_weigh_of<128, CELLS>(a, stream);
    else launch_weigh_of<256, CELLS>(a, stream);
}
void launch_weigh(const WeighArgs& a, hipStream_t stream) {
    if (a.cache.cells == kE2m1) launch_weigh_cells<kE2m1>(a, stream);
    else if (a.cache.cells == kE4m3) launch_weigh_cells<kE4m3>(a, stream);
    else launch_weigh_cells<kBf16>(a, stream);
}

}  // namespace patch
