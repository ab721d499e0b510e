// How an attention call's keys are split over workgroups, what joins the parts, and its launches for cells of 16 and 8 bits.
#include <algorithm>

#include "attention_kernels.h"

namespace patch {

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
            // that.  Taken at heads of 128 in bf16 and used for the other sizes too, as a ratio, and e4m3's for 4-bit cells.  The longest sequence is all that the host knows, and the
            // others are taken to be half as long on the whole: right within a factor of two or so where max_kv is close to the lengths, and if it is far
            // beyond them the front has too few workgroups (64 sequences of up to 9000 tokens, 8192 shared, the same inputs each time: 47 us, and 238 with max_kv = 65536).
            const double f = 3.0 * front_units * over(a->prefix, 64), o = (a->cache.cells == kBf16 ? 7.0 : 3.5) * 0.5 * notes * over(std::max<int64_t>(own, 1), 128);
            const int64_t share = (int64_t)(resident * f / (f + o));
            int64_t parts = std::max<int64_t>(over(share, front_units), 1);
            parts = std::min(std::min(parts, over(a->prefix, 128)), std::min(most - 2, std::max<int64_t>(kMostGroups / front_units, 1)));
            a->prefix_chunk = (int)up_to(over(a->prefix, parts), 128);
            a->prefix_parts = (int)over(a->prefix, a->prefix_chunk);
            a->front_blocks = (int)(a->prefix_parts * front_units);
            own_blocks = std::max<int64_t>(resident - a->front_blocks, resident / 4);
        }
        const int64_t longest = over(own, step_keys(D, a->cache.cells)), waves = 4 * own_blocks, wanted = std::max<int64_t>(waves / heads + 2, 4);
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

template <int D>
static void launch_merge(const AttnArgs& a, hipStream_t stream) {
    attend_merge_kernel<D><<<dim3((unsigned)a.seqs.n_tokens, (unsigned)a.heads), 256, 0, stream>>>(a);
}

void launch_attention(const AttnArgs& a, hipStream_t stream) {
    if (a.cache.cells == kE2m1) launch_attention4(a, stream);
    else if (a.cache.cells == kE4m3) launch_cells<kE4m3>(a, stream);
    else launch_cells<kBf16>(a, stream);
    if (a.parts == 1) return;
    if (a.cache.head_dim == 64) launch_merge<64>(a, stream);
    else if (a.cache.head_dim == 128) launch_merge<128>(a, stream);
    else launch_merge<256>(a, stream);
}

}  // namespace patch
