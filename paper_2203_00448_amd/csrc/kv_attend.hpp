// What the attention kernels of all cache formats share: the rows of a workgroup, the pages of a
// sequence, the partial results of chunks.
#pragma once

#include "kv.hpp"

namespace mp {

// The chunks of each row of a launch joined (kv_attend.hip).
hipError_t launch_kv_join(const KvAttend& k, hipStream_t st);

// Attention over the cache in 4 bits (kv4_attend.hip).
hipError_t launch_kv4_attend(const KvAttend& k, hipStream_t st);

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// The partial result of a row over a chunk of tokens: its weighted values, 2^(maximum + power) of
// them; the maximum of its weights' exponents, the sum of its weights below that, the power.  (One
// logarithm of maximum and sum would lose the sum beside a large maximum; values at their own size
// and weights at theirs could both leave the range of 32-bit floats where their product does not.)
struct Partials {
    float* o;        // [row][chunk][dim]
    float4_t* sums;  // [row][chunk]: maximum, sum, power
};

__device__ __forceinline__ Partials partials(const KvAttend& k) {
    const int64_t rows = k.a.s.n_tokens * (int64_t)k.group * k.a.c.heads * k.shape.n_chunks;
    Partials p;
    p.o = static_cast<float*>(k.ws);
    p.sums = reinterpret_cast<float4_t*>(p.o + rows * k.a.c.dim);
    return p;
}

// The rows [row0, ...) of a workgroup: rows of a sequence and key head are (token, query
// head) pairs in token order.
struct RowGroup {
    KvSeq q;
    int64_t row0;
    int32_t n_rows;  // of the sequence
};

// Row group `u` (of ROWS rows) of the launch.  With a block list every token is a sequence of its own.  Groups are fewer
// than 2^31, and the quotients in 32 bits and by a constant: in 64 they are a good part of a short call's time.
template <int ROWS>
__device__ __forceinline__ bool row_group(const KvAttend& k, uint32_t u, RowGroup* g) {
    const KvArgs& a = k.a;
    const uint32_t per = ((uint32_t)k.group + ROWS - 1) / ROWS;
    const uint32_t whole = per == 1 ? u : u / per;
    if (k.blocks) {
        const int64_t token = whole;
        int64_t i;
        g->q = kv_find(a, token, [&](int64_t b, int64_t) { return b; }, &i);
        if (!g->q.ok || i < 0 || i >= g->q.n) return false;
        // the sequence as it is for this token: its last one
        g->q.length -= (int32_t)(g->q.n - 1 - i);
        g->q.begin = token;
        g->q.n = 1;
        g->row0 = (int64_t)(u - whole * per) * ROWS;
    } else {
        int64_t first;
        if (a.s.begin) {
            // n tokens are at most n * group / rows + 1 row groups
            auto key = [&](int64_t b, int64_t i) { return b * k.group / ROWS + i; };
            g->q = kv_find(a, u, key, &first);
        } else {
            g->q = wave_one(kv_seq(a, whole, whole, (int64_t)whole + 1));
            first = u - whole * per;
        }
        if (!g->q.ok || first < 0) return false;
        g->row0 = first * ROWS;
    }
    const int64_t n = (int64_t)g->q.n * k.group;
    if (g->row0 >= n) return false;
    g->n_rows = (int32_t)n;
    return true;
}

// The place of a row: its token, its query head, the last position it sees (-1: none).
struct Row {
    int64_t token;
    int32_t head;
    int32_t last;
    bool live;
};
__device__ __forceinline__ Row row_of(const KvAttend& k, const RowGroup& g, int key_head,
                                      int64_t row) {
    Row r;
    r.live = row < g.n_rows;
    const int32_t i = r.live ? (int32_t)row : g.n_rows - 1;
    const int32_t t = i / k.group;
    r.token = g.q.begin + t;
    r.head = key_head * k.group + i % k.group;
    r.last = r.live ? max(-1, g.q.length - g.q.n + t) : -1;
    return r;
}

// The pages of a sequence as its blocks are walked: entries of its table row, kept within the
// row's last used block and the pool.
struct Pages {
    const int32_t* table;
    uint32_t last_block, n_blocks;
    uint32_t worst;  // the largest entry met
    __device__ __forceinline__ uint32_t entry(uint32_t block) const {
        return (uint32_t)table[min(block, last_block)];
    }
    __device__ __forceinline__ uint32_t page(uint32_t e) {
        worst = max(worst, e);
        return min(e, n_blocks - 1);
    }
    __device__ __forceinline__ bool bad() const { return worst >= n_blocks; }
};

// The sum of x over the wave.
__device__ __forceinline__ int wave_sum(int x) {
    const auto from = [](int v, auto dpp, auto rows) {
        return __builtin_amdgcn_update_dpp(0, v, decltype(dpp)::value, decltype(rows)::value, 0xf, false);
    };
    using All = std::integral_constant<int, 0xf>;
    x += from(x, std::integral_constant<int, 0x111>(), All());  // up by 1, 2, 4, 8 in rows of 16
    x += from(x, std::integral_constant<int, 0x112>(), All());
    x += from(x, std::integral_constant<int, 0x114>(), All());
    x += from(x, std::integral_constant<int, 0x118>(), All());
    x += from(x, std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xa>());  // row 0 to 1, 2 to 3
    x += from(x, std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xc>());  // half to half
    return __builtin_amdgcn_readlane(x, 63);
}

// Row group `u` of a launch of tiles: those that see the most first, so that the last ones to
// start are short.  A lane has a sequence; group j of a sequence is at level (earlier tokens in
// groups) + j, and u counts down the levels, sequences in order within one.  Where they are
// not ordered (more than 64 sequences, chunks, levels past 30 bits), the last sequences' last
// groups come first.  Prompts of 228-4096 tokens: 273 us, 286 without the order; in chunks it gained
// nothing.
template <int ROWS>
__device__ __forceinline__ bool tile_group(const KvAttend& k, uint32_t u, RowGroup* g) {
    const KvArgs& a = k.a;
    if (!k.shape.ordered) return row_group<ROWS>(k, (uint32_t)k.shape.units - 1 - u, g);
    const int lane = threadIdx.x & 63;
    KvSeq q = {};
    if (lane < a.s.n_seqs) q = kv_seq(a, lane, a.s.begin[lane], a.s.begin[lane + 1]);
    const bool some = lane < a.s.n_seqs && q.ok && q.n > 0;
    const int count = some ? (int)(((uint64_t)q.n * (uint32_t)k.group + ROWS - 1) / ROWS) : 0;
    const int low = some ? (int)((uint64_t)max(0, q.length - q.n) * (uint32_t)k.group / ROWS) : 0;
    if (u >= (uint32_t)wave_sum(count)) return false;
    // the least level that at most u groups are above
    const auto above = [&](int level) { return (uint32_t)wave_sum(min(count, max(0, low + count - 1 - level))); };
    int from = 0, to = wave_reduce(low + count, OpMax<int>());
    while (from < to) {
        const int level = (from + to) >> 1;
        if (above(level) <= u)
            to = level;
        else
            from = level + 1;
    }
    const int nth = (int)(u - above(from));
    const bool member = some && from >= low && from < low + count;
    const uint64_t members = __ballot(member);
    const int rank = __popcll(members & (((uint64_t)1 << lane) - 1));
    const int of = __ffsll((unsigned long long)__ballot(member && rank == nth)) - 1;
    g->q.s = of;
    g->q.length = __builtin_amdgcn_readlane(q.length, of);
    g->q.n = __builtin_amdgcn_readlane(q.n, of);
    g->q.begin = wave_one(__shfl(q.begin, of, kWave));
    g->q.ok = true;
    g->row0 = (int64_t)(from - __builtin_amdgcn_readlane(low, of)) * ROWS;
    g->n_rows = g->q.n * k.group;
    return true;
}

}  // namespace

}  // namespace mp
