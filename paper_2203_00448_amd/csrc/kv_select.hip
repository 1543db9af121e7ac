// Blocks of the 8-bit key/value cache selected for each row and key head.
//
// The score of a block is a product of 8-bit codes (the query's, made here, and the
// block's mean, kept by the write), so it is a whole number below 2^23 times powers of
// two: exact in 32 bits whatever the order of its sum, and the selection is one of exact
// numbers, the lowest index among equals.
#include "kv.hpp"
#include "internal.hpp"

namespace mp {

namespace {

constexpr int kThreads = 256;

// A row and key head of the launch: its sequence and its last position.
struct SelectRow {
    KvSeq q;
    int32_t blocks;  // p / block + 1, or 0 for a row that sees nothing
    bool ok;
};

__device__ __forceinline__ SelectRow select_row(const KvSelect& k, int64_t token) {
    const KvArgs& a = k.a;
    SelectRow r;
    int64_t s = token;
    if (a.s.begin) s = kv_find(a.s.n_seqs, token, [&](int64_t i) { return a.s.begin[i]; });
    r.q = kv_seq(a, s);
    const int64_t i = token - r.q.begin;
    r.ok = r.q.ok && i >= 0 && i < r.q.n;
    const int32_t last = r.q.length - r.q.n + (int32_t)i;
    r.blocks = r.ok && last >= 0 ? (last >> a.log_block) + 1 : 0;
    return r;
}

// Scores of 256 blocks for one row and key head, a block a thread: the block's mean is read
// once and multiplied by the codes of every query head, which lie in LDS.
__global__ __launch_bounds__(kThreads) void kv_score_kernel(KvSelect k, int32_t per_row) {
    extern __shared__ __align__(16) uint32_t codes[];  // [group][dim / 4], then group scales
    const KvArgs& a = k.a;
    const int dim = a.c.dim, words = dim / 4, tid = threadIdx.x, lane = tid & 63;
    float* const scales = reinterpret_cast<float*>(codes + k.group * words);
    if (blockIdx.x == 0) kv_check_begin(a);
    const int64_t row = blockIdx.x / per_row;
    const int64_t token = row / a.c.heads;
    const int head = (int)(row % a.c.heads);
    const SelectRow r = select_row(k, token);
    const int32_t b0 = (int32_t)(blockIdx.x % per_row) * kThreads;
    const int32_t lo = k.first, hi = r.blocks - k.recent;  // the blocks that are scored
    if (!r.ok || r.blocks <= k.keep || b0 >= hi || b0 + kThreads <= lo) return;
    // query codes: a wave for each head, eight dims a lane
    for (int g = tid >> 6; g < k.group; g += kThreads / kWave) {
        float x[8], top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 0.0f;
        if (lane * 8 < dim) load8(k.q, token, head * k.group + g, lane * 8, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = fabsf(x[i]);
            if (v < INFINITY) top = fmaxf(top, v);
        }
        top = wave_reduce(top, OpMax<float>());
        uint32_t frac;
        const int e = max(-100, exponent_of(top, &frac));
        const float f = pow2f(7 - e);
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float y = x[i] * f;
            const float c = y != y ? 0.0f : fminf(127.0f, fmaxf(-127.0f, __builtin_rintf(y)));
            w[i / 4] |= ((uint32_t)(int)c & 0xffu) << (8 * (i % 4));
        }
        if (lane * 8 < dim) {
            codes[g * words + lane * 2] = w[0];
            codes[g * words + lane * 2 + 1] = w[1];
        }
        if (lane == 0) scales[g] = pow2f(max(-126, e - 7));
    }
    __syncthreads();
    const int32_t b = b0 + tid;
    if (b < lo || b >= hi) return;
    int32_t page = a.s.table[r.q.s * a.s.table_stride + b];
    if (page < 0 || page >= a.c.n_blocks) {
        raise_status(a.status, MP_EINVAL);
        page = 0;
    }
    const int64_t at = (int64_t)page * a.c.heads + head;
    const uint2* mean = reinterpret_cast<const uint2*>(a.c.mean_code + at * dim);
    float best = -INFINITY;
    for (int g = 0; g < k.group; ++g) {
        int dot = 0;
        for (int i = 0; i < words / 2; ++i) {
            const uint2 w = mean[i];
            dot = __builtin_amdgcn_sdot4((int)w.x, (int)codes[g * words + 2 * i], dot, false);
            dot = __builtin_amdgcn_sdot4((int)w.y, (int)codes[g * words + 2 * i + 1], dot, false);
        }
        best = fmaxf(best, (float)dot * scales[g]);
    }
    k.scores[row * k.score_stride + b] = best * pow2f(max(-126, (int)a.c.mean_exp[at]));
}

// Larger scores to larger keys.
__device__ __forceinline__ uint32_t key_of(float score) {
    const uint32_t b = __float_as_uint(score + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The selection of one row and key head: the key of the last one taken by four passes of
// eight bits, then one pass that writes the taken blocks in order.
__global__ __launch_bounds__(kThreads) void kv_pick_kernel(KvSelect k) {
    __shared__ uint32_t hist[256];
    __shared__ int32_t scratch[kThreads / kWave];
    __shared__ uint32_t found_digit, found_left;
    const KvArgs& a = k.a;
    const int tid = threadIdx.x;
    if (blockIdx.x == 0) kv_check_begin(a);
    const int64_t row = blockIdx.x;
    const SelectRow r = select_row(k, row / a.c.heads);
    int32_t* const out = k.out + row * k.keep;
    if (r.blocks <= k.keep) {
        for (int i = tid; i < k.keep; i += kThreads) out[i] = i < r.blocks ? i : -1;
        return;
    }
    const float* const score = k.scores + row * k.score_stride;
    const int32_t lo = k.first, hi = r.blocks - k.recent;
    uint32_t want = (uint32_t)(k.keep - k.first - k.recent), prefix = 0;
    for (int shift = 24; want > 0 && shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int32_t b = lo + tid; b < hi; b += kThreads) {
            const uint32_t key = key_of(score[b]);
            if (shift == 24 || key >> (shift + 8) == prefix >> (shift + 8))
                atomicAdd(&hist[key >> shift & 255u], 1u);
        }
        __syncthreads();
        // keys of larger digits come first: this thread's digit is 255 - tid
        int32_t total;
        const uint32_t mine = hist[255 - tid];
        const uint32_t before = (uint32_t)block_exclusive_sum<kThreads>((int32_t)mine, &total, scratch);
        if (before < want && want <= before + mine) {
            found_digit = 255u - tid;
            found_left = want - before;
        }
        __syncthreads();
        prefix |= found_digit << shift;
        want = found_left;
        __syncthreads();
    }
    // all keys above `prefix`, and the first `want` of those equal to it
    const bool any = k.keep > k.first + k.recent;
    int32_t at = 0, ties = 0;
    for (int32_t b0 = 0; b0 < r.blocks; b0 += kThreads) {
        const int32_t b = b0 + tid;
        bool take = b < r.blocks && (b < lo || b >= hi), tie = false;
        if (any && b >= lo && b < hi) {
            const uint32_t key = key_of(score[b]);
            take = key > prefix;
            tie = key == prefix;
        }
        int32_t n_ties, n_take;
        const int32_t rank = ties + block_exclusive_sum<kThreads>((int32_t)tie, &n_ties, scratch);
        take |= tie && rank < (int32_t)want;
        const int32_t place = at + block_exclusive_sum<kThreads>((int32_t)take, &n_take, scratch);
        if (take && place < k.keep) out[place] = b;
        ties += n_ties;
        at += n_take;
    }
}

}  // namespace

size_t kv_select_workspace(const mp_kv_cache& c, const mp_kv_seqs& s, int64_t* score_stride) {
    const int64_t most = (s.longest + c.block - 1) / c.block;
    *score_stride = (most + 3) / 4 * 4;
    return (size_t)s.n_tokens * c.heads * *score_stride * sizeof(float);
}

hipError_t launch_kv_select(const KvSelect& k, hipStream_t st) {
    const int64_t rows = k.a.s.n_tokens * k.a.c.heads;
    if (rows == 0) return hipSuccess;
    const int64_t per_row = (k.score_stride + kThreads - 1) / kThreads;
    if (k.score_stride > k.keep) {
        const size_t lds = (size_t)k.group * (k.a.c.dim + 4);
        kv_score_kernel<<<dim3((uint32_t)(rows * per_row)), kThreads, lds, st>>>(k, (int32_t)per_row);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    kv_pick_kernel<<<dim3((uint32_t)rows), kThreads, 0, st>>>(k);
    return hipGetLastError();
}

}  // namespace mp
