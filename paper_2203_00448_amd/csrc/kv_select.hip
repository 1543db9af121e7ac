// Blocks of the 8-bit key/value cache selected for each row and key head.
//
// The score of a block is a product of 8-bit codes (the query's, made here, and the
// block's mean, kept by the write), so it is a whole number below 2^22 times powers of
// two: exact whatever the order of its sum, and the selection is one of exact numbers,
// the lowest index among equals.  Only the order of a row's scores counts: they are held 2^(13 + x)
// times too small, x the largest exponent of the key head's queries, which 32-bit floats hold
// for keys of any size, the least of them as subnormal ones.
//
// One launch: a workgroup takes one key head and a few consecutive tokens of a sequence,
// reads each block's mean once for all of them and keeps their scores in LDS; then each
// wave selects for one token after the other.  Bytes read are a 1 / (2 block) part of the
// cache's; what bounds a call of few tokens is the chain of dependent steps.  16 sequences of up to
// 1024 blocks, one token each, 8 heads: 16 us, of it query codes 2, scores 7, selection 5; 353 tokens of
// up to 386 blocks, 4 heads: 18 us.
#include "kv.hpp"

namespace mp {

namespace {

typedef int int4_t __attribute__((ext_vector_type(4)));
typedef int4_t mean4_t __attribute__((aligned(8)));  // as the means are: 8 bytes

constexpr int kMostTokens = 8;        // of a workgroup
constexpr int kLdsScores = 16 * 1024;  // scores that a workgroup holds in LDS
constexpr int kNoQuery = -10000;      // the exponent of a query of zeros
constexpr int kDown = -20;            // of scores below 2^(22 + 124)

// Larger scores to larger keys.
__device__ __forceinline__ uint32_t key_of(float score) {
    const uint32_t b = __float_as_uint(score + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The largest of a value over aligned groups of `span` lanes (1, 2, 4, 8 or 16), to all of them.
__device__ __forceinline__ float span_max(float x, int span) {
    const auto from = [](float v, auto dpp) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(dpp)::value,
                                                          0xf, 0xf, true));
    };
    if (span > 1) x = fmaxf(x, from(x, std::integral_constant<int, 0xb1>()));   // pairs exchanged
    if (span > 2) x = fmaxf(x, from(x, std::integral_constant<int, 0x4e>()));   // quads' halves
    if (span > 4) x = fmaxf(x, from(x, std::integral_constant<int, 0x141>()));  // eight mirrored
    if (span > 8) x = fmaxf(x, from(x, std::integral_constant<int, 0x140>()));  // sixteen mirrored
    return x;
}

// LDS of a selection by WAVES waves: a histogram for each pass, and two turns' counts.
template <int WAVES>
struct PickLds {
    uint32_t hist[4][256];
    uint32_t sure[2][WAVES], tied[2][WAVES];
};

// The selection for one token by WAVES waves: `scores` of blocks [0, blocks), those of [lo, hi)
// valid.  The key of the last block taken by passes of eight bits over a histogram, then one
// pass that writes the taken blocks in order.
template <int WAVES>
__device__ __forceinline__ void pick(const float* scores, int32_t blocks, int32_t lo, int32_t hi,
                                     int32_t want, PickLds<WAVES>* lds, int32_t* out) {
    const auto meet = []() {
        if (WAVES > 1)
            __syncthreads();
        else
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    };
    const int lane = threadIdx.x & 63, wave = WAVES > 1 ? threadIdx.x >> 6 : 0;
    const int me = wave * kWave + lane;
    const bool any = want > 0;
    uint32_t prefix = 0;
    uint32_t left = (uint32_t)want;
    if (any) {
        for (int i = me; i < 256; i += WAVES * kWave)
            *reinterpret_cast<uint4*>(&lds->hist[0][0] + i * 4) = make_uint4(0, 0, 0, 0);
        meet();
    }
    for (int shift = 24; any && shift >= 0; shift -= 8) {
        uint32_t* const hist = lds->hist[shift >> 3];
        for (int32_t b = lo + me; b < hi; b += WAVES * kWave) {
            const uint32_t key = key_of(scores[b]);
            if (shift == 24 || (key ^ prefix) >> (shift + 8) == 0)
                atomicAdd(&hist[key >> shift & 255u], 1u);
        }
        meet();
        // keys of larger digits come first: this lane's digits are 255 - 4 lane and the next three
        const uint4 c = *reinterpret_cast<const uint4*>(hist + 252 - lane * 4);
        const uint32_t mine = c.x + c.y + c.z + c.w;
        const uint32_t before = wave_inclusive_sum(mine) - mine;
        const int at = __ffsll((unsigned long long)__ballot(before < left && left <= before + mine)) - 1;
        const auto of = [&](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, at); };
        const uint32_t four[3] = {of(c.w), of(c.z), of(c.y)};
        left -= of(before);
        uint32_t digit = 255u - 4u * (uint32_t)at;
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (left > four[i] && digit == 255u - 4u * (uint32_t)at - i) {
                left -= four[i];
                --digit;
            }
        prefix |= digit << shift;
    }
    // all keys above `prefix`, and the first `left` of those equal to it
    uint32_t at = 0, ties = 0;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    int turn = 0;
    for (int32_t b0 = 0; b0 < blocks; b0 += WAVES * kWave, turn ^= 1) {
        const int32_t b = b0 + me;
        bool sure = b < blocks && (b < lo || b >= hi), tie = false;
        if (any && b >= lo && b < hi) {
            const uint32_t key = key_of(scores[b]);
            sure = key > prefix;
            tie = key == prefix;
        }
        const uint64_t tied = __ballot(tie), sures = __ballot(sure);
        uint32_t my_at = at, my_ties = ties, all = __popcll(sures), all_ties = __popcll(tied);
        if (WAVES > 1) {
            // what the waves before this one take of this turn, and all of them
            if (lane == 0) lds->sure[turn][wave] = all, lds->tied[turn][wave] = all_ties;
            __syncthreads();
            const uint32_t s = lane < WAVES ? lds->sure[turn][lane] : 0;
            const uint32_t t = lane < WAVES ? lds->tied[turn][lane] : 0;
            const uint32_t t_before = wave_inclusive_sum(t) - t;
            const uint32_t room = left > ties + t_before ? left - ties - t_before : 0;
            const uint32_t taken = s + min(t, room), to = wave_inclusive_sum(taken);
            my_at += (uint32_t)__builtin_amdgcn_readlane((int)(to - taken), wave);
            my_ties += (uint32_t)__builtin_amdgcn_readlane((int)t_before, wave);
            all = (uint32_t)__builtin_amdgcn_readlane((int)to, WAVES - 1);
            all_ties = (uint32_t)__builtin_amdgcn_readlane((int)(t_before + t), WAVES - 1);
        }
        const bool take = sure || (tie && my_ties + (uint32_t)__popcll(tied & below) < left);
        const uint64_t takes = __ballot(take);
        if (take) out[my_at + __popcll(takes & below)] = b;
        at += WAVES > 1 ? all : (uint32_t)__popcll(takes);
        ties += all_ties;
    }
}

// LDS: query codes [tokens][rows][dim] with rows padded by 16 bytes, their exponents, the
// histograms of the waves, and the scores unless they are in the workspace (GLOBAL).
//
// Scores by matrix instructions of 16 blocks x 16 query heads x 64 dims, the heads of as many
// tokens as fit (`span` columns each, heads repeated to a power of two): a lane holds 16 dims of
// a block's mean and of a head's codes, and gets four blocks' products with one head; the
// largest over a token's heads is over a span of lanes.
template <int D, int THREADS, bool GLOBAL>
__global__ __launch_bounds__(THREADS) void kv_select_kernel(KvSelect k) {
    extern __shared__ __align__(16) char lds_raw[];
    constexpr int DC = D / 64, PER_ROW = D / 8, ROW = D + 16;
    // waves that select for a token: all where there is one token
    constexpr int kTeam = THREADS == 1024 ? THREADS / kWave : 1;
    const KvArgs& a = k.a;
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (blockIdx.x == 0) kv_check_begin(a);
    const uint32_t heads = a.c.heads;
    const int head = (int)(blockIdx.x % heads);
    const int64_t u = blockIdx.x / heads;
    // n tokens are at most n / tokens + 1 groups
    int64_t j;
    const KvSeq q = kv_find(a, u, [&](int64_t b, int64_t i) { return b / k.tokens + i; }, &j);
    if (!q.ok || j < 0 || j * k.tokens >= q.n) return;
    const int32_t i0 = (int32_t)j * k.tokens, count = min(k.tokens, q.n - i0);
    // blocks of token t of this group: of its position / block + 1, or none
    auto blocks_of = [&](int t) {
        const int32_t last = q.length - q.n + i0 + t;
        return last >= 0 ? (last >> a.log_block) + 1 : 0;
    };
    const int32_t most = blocks_of(count - 1);
    int8_t* const codes = reinterpret_cast<int8_t*>(lds_raw);
    int* const q_exps = reinterpret_cast<int*>(codes + (size_t)k.tokens * k.group * ROW);
    PickLds<kTeam>* const picks = reinterpret_cast<PickLds<kTeam>*>(q_exps + (k.tokens * k.group + 3) / 4 * 4);
    __shared__ int tops[kMostTokens];  // the largest of a token's
    float* const scores = GLOBAL ? k.scores + ((q.begin + i0) * heads + head) * k.score_stride
                                 : reinterpret_cast<float*>(picks + THREADS / kWave / kTeam);
    const int64_t step = GLOBAL ? heads * k.score_stride : k.score_stride;  // to the next token's

    if (most > k.keep) {
        if (tid < count) tops[tid] = kNoQuery;
        __syncthreads();
        // query codes, eight dims a lane
        const int rows = count * k.group, row_in = tid / PER_ROW, d = tid % PER_ROW * 8;
        for (int r0 = 0; r0 < rows; r0 += THREADS / PER_ROW) {
            const int r = min(r0 + row_in, rows - 1);
            float x[8], top = 0.0f;
            to_float8(k.q, load8_16bit(k.q, q.begin + i0 + r / k.group, head * k.group + r % k.group, d), x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = fabsf(x[i]);
                if (v < INFINITY) top = fmaxf(top, v);
            }
#pragma unroll
            for (int o = PER_ROW / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
            const int e = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : kNoQuery;
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = __builtin_amdgcn_ldexpf(x[i], 7 - e);
                const float c = y != y ? 0.0f : fminf(127.0f, fmaxf(-127.0f, __builtin_rintf(y)));
                w[i / 4] |= ((uint32_t)(int)c & 0xffu) << (8 * (i % 4));
            }
            *reinterpret_cast<uint2*>(codes + r * ROW + d) = make_uint2(w[0], w[1]);
            if (d == 0) {
                q_exps[r] = e;
                atomicMax(&tops[r / k.group], e);
            }
        }
        __syncthreads();
        const int32_t lo = k.first, hi = most - k.recent;  // the blocks that some token has scored
        const int32_t* const table = a.s.table + q.s * a.s.table_stride;
        const int columns = (k.group + 15) / 16;
        int span = 1;
        while (span < 16 && span < k.group) span *= 2;
        // 64 blocks a turn: their table entries are read a turn ahead, all their means at once
        constexpr int kStep = THREADS / kWave * 64;
        int32_t entry[4];
        auto find = [&](int32_t b0) {
#pragma unroll
            for (int z = 0; z < 4; ++z) entry[z] = table[min(b0 + z * 16 + n, most - 1)];
        };
        const int32_t from = (lo & ~15) + wave * 64;
        if (from < hi) find(from);
        for (int32_t b0 = from; b0 < hi; b0 += kStep) {
            int4_t mean[4][DC];
            int exps[4];
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                int32_t page = entry[z];
                if (page < 0 || page >= a.c.n_blocks) {
                    raise_status(a.status, MP_EINVAL);
                    page = 0;
                }
                const int64_t at = (int64_t)page * heads + head;
#pragma unroll
                for (int c = 0; c < DC; ++c)
                    mean[z][c] = *reinterpret_cast<const mean4_t*>(a.c.mean_code + at * D + c * 64 + g * 16);
                exps[z] = a.c.mean_exp[at];
            }
            if (b0 + kStep < hi) find(b0 + kStep);
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                // of the four blocks whose products this lane gets
                int units[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) units[r] = __shfl(exps[z], g * 4 + r, kWave) + kDown;
                const int32_t b = b0 + z * 16;
                if (b >= hi) break;
                for (int t0 = 0; t0 < count; t0 += 16 / span) {
                    const int t = t0 + n / span;
                    float4_t best = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    for (int y = 0; y < columns; ++y) {
                        // columns past a token's last head repeat it
                        const int r = min(t, count - 1) * k.group + min(y * 16 + n % span, k.group - 1);
                        int4_t dot = {0, 0, 0, 0};
#pragma unroll
                        for (int c = 0; c < DC; ++c)
                            dot = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                                mean[z][c],
                                *reinterpret_cast<const int4_t*>(codes + r * ROW + c * 64 + g * 16), dot, 0, 0, 0);
                        const float f = pow2f(max(-126, q_exps[r] - tops[min(t, count - 1)]));
#pragma unroll
                        for (int i = 0; i < 4; ++i) best[i] = fmaxf(best[i], (float)dot[i] * f);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) best[i] = __builtin_amdgcn_ldexpf(span_max(best[i], span), units[i]);
                    if (n % span == 0 && t < count)
                        *reinterpret_cast<float4_t*>(scores + t * step + b + g * 4) = best;
                }
            }
        }
        __syncthreads();  // (with GLOBAL: of this workgroup's own stores, read by it alone)
    }
    for (int t = wave / kTeam; t < count; t += THREADS / kWave / kTeam) {
        const int32_t blocks = blocks_of(t);
        int32_t* const out = k.out + ((q.begin + i0 + t) * heads + head) * k.keep;
        if (blocks <= k.keep) {
            for (int i = kTeam > 1 ? tid : lane; i < k.keep; i += kTeam * kWave) out[i] = i < blocks ? i : -1;
        } else {
            pick<kTeam>(scores + t * step, blocks, k.first, blocks - k.recent, k.keep - k.first - k.recent,
                        picks + wave / kTeam, out);
        }
    }
}

// Tokens of a workgroup, where sequences have several: as many as its scores leave room for and
// leave 768 workgroups, three a compute unit (353 rows of 4 heads: two 19 us, four 22, eight 38).
int32_t tokens_of(const mp_kv_cache& c, const mp_kv_seqs& s, int64_t stride, bool global) {
    if (!s.begin || global || s.most_new < 2) return 1;
    const int64_t room = kLdsScores / stride, some = s.n_tokens * c.heads / 768;
    const int64_t most = some < 2 ? 2 : some > kMostTokens ? kMostTokens : some;
    return (int32_t)(room < 1 ? 1 : room < most ? room : most);
}

template <int D, int THREADS, bool GLOBAL>
hipError_t launch_form(const KvSelect& k, hipStream_t st) {
    constexpr size_t kPicks = THREADS == 1024 ? sizeof(PickLds<THREADS / kWave>) : THREADS / kWave * sizeof(PickLds<1>);
    size_t lds = (size_t)k.tokens * k.group * (D + 16) + ((size_t)k.tokens * k.group + 3) / 4 * 16 + kPicks;
    if (!GLOBAL) lds += (size_t)k.tokens * k.score_stride * sizeof(float);
    if (lds > 65536)
        if (hipError_t e = hipFuncSetAttribute((const void*)kv_select_kernel<D, THREADS, GLOBAL>,
                                               hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            e != hipSuccess)
            return e;
    kv_select_kernel<D, THREADS, GLOBAL><<<dim3((uint32_t)(k.units * k.a.c.heads)), THREADS, lds, st>>>(k);
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const KvSelect& k, bool global, hipStream_t st) {
    if (global) return launch_form<D, 1024, true>(k, st);
    if (k.tokens == 1) return launch_form<D, 1024, false>(k, st);
    return launch_form<D, 256, false>(k, st);
}

}  // namespace

KvSelectShape kv_select_shape(const mp_kv_cache& c, const mp_kv_seqs& s, int32_t q_heads) {
    KvSelectShape sh = {};
    const int64_t most = (s.longest + c.block - 1) / c.block, group = q_heads / c.heads;
    sh.score_stride = most < 16 ? 16 : (most + 15) / 16 * 16;
    // scores of a token lie in LDS where a workgroup can hold them, else in the workspace
    sh.global = sh.score_stride > kLdsScores;
    sh.tokens = tokens_of(c, s, sh.score_stride, sh.global);
    // query codes of many heads take room too
    while (sh.tokens > 1 && sh.tokens * group * (c.dim + 20) > 48 * 1024) --sh.tokens;
    sh.units = s.begin ? s.n_tokens / sh.tokens + s.n_seqs : s.n_seqs;
    // many threads where a workgroup has one token: it is alone with its blocks
    sh.ok = grid_ok(sh.units * c.heads, sh.tokens == 1 ? 1024 : 256);
    if (sh.ok && sh.global) sh.workspace = (size_t)s.n_tokens * c.heads * sh.score_stride * sizeof(float);
    return sh;
}

hipError_t launch_kv_select(const KvSelect& k, hipStream_t st) {
    if (k.a.s.n_tokens == 0) return hipSuccess;
    const bool global = k.score_stride > kLdsScores;
    switch (k.a.c.dim) {
        case 64: return launch_d<64>(k, global, st);
        case 128: return launch_d<128>(k, global, st);
        default: return launch_d<256>(k, global, st);
    }
}

}  // namespace mp
