// Attention over the 8-bit key/value cache.
//
// For a row (a query and one of its heads) with scores s_j = scale * q.k_j,
//   out = sum_j 2^(c s_j - m) v_j / sum_j 2^(c s_j - m),   c = log2 e, m >= max_j c s_j,
// in one pass over the cache with a running m: when it grows, what was summed so far is
// multiplied by 2^(m_old - m_new).
//
// The codes are exact in 16-bit floats (4 or 8 significant bits, no code beyond 448), so
// both products are matrix instructions on 16-bit floats with 32-bit sums, whatever the
// rows' type: queries are brought to [2^14, 2^15) by a power of two per row, which holds
// all bits of a bfloat16 or a 16-bit float down to 2^-29 of the row's largest.  The scale
// of a block's keys multiplies its scores.  That of its values joins the exponent of the
// weights, which enter the second product as w = 2^(c s_j - m + ve_j - vr + 15).  While the value
// exponents that a wave has met differ by no more than 10, vr is the largest of them; from then on
// m + vr follows the largest c s_j + ve_j of the row.  Either way no w reaches 2^16 (m may lag behind
// by less than one), and the row's largest contribution has one of 2^4 at least, normal down to 2^-14:
// a weight has its 11 bits down to 2^-18 of that, and steps of 2^-28 of it below, whatever the sizes
// of other blocks.  The sum of weights takes 2^(c s_j - m) back from w in 32 bits.
//
// Both products are taken transposed, S^T = K Q^T and O^T = V^T W^T: the weights then
// come out of the first product in the lanes that the second one wants them in, as long
// as the token that a lane's key row holds is chosen for it, and the maximum and the sum
// of a row are over one lane's registers and the few lanes of its column.
#include "kv_attend.hpp"

namespace mp {

namespace {

constexpr int kWeightShift = 15;   // weights reach 2^15
constexpr int kLeastShift = -80;   // of a block's value exponent below vr: its weights are zeros
constexpr int kSpread = 10;        // of value exponents that share one vr
// The exponent of a weight is one multiply-add, c s - m, which is off the rounded m by half of its
// last place.  Scores beyond this are rounded, as the maximum was, and taken from it first: none is
// above it then, and what is added to the exponent does not vanish beside it.
constexpr float kLargeScore = 0x1p16f;
// How far (in powers of two) a score up to that size may be above the running maximum before that
// follows.  The difference of the two is exact; with half a place of the score (2^-9) and of the
// exponent's sum (2^-8) a weight reaches 2^15.996, where 16-bit floats end at 2^15.9995.
constexpr float kSlack = 0.99f;

// c s - m with the product rounded by itself: not positive where m is the largest such product.
__device__ __forceinline__ float below_maximum(float s, float c, float m) {
#pragma clang fp contract(off)
    return s * c - m;
}

constexpr int kStep = 64;          // tokens a wave takes at a time

// The value exponents that a wave has met.
struct Met {
    int lo = 127, hi = -128;
    __device__ __forceinline__ void add(int ve) {
        lo = min(lo, ve);
        hi = max(hi, ve);
    }
    __device__ __forceinline__ bool apart() const { return hi - lo > kSpread; }
};

// vr for a new maximum: `top` the largest c s - new_m + ve of this step, what was summed so far at vr.
__device__ __forceinline__ int joint_exp(float top, float m, int vr, float new_m) {
    const float most = fmaxf(top, (m - new_m) + (float)vr);
    return new_m == -INFINITY ? vr : (int)ceilf(most);
}

// What is summed so far, at m and vr, brought to new ones (base: new_m, or 0 for none).
__device__ __forceinline__ float rescale(float m, int vr, float base, int new_vr) {
    return __builtin_amdgcn_exp2f((m - base) + (float)(vr - new_vr));
}

// 2^-shift, where a weight's share of its row's sum is at most 2^-111 once that is out of range.
__device__ __forceinline__ float back_from(int shift) { return pow2f(max(-126, -shift)); }

// A row's query as it lies in memory: lane (column n, quarter g) holds dims [64 c + 16 g, + 16).
template <int D>
struct Query {
    uint4 w[D / 64][2];
};
template <int D>
__device__ __forceinline__ Query<D> load_query(const KvAttend& k, const Row& r, int g) {
    Query<D> x;
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int i = 0; i < 2; ++i) x.w[c][i] = load8_16bit(k.q, r.token, r.head, c * 64 + g * 16 + i * 8);
    return x;
}

// The same as the factor of the first product; `scale` becomes what its scores are multiplied
// by, not negative: the query takes the sign.
template <int D>
__device__ __forceinline__ void query_factor(const KvAttend& k, const Query<D>& raw,
                                             half8_t (&q)[D / 64][2], float* scale) {
    float x[D / 64][16], top = 0.0f;
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
        to_float8(k.q, raw.w[c][0], x[c]);
        to_float8(k.q, raw.w[c][1], x[c] + 8);
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(x[c][i]));
    }
    top = fmaxf(top, __shfl_xor(top, 16, kWave));
    top = fmaxf(top, __shfl_xor(top, 32, kWave));
    uint32_t frac;
    const int e = min(127, max(-90, exponent_of(top, &frac)));
    const float f = k.scale < 0.0f ? -pow2f(15 - e) : pow2f(15 - e);
#pragma unroll
    for (int c = 0; c < D / 64; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) q[c][i / 8][i % 8] = (_Float16)(x[c][i] * f);
    *scale = fabsf(k.scale) * kLog2e * pow2f(max(-126, e - 15));
}

// Of 16 places' codes those of the first n, which alone exist.  No branches: the step that needs it
// is a sequence's last, and every other wave waits for it.
struct FirstCodes {
    uint32_t mask[4];
    __device__ __forceinline__ explicit FirstCodes(int n) {
#pragma unroll
        for (int i = 0; i < 4; ++i) mask[i] = (uint32_t)(((uint64_t)1 << (8 * min(4, max(0, n - 4 * i)))) - 1);
    }
    __device__ __forceinline__ uint4 operator()(uint4 w) const {
        return make_uint4(w.x & mask[0], w.y & mask[1], w.z & mask[2], w.w & mask[3]);
    }
};

// Few rows: 16 columns of rows, one key head, one chunk of tokens.  Each of four or eight waves
// takes every fourth or eighth step of 64 tokens, with its own running maxima, and they are joined
// at the end.  A wave reads the codes straight into registers, the next step's keys as soon as
// this one's are used, the values likewise; nothing is shared, so there is no barrier in
// the loop and what hides the latency is the other waves of the SIMD.
//
// Tokens: key row m of tile t holds token 16 (m / 4) + 4 t + m % 4 of the step.  Lane
// quarter g then has the scores of tokens [16 g, 16 g + 16), four from each tile, which
// are the columns of 16 bytes of each row of values.
//
// What bounds it is memory where there are many workgroups: 64 sequences of 1-16384 tokens 151 us,
// 5.0 TB/s, two of 131072 103 us, 5.2 TB/s (a large copy: 5.2); one of 1000 tokens 11 us, a chain of
// dependent loads (length, table, codes) and 16 steps.  Heads of 256 likewise, with one wave a SIMD: 64
// sequences of 8192 tokens 400 us, 5.4 TB/s (heads of 128: 195 us, 5.5); with 4 new tokens each of
// 4096 305 us, 3.5 TB/s, where a step's 16 columns are all rows and its products show (138 us, 3.9).
// Three waves a SIMD have 168 registers: heads of 128 spill up to three of them.
//
// LIST: one token, and the blocks listed for it.
template <int D, bool INT8, bool LIST, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES == 8 ? 2 : D == 256 ? 1 : 3) void kv_rows_kernel(KvAttend k) {
    constexpr int DT = D / 16, DC = D / 64;
    constexpr bool kEarly = WAVES == 8 && !LIST;  // values before the query
    __shared__ __align__(16) float so[WAVES][16][D + 4];
    __shared__ float sm[WAVES][16], sl[WAVES][16];
    __shared__ int svr[WAVES][16];
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KvArgs& a = k.a;
    if (blockIdx.x == 0) kv_check_begin(a);
    const uint32_t heads = a.c.heads, n_chunks = (uint32_t)k.shape.n_chunks;
    const int head = (int)(blockIdx.x % heads);
    // chunks slowest: workgroups go to the XCDs in turn, and first chunks, which every row group
    // has, must not all meet one of them
    const uint32_t rest = blockIdx.x / heads, units = (uint32_t)k.shape.units, chunk = rest / units;
    RowGroup rg;
    if (!row_group<16>(k, rest % units, &rg)) return;
    const int64_t last_row = min((int64_t)rg.n_rows, rg.row0 + 16) - 1;
    const int32_t most = row_of(k, rg, head, last_row).last;  // the last position any row sees
    const int32_t least = row_of(k, rg, head, rg.row0).last;  // all rows see up to here
    const int lb = a.log_block, block = 1 << lb;
    const int64_t start = chunk * k.shape.chunk;
    const int64_t end_all = LIST ? (int64_t)k.keep << lb : (int64_t)most + 1;
    if (chunk > 0 && start >= end_all) return;
    const int32_t x1 = (int32_t)min(end_all, start + k.shape.chunk);

    Pages pages = {a.s.table + rg.q.s * a.s.table_stride, (uint32_t)max(most, 0) >> lb,
                   (uint32_t)a.c.n_blocks, 0};
    const int32_t* const list = LIST ? k.blocks + (rg.q.begin * heads + head) * k.keep : nullptr;
    const uint32_t page_size = heads * (uint32_t)D << lb;
    const int k_slot = ((n >> 2) * 16) & (block - 1), v_slot = (g * 16) & (block - 1);
    const uint32_t k_at = ((uint32_t)head * D << lb) + (k_slot + (n & 3)) * D + g * 16;
    const uint32_t v_at = ((uint32_t)head * D << lb) + ((n << lb) | v_slot);
    uint4 kw[4][DC], vw[DT];
    // of the loaded step: the exponents of tokens [16 g, + 16), the position of the first;
    // of the one after: the table entries of the keys' and the values' tokens
    int ke = 0, ve = 0;
    int32_t pos = 0, next_pos = 0;
    uint32_t k_entry = 0, v_entry = 0;
    const int32_t kNowhere = INT32_MAX - 64;  // the position of a place that names no block
    auto named = [&](int32_t x) -> int32_t {
        const int32_t b = x >> lb;
        const int32_t id = b < k.keep ? list[b] : -1;
        const bool seen = id >= 0 && id <= most >> lb;  // none where most is -1
        if (id != -1 && !seen) pages.worst = ~0u;
        return seen ? id : -1;
    };
    auto find = [&](int32_t x) {
        if (LIST) {
            const int32_t kb = named(x + (n >> 2) * 16), vb = named(x + g * 16);
            k_entry = kb < 0 ? 0 : pages.entry((uint32_t)kb);
            v_entry = vb < 0 ? 0 : pages.entry((uint32_t)vb);
            next_pos = vb < 0 ? kNowhere : (vb << lb) + v_slot;
        } else {
            k_entry = pages.entry((uint32_t)(x + (n >> 2) * 16) >> lb);
            v_entry = pages.entry((uint32_t)(x + g * 16) >> lb);
            next_pos = x + g * 16;
        }
    };
    auto load_keys = [&]() {
        const uint8_t* const p = a.c.k_code + ((uint64_t)pages.page(k_entry) * page_size + k_at);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < DC; ++c)
                kw[t][c] = *reinterpret_cast<const uint4*>(p + t * 4 * D + c * 64);
    };
    auto load_values = [&]() {
        const uint32_t page = pages.page(v_entry);
        const uint8_t* const p = a.c.v_code + ((uint64_t)page * page_size + v_at);
#pragma unroll
        for (int t = 0; t < DT; ++t) vw[t] = *reinterpret_cast<const uint4*>(p + (t * 16 << lb));
        ke = a.c.k_exp[(uint64_t)page * heads + head];
        ve = a.c.v_exp[(uint64_t)page * heads + head];
        pos = next_pos;
    };
    const Row row = row_of(k, rg, head, rg.row0 + n);
    const Query<D> raw_q = load_query<D>(k, row, g);
    int32_t x = (int32_t)start + wave * kStep;
    const int32_t stride = WAVES * kStep;
    if (x < x1) {
        find(x);
        load_keys();
        if (kEarly) load_values();
    }
    half8_t q[DC][2];
    float scale;
    query_factor<D>(k, raw_q, q, &scale);
    // the values after the query, whose conversion wants registers, where three waves share them: 64
    // sequences of 1-16384 tokens 152 us, 159 with these loads before it
    if (x < x1) {
        if (!kEarly) load_values();
        if (x + stride < x1) find(x + stride);
    }
    float4_t acc[DT];
    float m = -INFINITY, l = 0.0f;
    int vr = 0;
    Met met;
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = float4_t{0, 0, 0, 0};

    for (; x < x1; x += stride) {
        float s[16];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            float4_t z = {0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < DC; ++c) {
                z = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    codes_to_half<INT8>(kw[t][c].x, kw[t][c].y), q[c][0], z, 0, 0, 0);
                z = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    codes_to_half<INT8>(kw[t][c].z, kw[t][c].w), q[c][1], z, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) s[t * 4 + r] = z[r];
        }
        const bool more = x + stride < x1;
        if (more) load_keys();
        // whether some row does not see some token of the step
        const bool masked = LIST ? __any(pos + 15 > least) : x + kStep - 1 > least;
        if (masked) {
            const int seen = row.last - pos;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = i > seen ? -INFINITY : s[i];
            // places past the end may hold anything
            const FirstCodes first(most - pos + 1);
#pragma unroll
            for (int t = 0; t < DT; ++t) vw[t] = first(vw[t]);
        }
        float c = fmaxf(scale * pow2f(ke), 1.17549435e-38f);  // -inf * 0 is no score
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        const float mine = top;
        top *= c;
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        // places that name no block have no exponent
        const int was = met.hi;
        const auto meet = [&](int of) {
            if (!LIST || __builtin_amdgcn_readlane(pos, of) != kNowhere) met.add(__builtin_amdgcn_readlane(ve, of));
        };
        meet(0);
        if (lb < 6) meet(16), meet(32), meet(48);
        const float new_m = fmaxf(m, top);
        const float base = new_m == -INFINITY ? 0.0f : new_m;
        int new_vr = met.hi;
        if (met.apart()) {
            float most = below_maximum(mine, c, base) + (float)ve;
            most = fmaxf(most, __shfl_xor(most, 16, kWave));
            most = fmaxf(most, __shfl_xor(most, 32, kWave));
            new_vr = joint_exp(most, m, vr, new_m);
        }
        float from = base;  // taken from the scores with the multiply-add
        if (__any(fabsf(base) > kLargeScore)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = below_maximum(s[i], c, base);
            c = 1.0f;
            from = 0.0f;
        }
        if (met.apart() || met.hi > was || __any(new_m > m)) {
            const float fall = __builtin_amdgcn_exp2f(m - base), both = rescale(m, vr, base, new_vr);
#pragma unroll
            for (int t = 0; t < DT; ++t) acc[t] *= both;
            l *= fall;
            m = new_m;
            vr = new_vr;
        }
        const int shift = max(kLeastShift, ve - vr) + kWeightShift;
        const float add = (float)shift - from;
        float sum = 0.0f;
        half8_t w[2];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, add));
            sum += e;
            w[i / 8][i % 8] = (_Float16)e;
        }
        l += sum * back_from(shift);
#pragma unroll
        for (int t = 0; t < DT; ++t) {
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half<INT8>(vw[t].x, vw[t].y),
                                                            w[0], acc[t], 0, 0, 0);
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(codes_to_half<INT8>(vw[t].z, vw[t].w),
                                                            w[1], acc[t], 0, 0, 0);
        }
        if (more) {
            load_values();
            if (x + 2 * stride < x1) find(x + 2 * stride);
        }
    }
    if (pages.bad()) raise_status(a.status, MP_EINVAL);

    // the waves' results of a row joined
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (g == 0) {
        sm[wave][n] = m;
        sl[wave][n] = l;
        svr[wave][n] = vr;
    }
#pragma unroll
    for (int t = 0; t < DT; ++t)
        *reinterpret_cast<float4_t*>(&so[wave][n][t * 16 + g * 4]) = acc[t];
    __syncthreads();
    if (WAVES > 4 && threadIdx.x >= 256) return;
    const int col = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * (D / 16);
    float top = sm[0][col];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, sm[w][col]);
    const float base = top == -INFINITY ? 0.0f : top;
    // what a wave summed is 2^of[w] its numbers, counted from base
    float of[WAVES], most_of = -INFINITY;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        of[w] = (sm[w][col] - base) + (float)svr[w][col];
        most_of = fmaxf(most_of, of[w]);
    }
    if (most_of == -INFINITY) most_of = 0.0f;
    float total = 0.0f, o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm[w][col] - base);
        const float fv = __builtin_amdgcn_exp2f(of[w] - most_of);
        total += sl[w][col] * f;
#pragma unroll
        for (int i = 0; i < D / 16; i += 4) {
            const float4_t y = *reinterpret_cast<const float4_t*>(&so[w][col][d0 + i]);
#pragma unroll
            for (int z = 0; z < 4; ++z) o[i + z] += y[z] * fv;
        }
    }
    const Row r = row_of(k, rg, head, rg.row0 + col);
    if (!r.live) return;
    const int64_t index = r.token * (int64_t)k.group * heads + r.head;
    if (n_chunks > 1) {
        const Partials part_out = partials(k);
        float* to = part_out.o + (index * n_chunks + chunk) * D + d0;
#pragma unroll
        for (int i = 0; i < D / 16; i += 4)
            *reinterpret_cast<float4_t*>(to + i) = float4_t{o[i], o[i + 1], o[i + 2], o[i + 3]};
        if (d0 == 0)
            part_out.sums[index * n_chunks + chunk] = float4_t{top, total, most_of - (float)kWeightShift, 0};
    } else {
        // a row that sees nothing: weights and sums are zero
        const float norm = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
        const float back = norm * __builtin_amdgcn_exp2f(most_of - (float)kWeightShift);
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] *= back;
        constexpr int kOnce = D / 16 >= 8 ? 8 : 4;
#pragma unroll
        for (int i = 0; i < D / 16; i += kOnce) store_16bit<kOnce>(k.out, r.token, r.head, d0 + i, o + i);
        if (k.lse && d0 == 0)
            k.lse[index] = total > 0.0f ? (base + log2f(total)) * kLn2 : total == 0.0f ? -INFINITY : total;
    }
}

// A row's query for the form of 32 rows a wave: half h of the wave has dims 16 i + 8 h + [0, 8).
// `scale` as query_factor.
template <int D>
__device__ __forceinline__ void load_rows(const KvAttend& k, const Row& row, int h,
                                          half8_t (&q)[D / 16], float* scale) {
    uint4 raw[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) raw[i] = load8_16bit(k.q, row.token, row.head, i * 16 + h * 8);
    float x[D / 16][8], top = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
        to_float8(k.q, raw[i], x[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[i][j]));
    }
    top = fmaxf(top, __shfl_xor(top, 32, kWave));
    uint32_t frac;
    const int e = min(127, max(-90, exponent_of(top, &frac)));
    const float f = k.scale < 0.0f ? -pow2f(15 - e) : pow2f(15 - e);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) q[i][j] = (_Float16)(x[i][j] * f);
    *scale = fabsf(k.scale) * kLog2e * pow2f(max(-126, e - 15));
}

// The result of a wave of 32 rows, a column each: lane half h has dims 4 h + [0, 4) of every eight.
template <int D>
__device__ __forceinline__ void store_rows(const KvAttend& k, const Row& row, uint32_t chunk,
                                           const float16_t (&acc)[D / 32], float m, float l,
                                           int vr, int h) {
    const float total = l + __shfl_xor(l, 32, kWave);
    if (!row.live) return;
    const uint32_t n_chunks = (uint32_t)k.shape.n_chunks;
    // a row that sees nothing: weights and sums are zero
    const float norm = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
    const int64_t index = row.token * (int64_t)k.group * k.a.c.heads + row.head;
    const Partials part_out = partials(k);
    const bool whole = n_chunks == 1;
    const float f = whole ? norm * pow2f(max(-126, vr - kWeightShift)) : 1.0f;
    float* const to = part_out.o + (index * n_chunks + chunk) * D;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int d = t * 32 + r * 2 + 4 * h;
            float o[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = acc[t][r + i] * f;
            if (whole)
                store_16bit<4>(k.out, row.token, row.head, d, o);
            else
                *reinterpret_cast<float4_t*>(to + d) = float4_t{o[0], o[1], o[2], o[3]};
        }
    if (h == 0) {
        if (!whole)
            part_out.sums[index * n_chunks + chunk] = float4_t{m, total, (float)(vr - kWeightShift), 0};
        else if (k.lse)
            k.lse[index] = total > 0.0f ? (m + log2f(total)) * kLn2 : total == 0.0f ? -INFINITY : total;
    }
}

// vr of a row for a tile whose blocks' value exponents are apart, before its scores are changed: N equal
// parts of one exponent each.
template <int N>
__device__ __forceinline__ int tile_exp(const float16_t (&s)[2], const float (&c)[N], const int (&ve)[N], float m,
                                        int vr, float new_m) {
    float most = -INFINITY;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float part = -INFINITY;
#pragma unroll
        for (int r = i * (32 / N); r < (i + 1) * (32 / N); ++r) part = fmaxf(part, s[r / 16][r % 16]);
        most = fmaxf(most, below_maximum(part, c[i], new_m) + (float)ve[i]);
    }
    most = fmaxf(most, __shfl_xor(most, 32, kWave));
    return joint_exp(most, m, vr, new_m);
}

// For each part of a tile, what is added to a weight's exponent, and the factor that takes the
// shift back out of its sum.  Where exponents are not apart vr is met.hi in all lanes, and the
// arithmetic is left to scalar registers.
template <int N>
__device__ __forceinline__ void weight_shifts(const Met& met, int vr, const int (&ve)[N], float from,
                                              float (&add)[N], float (&back)[N]) {
    if (met.apart()) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int shift = max(kLeastShift, ve[i] - vr) + kWeightShift;
            add[i] = (float)shift - from;
            back[i] = back_from(shift);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int shift = ve[i] - met.hi + kWeightShift;
        add[i] = (float)shift - from;
        back[i] = pow2f(-shift);
    }
}

// Many rows: four waves of 32 rows, one key head, one chunk of tokens, in tiles of 64 tokens
// whose codes the workgroup turns into 16-bit floats once, in LDS, for all 128 rows.  Two
// tiles' room: while one is computed the next one's codes, already in registers, are
// converted into the other and the loads of the one after are on their way, so a tile
// costs one barrier.
//
// Measured, 333 rows of heads of 64 after 20000 tokens: 117 us with the join, 466 TFLOP/s.  Of a
// tile's work per wave the softmax's vector instructions take twice the cycles of its 16 products.
// Four prompts of 4096 tokens, 32 query heads over 8: heads of 64 369 us, 745 TFLOP/s; of 256 1817 us,
// 605 TFLOP/s, by one wave a SIMD beside whose softmax nothing runs.  With value exponents apart
// (2^15): 403 and 2103 us, the row's largest product of weight and scale being looked for.
//
// Keys lie by row of the instruction: row m of 32 is token m with bits 2 and 3 exchanged,
// so that a lane's scores are those of eight consecutive tokens, as the second product
// takes them.  Both arrays have their 16-byte pieces exchanged by the row's low bits, so that
// the lanes of a read, which go down the rows, meet different banks.
template <int D>
struct TileLds {
    uint4 k[64][D / 8];  // [32 * half + row][piece ^ k_key]
    uint4 v[D][8];       // [dim][piece ^ v_key]: eight tokens a piece
};
// 16 lanes of a read share a turn at the 64 banks, 0-3 with 12-15, 20-23 and 24-27: rows of 256
// bytes need 16 different keys among them, rows of 128 bytes 8 for each parity of the row.
template <int D>
__device__ __forceinline__ int k_key(int row) {
    return D == 64 ? row >> 1 & 7 : row & 15;
}
__device__ __forceinline__ int v_key(int dim) { return dim >> 1 & 7; }

template <int D, bool INT8>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void kv_tiles_kernel(KvAttend k) {
    constexpr int KS = D / 16, DT = D / 32, ROW = D / 16;  // ROW: loads of a token's keys
    constexpr int KL = 64 * ROW / 256, VL = D * 4 / 256;   // loads of a thread for a tile
    extern __shared__ __align__(16) char lds_raw[];
    TileLds<D>* const lds = reinterpret_cast<TileLds<D>*>(lds_raw);
    const int tid = threadIdx.x, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const KvArgs& a = k.a;
    if (blockIdx.x == 0) kv_check_begin(a);
    // key heads fastest: workgroups of one head share an XCD's L2 where 8 and the number of
    // heads divide
    const uint32_t heads = a.c.heads, n_chunks = (uint32_t)k.shape.n_chunks;
    const int head = (int)(blockIdx.x % heads);
    const uint32_t rest = blockIdx.x / heads, chunk = rest % n_chunks;
    RowGroup rg;
    if (!tile_group<128>(k, rest / n_chunks, &rg)) return;
    const int32_t most = row_of(k, rg, head, min((int64_t)rg.n_rows, rg.row0 + 128) - 1).last;
    const int64_t start = chunk * k.shape.chunk;
    if (chunk > 0 && start > most) return;
    const int32_t x0 = (int32_t)start;
    const int32_t x1 = (int32_t)min((int64_t)most + 1, start + k.shape.chunk);

    // this wave's rows: the last position that any sees, and the last that all see
    const int64_t wave_row0 = rg.row0 + 32 * wave;
    const bool awake = wave_row0 < rg.n_rows;
    const int32_t wave_most = awake ? row_of(k, rg, head, min((int64_t)rg.n_rows, wave_row0 + 32) - 1).last : -1;
    const int32_t wave_least = awake ? row_of(k, rg, head, wave_row0).last : -1;
    const Row row = row_of(k, rg, head, wave_row0 + n);

    half8_t q[KS];
    float scale;
    load_rows<D>(k, row, h, q, &scale);

    float16_t acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = float16_t{};
    float m = -INFINITY, l = 0.0f;
    int vr = 0;
    Met met;

    // a thread's loads of a tile: 16 dims of KL tokens' keys, 16 tokens of VL dims' values; the
    // table entries are read a tile ahead of them
    const int lb = a.log_block, block = 1 << lb;
    const uint32_t page_size = heads * (uint32_t)D << lb;
    Pages pages = {a.s.table + rg.q.s * a.s.table_stride, (uint32_t)max(most, 0) >> lb,
                   (uint32_t)a.c.n_blocks, 0};
    // the 16 tokens that a wave's keys of one load lie in: their block is the same for the wave
    auto group_of = [&](int i) { return (wave * (64 / ROW) + i * (256 / ROW)) >> 4; };
    const uint32_t k_at = ((uint32_t)head * D << lb) + (tid % ROW) * 16;
    const uint32_t v_at =
        ((uint32_t)head * D << lb) + (((tid >> 2) << lb) | ((tid & 3) * 16 & (block - 1)));
    uint4 kw[KL], vw[VL];
    uint32_t k_entry[KL], v_entry;
    int my_ke = 0, my_ve = 0;  // of tokens [16 (tid % 4), + 16) of the loaded tile
    auto find = [&](int32_t x) {
#pragma unroll
        for (int i = 0; i < KL; ++i)
            k_entry[i] = pages.entry((uint32_t)(x + group_of(i) * 16) >> lb);
        v_entry = pages.entry((uint32_t)(x + (tid & 3) * 16) >> lb);
    };
    auto load = [&]() {
#pragma unroll
        for (int i = 0; i < KL; ++i) {
            const uint32_t slot = (tid / ROW + i * (256 / ROW)) & (block - 1);
            const uint32_t page = pages.page(__builtin_amdgcn_readfirstlane(k_entry[i]));
            kw[i] = *reinterpret_cast<const uint4*>(a.c.k_code + (uint64_t)page * page_size +
                                                    (k_at + slot * D));
        }
        const uint32_t page = pages.page(v_entry);
        const uint8_t* const v = a.c.v_code + (uint64_t)page * page_size + v_at;
#pragma unroll
        for (int i = 0; i < VL; ++i) vw[i] = *reinterpret_cast<const uint4*>(v + (i * 64 << lb));
        my_ke = a.c.k_exp[(uint64_t)page * heads + head];
        my_ve = a.c.v_exp[(uint64_t)page * heads + head];
    };
    // the loaded codes (of the tile at x) as 16-bit floats in LDS; places past the end, which may
    // hold anything, as zeros among the values
    auto put = [&](int buf, int32_t x) {
        const bool tail = x + 63 > most;
        const FirstCodes first(most - (x + (tid & 3) * 16) + 1);
#pragma unroll
        for (int i = 0; i < KL; ++i) {
            const int t = tid / ROW + i * (256 / ROW), piece = tid % ROW * 2;
            const int r = (t & 0x33) | (t & 4) << 1 | (t & 8) >> 1;
            uint4* const to = lds[buf].k[r];
            to[piece ^ k_key<D>(r)] = __builtin_bit_cast(uint4, codes_to_half<INT8>(kw[i].x, kw[i].y));
            to[(piece ^ k_key<D>(r)) ^ 1] = __builtin_bit_cast(uint4, codes_to_half<INT8>(kw[i].z, kw[i].w));
        }
#pragma unroll
        for (int i = 0; i < VL; ++i) {
            const int d = (tid >> 2) + i * 64, piece = (tid & 3) * 2;
            if (tail) vw[i] = first(vw[i]);
            uint4* const to = lds[buf].v[d];
            to[piece ^ v_key(d)] = __builtin_bit_cast(uint4, codes_to_half<INT8>(vw[i].x, vw[i].y));
            to[(piece ^ v_key(d)) ^ 1] = __builtin_bit_cast(uint4, codes_to_half<INT8>(vw[i].z, vw[i].w));
        }
    };

    int buf = 0;
    int ke[4], ve[4];  // of the tile in `buf`
    if (x0 < x1) {
        find(x0);
        load();
        find(x0 + 64);
        put(0, x0);
    }
    for (int32_t x = x0; x < x1; x += 64, buf ^= 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            ke[i] = __builtin_amdgcn_readlane(my_ke, i);
            ve[i] = __builtin_amdgcn_readlane(my_ve, i);
        }
        if (x + 64 < x1) {
            load();
            find(x + 128);
        }
        __syncthreads();  // the tile is whole; the other one is read no more
        if (x <= wave_most) {
            float16_t s[2] = {float16_t{}, float16_t{}};
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const int r = t * 32 + n;
                    const half8_t f = __builtin_bit_cast(half8_t, lds[buf].k[r][(i * 2 + h) ^ k_key<D>(r)]);
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, q[i], s[t], 0, 0, 0);
                }
            // register r of product t is token 32 t + 16 (r / 8) + 8 h + r % 8
            const bool masked = x + 63 > wave_least;
            if (masked) {
                const int seen = row.last - x - h * 8;
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[t][r] = t * 32 + (r >> 3) * 16 + (r & 7) > seen ? -INFINITY : s[t][r];
            }
            float c[4], top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                c[i] = fmaxf(scale * pow2f(ke[i]), 1.17549435e-38f);  // -inf * 0 is no score
                float part = -INFINITY;
#pragma unroll
                for (int r = 0; r < 8; ++r) part = fmaxf(part, s[i / 2][i % 2 * 8 + r]);
                top = fmaxf(top, part * c[i]);
            }
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float new_m = fmaxf(m, top);
            const float base = new_m == -INFINITY ? 0.0f : new_m;
            const int was = met.hi;
#pragma unroll
            for (int i = 0; i < 4; ++i) met.add(ve[i]);
            int new_vr = met.hi;
            if (met.apart()) new_vr = tile_exp<4>(s, c, ve, m, vr, new_m);
            const bool large = __any(fabsf(base) > kLargeScore);
            if (large) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        s[i / 2][i % 2 * 8 + r] = below_maximum(s[i / 2][i % 2 * 8 + r], c[i], base);
                    c[i] = 1.0f;
                }
            }
            const bool moved = large || met.hi > was || met.apart();
            if (__any(new_m - m > kSlack || moved)) {
                const float fall = __builtin_amdgcn_exp2f(m - base), both = rescale(m, vr, base, new_vr);
#pragma unroll
                for (int t = 0; t < DT; ++t) acc[t] *= both;
                l *= fall;
                m = new_m;
                vr = new_vr;
            }
            const float from = large || m == -INFINITY ? 0.0f : m;  // taken from the scores yet
            half8_t w[4];
            float add[4], back[4];
            weight_shifts(met, vr, ve, from, add, back);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float sum = 0.0f;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][i % 2 * 8 + r], c[i], add[i]));
                    sum += e;
                    w[i][r] = (_Float16)e;
                }
                l += sum * back[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    const int d = t * 32 + n;
                    const half8_t f = __builtin_bit_cast(half8_t, lds[buf].v[d][(i * 2 + h) ^ v_key(d)]);
                    acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f, w[i], acc[t], 0, 0, 0);
                }
        }
        if (x + 64 < x1) put(buf ^ 1, x + 64);
    }
    if (pages.bad()) raise_status(a.status, MP_EINVAL);
    store_rows<D>(k, row, chunk, acc, m, l, vr, h);
}

// Many rows, heads of 128: two teams of four waves, 32 rows each wave, over one key head
// and one chunk of tokens in tiles of 64.  Of a SIMD's two waves one is of each team, and
// the teams take turns: while one is at its matrix products (the last tile's second one,
// this tile's first) the other is at its softmax; a barrier ends a turn.  Matrix and vector
// instructions of two waves run beside each other on a SIMD, but left alone the waves fall
// into step, as they meet at every tile's barrier, and wait for the same unit.
//
// A team's half of the conversion and of the loads for the next tiles goes between its matrix
// instructions, whose 32 cycles leave room for seven others: in the turn of the first product
// of tile i the keys of tile i + 1 and the values of tile i are put into LDS, loaded in the turn
// before, and keys i + 2 and values i + 1 are loaded.  With team 0 at tile i in turn 2 i
// and team 1 in turn 2 i + 1, keys i are read in these two turns and values i in the next two:
// each is whole the turn before, and two tiles' room is enough for both.
//
// Measured, prompts of 228-4096 tokens, 32 query heads over 8: 276 us, 838 TFLOP/s; four of 4096 tokens
// 575 us, 956 TFLOP/s (620 with value exponents apart).  A turn takes 1850
// cycles: 1510 of products (1024 of matrix instructions; reading their factors takes the LDS as
// long, as each serves one instruction) beside a softmax of 830, the rest barriers.
//
// EXPS: exponents of a tile, 1 where a block is a tile.
template <bool INT8, int EXPS>
__global__ __launch_bounds__(512, 2) void kv_pair_kernel(KvAttend k) {
    constexpr int D = 128, KS = D / 16, DT = D / 32, ROW = D / 16;  // ROW: loads of a token's keys
    constexpr int LOADS = 2;  // of a thread for its team's half of a tile: of keys, of values
    extern __shared__ __align__(16) char lds_raw[];
    TileLds<D>* const lds = reinterpret_cast<TileLds<D>*>(lds_raw);
    const int tid = threadIdx.x & 255, lane = tid & 63, n = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), team = wave >> 2;
    const KvArgs& a = k.a;
    if (blockIdx.x == 0) kv_check_begin(a);
    // key heads fastest: workgroups of one head share an XCD's L2 where 8 and the number of
    // heads divide
    const uint32_t heads = a.c.heads, n_chunks = (uint32_t)k.shape.n_chunks;
    const int head = (int)(blockIdx.x % heads);
    const uint32_t rest = blockIdx.x / heads, chunk = rest % n_chunks;
    RowGroup rg;
    if (!tile_group<256>(k, rest / n_chunks, &rg)) return;
    const int32_t most = row_of(k, rg, head, min((int64_t)rg.n_rows, rg.row0 + 256) - 1).last;
    const int64_t start = chunk * k.shape.chunk;
    if (chunk > 0 && start > most) return;
    const int32_t x0 = (int32_t)start;
    const int32_t x1 = (int32_t)min((int64_t)most + 1, start + k.shape.chunk);
    const int32_t tiles = (x1 - x0 + 63) >> 6;  // 0 where no row sees anything

    // this wave's rows, and the last position that all of them see
    const int64_t wave_row0 = rg.row0 + 32 * wave;
    const bool awake = wave_row0 < rg.n_rows;  // has rows
    const int32_t wave_least = row_of(k, rg, head, wave_row0).last;
    const Row row = row_of(k, rg, head, wave_row0 + n);

    const int lb = a.log_block, block = 1 << lb;
    const uint32_t page_size = heads * (uint32_t)D << lb;
    Pages pages = {a.s.table + rg.q.s * a.s.table_stride, (uint32_t)max(most, 0) >> lb,
                   (uint32_t)a.c.n_blocks, 0};
    // load r: whether of values, the first token of its 16 in the tile, its place in a block's
    // codes, in LDS; table entries are read a tile ahead of the loads
    bool is_v[LOADS];
    int first[LOADS];
    const uint8_t* from[LOADS];
    uint4* to[LOADS];
    int piece[LOADS];
    uint4 codes[LOADS];
    uint32_t entry[LOADS];
#pragma unroll
    for (int r = 0; r < LOADS; ++r) {
        is_v[r] = r == 1;
        const int i = tid;
        const int token = team * 32 + i / ROW, dim = team * (D / 2) + i / 4;
        const int key_row = (token & 0x33) | (token & 4) << 1 | (token & 8) >> 1;
        first[r] = is_v[r] ? (i & 3) * 16 : token & 48;
        const uint32_t at = is_v[r] ? ((uint32_t)dim << lb) | (first[r] & (block - 1))
                                    : (uint32_t)(token & (block - 1)) * D + i % ROW * 16;
        from[r] = (is_v[r] ? a.c.v_code : a.c.k_code) + ((uint32_t)head * D << lb) + at;
        to[r] = is_v[r] ? lds[0].v[dim] : lds[0].k[key_row];
        piece[r] = is_v[r] ? ((i & 3) * 2) ^ v_key(dim) : (i % ROW * 2) ^ k_key<D>(key_row);
        codes[r] = make_uint4(0, 0, 0, 0);
        entry[r] = 0;
    }
    // the tile of load r, with that of keys a tile ahead of that of values
    auto tile_of = [&](int r, int v_tile) { return v_tile + (is_v[r] ? 0 : 1); };
    auto find = [&](int r, int v_tile) {
        entry[r] = pages.entry((uint32_t)(x0 + tile_of(r, v_tile) * 64 + first[r]) >> lb);
    };
    auto load = [&](int r) {
        codes[r] = *reinterpret_cast<const uint4*>(from[r] + (uint64_t)pages.page(entry[r]) * page_size);
    };
    auto put = [&](int r, int v_tile, int half) {
        uint4* const at = to[r] + (tile_of(r, v_tile) & 1) * (int)(sizeof(TileLds<D>) / 16);
        const uint32_t lo = half ? codes[r].z : codes[r].x, hi = half ? codes[r].w : codes[r].y;
        at[piece[r] ^ half] = __builtin_bit_cast(uint4, codes_to_half<INT8>(lo, hi));
    };
    // places past the end, which may hold anything, are zeros among the values
    auto end_values = [&](int v_tile) {
        if (x0 + v_tile * 64 + 63 <= most) return;
#pragma unroll
        for (int r = 0; r < LOADS; ++r)
            if (is_v[r]) codes[r] = FirstCodes(most - (x0 + v_tile * 64 + first[r]) + 1)(codes[r]);
    };
    // the exponents of tokens [16 (tid % 4), + 16) of a tile
    uint32_t exp_entry = 0;
    int exp_k = 0, exp_v = 0;
    auto find_exps = [&](int tile) {
        exp_entry = pages.entry((uint32_t)(x0 + tile * 64 + (tid & 3) * 16) >> lb);
    };
    auto load_exps = [&]() {
        const uint64_t at = (uint64_t)pages.page(exp_entry) * heads + head;
        exp_k = a.c.k_exp[at];
        exp_v = a.c.v_exp[at];
    };
    int ke[EXPS] = {}, ve[EXPS] = {};
    auto read_exps = [&]() {
#pragma unroll
        for (int i = 0; i < EXPS; ++i) {
            ke[i] = __builtin_amdgcn_readlane(exp_k, i);
            ve[i] = __builtin_amdgcn_readlane(exp_v, i);
        }
    };
    if (tiles > 0) {
        find_exps(0);
#pragma unroll
        for (int r = 0; r < LOADS; ++r) find(r, -1);  // keys 0
        load_exps();
#pragma unroll
        for (int r = 0; r < LOADS; ++r) load(r);
        find_exps(1);
#pragma unroll
        for (int r = 0; r < LOADS; ++r) find(r, 0);  // keys 1, values 0
    }

    half8_t q[KS];
    float scale;
    load_rows<D>(k, row, h, q, &scale);
    float16_t acc[DT], s[2];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = float16_t{};
    s[0] = s[1] = float16_t{};
    half8_t w[4] = {};
    float m = -INFINITY, l = 0.0f;
    int vr = 0;
    Met met;

    auto turn = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };
    // Piece `p` of a team's moving of data in the turn of tile i's first product: 2 LOADS pieces
    // put keys i + 1 and values i, the others load the ones after.
    constexpr int kPieces = 4 * LOADS + 1;
    auto move = [&](int p, int i) {
        if (p < 2 * LOADS) {
            put(p / 2, i, p % 2);
        } else if (p < 3 * LOADS) {
            load(p - 2 * LOADS);
        } else if (p < 4 * LOADS) {
            find(p - 3 * LOADS, i + 2);
        } else {
            load_exps();
            find_exps(i + 2);
        }
    };
    // Factors from LDS: keys of instruction step i, product t; values of step i, dims t.  A lane's
    // place in a row is its own but for the step's bits.
    const int k_from = n * (D / 8), k_mine = h ^ k_key<D>(n), v_from = n * 8, v_mine = h ^ v_key(n);
    auto k_factor = [&](int tile, int i, int t) {
        const uint4* const at = &lds[tile & 1].k[0][0] + t * 32 * (D / 8) + k_from;
        return __builtin_bit_cast(half8_t, at[k_mine ^ (i * 2)]);
    };
    auto v_factor = [&](int tile, int i, int t) {
        const uint4* const at = &lds[tile & 1].v[0][0] + t * 32 * 8 + v_from;
        return __builtin_bit_cast(half8_t, at[v_mine ^ (i * 2)]);
    };
    // The second product of tile i - 1 (SECOND) and the first of tile i (FIRST), factors read kAhead
    // instructions ahead of their use: left to itself the compiler reads each just before.
    auto products = [&](auto second, auto first_too, int i) {
        constexpr int kSecond = second() ? 4 * DT : 0, kAll = kSecond + (first_too() ? 2 * KS : 0);
        constexpr int kAhead = 6;
        __builtin_amdgcn_s_setprio(1);  // the other wave's vector instructions fill what these leave
        half8_t f[kAhead];
        auto factor = [&](int j) {
            return j < kSecond ? v_factor(i - 1, j / DT, j % DT)
                               : k_factor(i, (j - kSecond) / 2, (j - kSecond) % 2);
        };
#pragma unroll
        for (int j = 0; j < kAhead; ++j) f[j] = factor(j);
        __builtin_amdgcn_sched_barrier(0);
        if (first_too()) s[0] = s[1] = float16_t{};
#pragma unroll
        for (int j = 0; j < kAll; ++j) {
            const half8_t use = f[j % kAhead];
            if (j < kSecond) {
                acc[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(use, w[j / DT], acc[j % DT], 0, 0, 0);
            } else {
                const int z = j - kSecond;
                s[z % 2] = __builtin_amdgcn_mfma_f32_32x32x16_f16(use, q[z / 2], s[z % 2], 0, 0, 0);
            }
            if (j + kAhead < kAll) f[j % kAhead] = factor(j + kAhead);
            if (first_too() && j % 2 == 1 && j / 2 < kPieces) move(j / 2, i);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (first_too())
#pragma unroll
            for (int p = kAll / 2; p < kPieces; ++p) move(p, i);
    };
    using Yes = std::true_type;
    using No = std::false_type;

    // keys 0 put before the first turn; then keys 1 and values 0 on their way
    if (tiles > 0) {
#pragma unroll
        for (int r = 0; r < LOADS; ++r)
            if (!is_v[r]) put(r, -1, 0), put(r, -1, 1);
        read_exps();
#pragma unroll
        for (int r = 0; r < LOADS; ++r) load(r), find(r, 1);
        end_values(0);
    }
    turn();
    if (team) turn();
    if (!awake) {  // only moves data
        for (int tile = 0; tile < tiles; ++tile) {
            for (int p = 0; p < kPieces; ++p) move(p, tile);
            turn();
            end_values(tile + 1);
            turn();
        }
        if (!team) turn();
        if (pages.bad()) raise_status(a.status, MP_EINVAL);
        return;
    }
    if (tiles > 0) products(No{}, Yes{}, 0);
    for (int tile = 0; tile < tiles; ++tile) {
        const int32_t x = x0 + tile * 64;
        turn();
        end_values(tile + 1);
        // register r of product t is token 32 t + 16 (r / 8) + 8 h + r % 8
        const bool masked = x + 63 > wave_least;
        if (masked) {
            const int seen = row.last - x - h * 8;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[t][r] = t * 32 + (r >> 3) * 16 + (r & 7) > seen ? -INFINITY : s[t][r];
        }
        constexpr int kOf = 32 / EXPS;  // a lane's scores of one exponent
        float c[EXPS], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < EXPS; ++i) {
            c[i] = fmaxf(scale * pow2f(ke[i]), 1.17549435e-38f);  // -inf * 0 is no score
            float part = -INFINITY;
#pragma unroll
            for (int r = i * kOf; r < (i + 1) * kOf; ++r) part = fmaxf(part, s[r / 16][r % 16]);
            top = fmaxf(top, part * c[i]);
        }
        {
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
        }
        const float new_m = fmaxf(m, top);
        const int was = met.hi;
#pragma unroll
        for (int i = 0; i < EXPS; ++i) met.add(ve[i]);
        bool large = false;
        const bool moved = met.hi > was || met.apart();
        if (__any(new_m - m > kSlack || fabsf(new_m) > kLargeScore || moved)) {
            const float base = new_m == -INFINITY ? 0.0f : new_m;
            int new_vr = met.hi;
            if (met.apart()) new_vr = tile_exp<EXPS>(s, c, ve, m, vr, new_m);
            large = __any(fabsf(base) > kLargeScore);
            if (large) {
#pragma unroll
                for (int i = 0; i < EXPS; ++i) {
#pragma unroll
                    for (int r = i * kOf; r < (i + 1) * kOf; ++r)
                        s[r / 16][r % 16] = below_maximum(s[r / 16][r % 16], c[i], base);
                    c[i] = 1.0f;
                }
            }
            const float fall = __builtin_amdgcn_exp2f(m - base), both = rescale(m, vr, base, new_vr);
#pragma unroll
            for (int t = 0; t < DT; ++t) acc[t] *= both;
            l *= fall;
            m = new_m;
            vr = new_vr;
        }
        const float origin = large || m == -INFINITY ? 0.0f : m;  // taken from the scores yet
        float add[EXPS], back[EXPS];
        weight_shifts(met, vr, ve, origin, add, back);
#pragma unroll
        for (int i = 0; i < EXPS; ++i) {
            float sum = 0.0f;
#pragma unroll
            for (int r = i * kOf; r < (i + 1) * kOf; ++r) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r / 16][r % 16], c[i], add[i]));
                sum += e;
                w[r / 8][r % 8] = (_Float16)e;
            }
            l += sum * back[i];
        }
        read_exps();  // of the next tile, loaded a tile ago
        turn();
        products(Yes{}, Yes{}, tile + 1);  // the last one's scores are of no tile
    }
    if (!team) turn();
    if (pages.bad()) raise_status(a.status, MP_EINVAL);
    store_rows<D>(k, row, chunk, acc, m, l, vr, h);
}

// The chunks of a row joined, by WAVES waves: one where there are few chunks, four of a
// workgroup where one alone would take many turns.  The chunks' maxima and sums are read by the
// lanes at once, their results four dims a lane and a few chunks at a time.  4-6 us for 2048 rows of
// 8-64 chunks: the launch and three dependent loads.
template <int D, int WAVES>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttend k) {
    constexpr int LANES = D / 4, SIDE = kWave / LANES;  // lanes of a chunk, chunks side by side
    __shared__ __align__(16) float so[4][D];
    const KvArgs& a = k.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int heads = k.group * a.c.heads;
    const uint32_t index = WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
    if (index >= (uint64_t)a.s.n_tokens * heads) return;
    const uint32_t token = index / heads;
    const Partials p = partials(k);
    const int32_t n_chunks = (int32_t)k.shape.n_chunks;
    const float4_t* const sums = p.sums + (int64_t)index * n_chunks;
    const float* const o = p.o + (int64_t)index * n_chunks * D;
    // read beside the sequence's length: the first chunks' sums, written or not
    const float4_t first = sums[min(lane, n_chunks - 1)];
    int64_t of;
    const KvSeq q = kv_find(a, token, [&](int64_t b, int64_t) { return b; }, &of);
    const bool ok = q.ok && token >= q.begin && token < q.begin + q.n;
    if (!ok) return;  // the same for all waves of a row
    // chunks that the row's last position reaches (one at least), or all of a block list
    const int64_t seen = k.blocks ? (int64_t)k.keep << a.log_block
                                  : (int64_t)q.length - (q.n - 1 - (token - q.begin));
    const int32_t chunks = (int32_t)min((int64_t)n_chunks, max((int64_t)1, (seen + k.shape.chunk - 1) / k.shape.chunk));
    float top = -INFINITY;
    if (lane < chunks) top = first[0];
    for (int32_t c = lane + kWave; c < chunks; c += kWave) top = fmaxf(top, sums[c][0]);
    top = wave_reduce(top, OpMax<float>());
    const float base = top == -INFINITY ? 0.0f : top;
    // the chunks' values at one power
    float power = -INFINITY;
    if (lane < chunks) power = (first[0] - base) + first[2];
    for (int32_t c = lane + kWave; c < chunks; c += kWave) power = fmaxf(power, (sums[c][0] - base) + sums[c][2]);
    power = wave_reduce(power, OpMax<float>());
    if (power == -INFINITY) power = 0.0f;
    const int side = lane / LANES, d = lane % LANES * 4;
    float4_t x = {0, 0, 0, 0};
    float total = 0.0f;
    for (int32_t c0 = 0; c0 < chunks; c0 += kWave) {
        const int32_t mine = c0 + lane;
        float w = 0.0f;
        if (mine < chunks) {
            const float4_t of = c0 == 0 ? first : sums[mine];
            total += of[1] * __builtin_amdgcn_exp2f(of[0] - base);
            w = __builtin_amdgcn_exp2f((of[0] - base) + of[2] - power);
        }
        const int32_t here = min(kWave, chunks - c0);
        for (int32_t c = (WAVES == 1 ? 0 : wave * SIDE); c < here; c += WAVES * SIDE) {
            // a place past the last chunk has no weight, and reads the last one
            const int32_t at = min(c + side, here - 1);
            const float f = __shfl(w, min(c + side, kWave - 1), kWave);
            x += (c + side < here ? f : 0.0f) * *reinterpret_cast<const float4_t*>(o + (int64_t)(c0 + at) * D + d);
        }
    }
    total = wave_reduce(total, OpAdd<float>());
#pragma unroll
    for (int i = LANES; i < kWave; i <<= 1)
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] += __shfl_xor(x[j], i, kWave);
    if (WAVES > 1) {
        if (side == 0) *reinterpret_cast<float4_t*>(&so[wave][d]) = x;
        __syncthreads();
        if (wave > 0) return;
        x = float4_t{0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < 4; ++w) x += *reinterpret_cast<const float4_t*>(&so[w][d]);
    }
    // a row that sees nothing: weights and sums are zero
    const float norm = (total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total) * __builtin_amdgcn_exp2f(power);
    if (side == 0) {
        const float y[4] = {x[0] * norm, x[1] * norm, x[2] * norm, x[3] * norm};
        store_16bit<4>(k.out, token, (int)(index % heads), d, y);
    }
    if (k.lse && lane == 0)
        k.lse[index] = total > 0.0f ? (base + log2f(total)) * kLn2 : total == 0.0f ? -INFINITY : total;
}

// Eight waves where every workgroup has a compute unit of its own: half the steps of each.  16
// sequences of 1-65536 tokens, 64 listed blocks of 64: 43 us with the selection, 49 by four waves.
template <int D, bool INT8, bool LIST>
void launch_rows(const KvAttend& k, dim3 grid, hipStream_t st) {
    if constexpr (D < 256) {
        if (grid.x <= 256) {
            kv_rows_kernel<D, INT8, LIST, 8><<<grid, 512, 0, st>>>(k);
            return;
        }
    }
    kv_rows_kernel<D, INT8, LIST, 4><<<grid, 256, 0, st>>>(k);
}

template <int D, bool INT8>
hipError_t launch_d(const KvAttend& k, hipStream_t st) {
    const KvAttendShape& sh = k.shape;
    const dim3 grid((uint32_t)(sh.units * k.a.c.heads * sh.n_chunks));
    constexpr int kLds = 2 * sizeof(TileLds<D>), kPairLds = 2 * sizeof(TileLds<128>);
    if (sh.form == KvForm::tiles) {
        if (kLds > 65536)
            if (hipError_t e = hipFuncSetAttribute((const void*)kv_tiles_kernel<D, INT8>,
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
                e != hipSuccess)
                return e;
        kv_tiles_kernel<D, INT8><<<grid, 256, kLds, st>>>(k);
    } else if (sh.form == KvForm::pair) {  // heads of 128
        if (k.a.c.block == 64)
            kv_pair_kernel<INT8, 1><<<grid, 512, kPairLds, st>>>(k);
        else
            kv_pair_kernel<INT8, 4><<<grid, 512, kPairLds, st>>>(k);
    } else if (k.blocks) {
        launch_rows<D, INT8, true>(k, grid, st);
    } else {
        launch_rows<D, INT8, false>(k, grid, st);
    }
    return hipGetLastError();
}

template <int D>
void launch_join(const KvAttend& k, hipStream_t st) {
    const int64_t rows = k.a.s.n_tokens * (int64_t)k.group * k.a.c.heads;
    if (k.shape.n_chunks > 16)
        kv_join_kernel<D, 4><<<dim3((uint32_t)rows), 256, 0, st>>>(k);
    else
        kv_join_kernel<D, 1><<<dim3((uint32_t)((rows + 3) / 4)), 256, 0, st>>>(k);
}

hipError_t launch_8bit(const KvAttend& k, hipStream_t st) {
    const bool i8 = k.a.c.kind == MP_KV_INT8;
    switch (k.a.c.dim) {
        case 64: return i8 ? launch_d<64, true>(k, st) : launch_d<64, false>(k, st);
        case 128: return i8 ? launch_d<128, true>(k, st) : launch_d<128, false>(k, st);
        default: return i8 ? launch_d<256, true>(k, st) : launch_d<256, false>(k, st);
    }
}

}  // namespace

hipError_t launch_kv_join(const KvAttend& k, hipStream_t st) {
    switch (k.a.c.dim) {
        case 64: launch_join<64>(k, st); break;
        case 128: launch_join<128>(k, st); break;
        default: launch_join<256>(k, st);
    }
    return hipGetLastError();
}

// Chunks of a sequence for tiles in 4 bits: one, or as many as nearly fill up to four rounds of workgroups, by the
// estimated time.  A last round that is not full takes `alone` of a full one and as much of the rest as it is full: its
// workgroups have a compute unit to themselves.  Every chunk writes its rows' results in 32 bits, which the join
// reads.  Sequences of different lengths do not have all chunks: one round of them would not be even; with heads of
// 64, rounds are not even either, and four workgroups a compute unit it is.  us, by four a unit always and by this, 32
// query heads over 8:
//   333 rows after 20000 tokens, heads of 64 105, 98; of 128, 16-bit floats 195, 169 (12 and 5 chunks); 3 such
//   sequences, bfloat16 442, 416; 200 rows, heads of 256 427, 365; 64 rows each of 16 sequences of 8000 195, 177;
//   4 sequences of 2048 tokens, 700 new, heads of 64 111, 62 (one chunk), of 128 172, 113, of 256 437, 312; one of
//   2048, all new, 105, 64; 16 new rows of each of 32 sequences of 1000 tokens, heads of 64, 24 in one chunk, 32 in three.
// Chunks of 128 tokens at least: 100 rows after 412 tokens 20 us in one chunk, 16 by this; 33 rows of 4 sequences of
// 4000 tokens, 8 query heads over 2 of 256, 56 in chunks of 512 and 42.
static int64_t kv4_tile_chunks(const mp_kv_cache& c, const mp_kv_seqs& s, int32_t q_heads,
                               int32_t dtype, int64_t units) {
    const int64_t group = q_heads / c.heads;
    int64_t groups = (std::min(s.most_new, s.n_tokens) * group + 127) / 128;  // of a sequence, and of all
    groups = (s.n_seqs > 0 && groups > units / s.n_seqs ? units : std::max<int64_t>(groups * s.n_seqs, 1)) * c.heads;
    const int64_t places = 256 * (c.dim == 256 ? 1 : c.dim == 128 ? 2 : dtype == MP_F16 ? 3 : 4);
    const double alone = c.dim == 256 ? 1.0 : c.dim == 128 ? 0.6 : dtype == MP_F16 ? 0.4 : 0.3;
    const double work = 4.0 * 128 * groups * s.longest * c.dim / (c.dim == 256 ? 5e8 : 8e8);  // us
    const double join = 8.0 * s.n_tokens * q_heads * (c.dim + 4) / 4.9e6;
    int64_t best = 1;
    double least = 0;
    for (int64_t round = 0; round <= 4; ++round) {
        int64_t chunks = round == 0 ? 1 : round * places / groups;
        if (round > 0 && s.n_seqs > 1) {
            if (c.dim > 64 ? round == 1 : round > 1) continue;
            if (c.dim == 64) chunks = (4 * 256 + units * c.heads - 1) / (units * c.heads);
        }
        if (chunks < 1) continue;
        chunks = std::min(chunks, std::max<int64_t>(s.longest / 128, 1));
        const double full = (double)(groups * chunks) / places, rest = full - floor(full);
        const double cost = work / full * (floor(full) + (rest > 0 ? alone + (1 - alone) * rest : 0)) +
                            (chunks > 1 ? 5 + join * chunks : 0) + 3 * std::max(full, 1.0);
        if (round == 0 || cost < least) best = chunks, least = cost;
    }
    return best;
}

KvAttendShape kv_attend_shape(const mp_kv_cache& c, const mp_kv_seqs& s, int32_t q_heads,
                              int64_t keep, int32_t dtype) {
    KvAttendShape sh = {};
    const int64_t group = q_heads / c.heads;
    // The form by the rows of the longest piece (new tokens times query heads a key head).  Rows against
    // tiles, us, query heads 4 a key head, dim 128: 64 sequences of 1-5000 tokens, 5 new 57 / 134; 4
    // of them, 16 new 29 / 30, 32 new 38 / 31.  A short piece of a short sequence (64 of 16 tokens,
    // all new: 19 / 12) has little to share between row groups.
    // Tiles against pairs, us, 8 key heads, new tokens of each sequence of 2048 (or 8192) tokens:
    //             512 new      1024 new     2048 new     2048 of 8192
    //   1 seq.    46 / 44      79 / 75      107 / 131    339 / 298
    //   4         125 / 143    132 / 211    183 / 168    1063 / 870
    //   16        302 / 269    522 / 458    745 / 672    4424 / 3539
    //   64        1284 / 1112  2222 / 1933  3156 / 2824
    // So a pair's workgroup, alone on its compute unit, wins by 10-20% where there are many of them and
    // loses where about one or two a compute unit are left to end alone (256 and 512 workgroups: the two
    // entries at which this rule, 4096 rows, picks the slower form).  Shorter pieces gain by pairs only with
    // over 1000 workgroups of long sequences (16 of 8192 tokens, 100 new: 387 / 352), and lose otherwise
    // (64 of 2048, 32 new: 98 / 167; of 512, all new: 310 / 361).
    const int64_t piece = (s.most_new < s.n_tokens ? s.most_new : s.n_tokens) * group;
    // In 4 bits tiles take little chunks too.  Rows against tiles, us, 32 query heads over 8, heads of 64, 128 and 256,
    // bfloat16 (16-bit floats of 256: 137 / 174 and 156 / 207):
    //                                 32 rows                       48 rows                     64 rows
    //   16 sequences of 4096 tokens   35 / 29, 38 / 47, 85 / 127    41 / 36, 52 / 55, 115 / 131  44 / 40, 58 / 58, 133 / 135
    //   64 of 4096                    81 / 75, 120 / 111, 286 / 447 114 / 100, 166 / 137, 393 / 448 136 / 103, 208 / 135, 505 / 451
    //   two of 40000                                                46 / 34, 62 / 61, 129 / 152  49 / 38, 67 / 63, 154 / 157
    const int64_t most_by_rows = c.kind != MP_KV_E2M1 || (c.dim == 256 && dtype == MP_F16) ? 64 : 48;
    if (keep > 0 || !s.begin || piece <= 16 || (piece <= most_by_rows && s.longest > 512))
        sh.form = KvForm::rows;
    else
        sh.form = c.dim == 128 && piece >= 4096 ? KvForm::pair : KvForm::tiles;
    // In 4 bits pairs are for bfloat16 rows (16-bit floats would want registers for both forms of their tiles) and for
    // launches of four rounds of workgroups.  Tiles against pairs, us, as above:
    //             1024 new     2048 new     2048 of 8192
    //   1 seq.    69 / 76      64 / 132     277 / 310
    //   4         122 / 213    169 / 168    970 / 860
    //   16        485 / 465    680 / 672
    if (c.kind == MP_KV_E2M1 && sh.form == KvForm::pair &&
        (dtype != MP_BF16 || (s.n_tokens * group / 256 + s.n_seqs) * c.heads < 1024))
        sh.form = KvForm::tiles;
    sh.rows = sh.form == KvForm::rows ? 16 : sh.form == KvForm::tiles ? 128 : 256;
    const int64_t per = (group + sh.rows - 1) / sh.rows;
    if (keep > 0)
        sh.units = s.n_tokens * per;
    else if (s.begin)
        sh.units = s.n_tokens * group / sh.rows + s.n_seqs;
    else
        sh.units = s.n_seqs * per;
    if (c.kind == MP_KV_E2M1 && sh.form == KvForm::rows && s.begin) {
        // (most_new may be anything: no product of it)
        if (s.n_seqs > 1 && s.most_new > 0 && s.n_tokens % s.n_seqs == 0 && s.n_tokens / s.n_seqs == s.most_new) {
            sh.each = (uint32_t)piece;
            sh.units = s.n_seqs * ((piece + 15) / 16 + 1);
        }
        sh.units |= sh.each ? 0 : 1;  // for `spread`
    }
    const int64_t longest = keep > 0 ? keep * c.block : s.longest;
    // Tokens of a workgroup: a workgroup's start, end and part of the join cost as much as some
    // hundred tokens, few long ones leave compute units idle.  2048, or less where that makes
    // fewer workgroups than compute units, 512 at least and all in one up to 1024.  Measured with
    // 512 / 1024 / 2048 / 4096: 64 sequences of 1-16384 tokens 155 / 146 / 149 / 157 us, of 8192
    // each 196 / 186 / 182 / 179, one of 4000 13 / 16 / 21 / 28, 32 of 1-1000 17 / 13 / 13 / 13.
    // Tiles are split only as far as four workgroups a compute unit need it (in 4 bits: as above): a piece of 333 rows
    // after 20000 tokens 118 us (two: 149, eight: 114), prompts that fill the device without
    // chunks 290 us (559 in chunks of 2048: the partial results are 32-bit).
    const int64_t wide = sh.units * c.heads;
    // In 4 bits by the row groups that there are where all sequences have alike: the bound counts one too many of
    // each.  64 sequences of 4096 tokens, 4 new: 80 us, 93 by the bound, in two chunks.
    int64_t busy = wide;
    if (c.kind == MP_KV_E2M1 && sh.form == KvForm::rows && s.begin) {
        const int64_t least = s.n_tokens * group / sh.rows;
        busy = (least > s.n_seqs ? least : s.n_seqs) * c.heads;
        if (sh.each) busy = s.n_seqs * ((piece + 15) / 16) * c.heads;
    }
    int64_t chunk = longest < ((int64_t)2048 * 256) / (busy > 0 ? busy : 1) ? longest * busy / 256 : 2048;
    // In 4 bits two workgroups a compute unit are one round of a launch: where chunks up to 4096 make that
    // many, those.  Measured with 1024 / 2048 / 4096: two sequences of 131072 75 / 63 / 59 us; 64 of 1-16384 tokens,
    // which are more, 104 / 95 / 99.
    if (c.kind == MP_KV_E2M1 && busy > 0 && chunk == 2048 && longest <= (int64_t)4096 * 512 / busy)
        chunk = longest * busy / 512;
    if (chunk < 512) chunk = 512;
    if (longest <= 1024) chunk = 1024;
    if (sh.form != KvForm::rows) {
        int64_t chunks = wide > 0 ? (4 * 256 + wide - 1) / wide : 1;
        if (c.kind == MP_KV_E2M1 && sh.form == KvForm::tiles) chunks = kv4_tile_chunks(c, s, q_heads, dtype, sh.units);
        chunk = (longest + chunks - 1) / chunks;
        if (c.kind != MP_KV_E2M1 && chunk < 512) chunk = 512;
    }
    // a multiple of what the waves of a workgroup take together
    const int64_t together = c.kind == MP_KV_E2M1 && sh.form != KvForm::rows ? 128 : 256;
    sh.chunk = (std::max<int64_t>(chunk, together) + together - 1) / together * together;
    sh.n_chunks = longest > 0 ? (longest + sh.chunk - 1) / sh.chunk : 1;
    const int64_t rows = s.n_tokens * q_heads, most = INT32_MAX;
    // the product of workgroups and chunks may be past 64 bits
    sh.ok = rows < most && wide < most && (wide == 0 || sh.n_chunks <= most / wide) &&
            grid_ok(wide * sh.n_chunks, sh.form == KvForm::pair ? 512 : 256);
    if (sh.ok && sh.n_chunks > 1)
        sh.ok = sh.n_chunks > 16 ? grid_ok(rows, 256) : grid_ok((rows + 3) / 4, 256);
    sh.workspace = sh.ok && sh.n_chunks > 1 ? (size_t)rows * sh.n_chunks * (c.dim + 4) * 4 : 0;
    // a level of a row group (the rows before it over the group's) has 30 bits
    sh.ordered = sh.form != KvForm::rows && s.begin && s.n_seqs <= 64 && sh.n_chunks == 1 &&
                 s.longest < ((int64_t)1 << 30) * sh.rows / group;
    // The bound on the row groups has an empty one for most sequences, and workgroups go to the compute units in
    // turn, wherever others have ended: empty ones at even distances leave some units three and others none.  Where
    // all sequences have as many rows (`each`), the empty ones go last: 64 sequences of 4096 tokens, 4 new, 4 query heads
    // a key head, 51 us, 80 in order; 2 new 52 and 49; 16 sequences, 8 new, 31.  Else neighbours are about 0.618 of the
    // (odd) count apart: these three 63, 60 and 39.
    sh.spread = 1;
    if (s.begin && sh.units > 2 && sh.units < most) {
        const auto common = [](int64_t a, int64_t b) {
            while (b) {
                const int64_t r = a % b;
                a = b, b = r;
            }
            return a;
        };
        int64_t step = sh.units * 618 / 1000;
        while (common(sh.units, step) != 1) ++step;
        sh.spread = (uint32_t)step;
    }
    return sh;
}

hipError_t launch_kv_attend(const KvAttend& k, hipStream_t st) {
    if (k.a.s.n_tokens == 0) return hipSuccess;
    const hipError_t e = k.a.c.kind == MP_KV_E2M1 ? launch_kv4_attend(k, st) : launch_8bit(k, st);
    if (e != hipSuccess || k.shape.n_chunks == 1) return e;
    return launch_kv_join(k, st);
}

}  // namespace mp
