// Attention over the 4-bit key/value cache.
//
// For a row (a query and one of its heads) with scores s_j = scale * q.k_j,
//   out = sum_j 2^(c s_j - M - 24) v_j / sum_j 2^(c s_j - M - 24),   c = log2 e, M = max_j c s_j,
// in one pass over the cache with a running M: when it grows, what was summed so far is multiplied
// by 2^(M_old - M_new).
//
// A code times its group's scale has two significant bits: exact in bfloat16, whose exponents hold every
// scale.  So both products are matrix instructions on bfloat16 with 32-bit sums, and no scale is
// left to be followed: sizes that differ between tokens, groups or blocks cost nothing.  Queries are
// brought to [2^-4, 2^-3) by a power of two per row, and weights lie 24 powers below one, so that no product
// leaves the range of 32-bit floats.  A 16-bit float query is two bfloat16 pieces, which hold it
// exactly, and a weight two pieces (16 bits), where few rows share what is read and the products are
// free beside it.  In tiles, whose time is the products', a weight has as many bits as the results: one piece
// (8 bits) of bfloat16 rows; of rows of 16-bit floats such a float (11 bits), which takes codes and queries
// as such floats too, as far as these hold them.
//
// The instructions that take codes of 4 bits with their scales as they are were not used: beside 8-bit factors
// of different sizes their sums are off by up to 2^-11 of the largest product.
//
// Both products are taken transposed, S^T = K Q^T and O^T = V^T W^T: the weights come out of the first
// in the lanes that the second one wants them in.
#include "kv_attend.hpp"

namespace mp {

namespace {

typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf8_t __attribute__((ext_vector_type(8)));
typedef short short4_t __attribute__((ext_vector_type(4)));

constexpr int kStep = 64;           // tokens a wave takes at a time
constexpr float kBelow = 24.0f;     // of a row's largest weight below one, in powers of two
constexpr int kQueryExp = -4;       // of a row's largest query value
constexpr int kKeyDown = 19;        // as 16-bit floats these are at 2^15, and keys this many powers smaller
// How far the largest weight may grow above that before the running maximum follows: bfloat16 weights
// lose no bits by it.
constexpr float kSlack = 6.0f;
// The exponent of a weight is one multiply-add, c s - (M + 24), which is off a rounded M by half of its last place.
// Scores beyond this are rounded first, so that none is above its maximum by more than that may lag.
constexpr float kLargeScore = 0x1p16f;

// c s, and c s - m with the product rounded by itself.
__device__ __forceinline__ float score_of(float s, float c) {
#pragma clang fp contract(off)
    return s * c;
}
__device__ __forceinline__ float below_maximum(float s, float c, float m) {
#pragma clang fp contract(off)
    return s * c - m;
}

// A row's running maximum of c s: with the shift, M + 24, which weights are 2^(c s - m) below; or, once some
// maximum of the wave is large (`far`), M itself.
struct Maximum {
    float m = -INFINITY;
    bool far = false;
};
// It follows `top`, the largest of these scores, where it is more than `lag` behind.  Then `fall(f)` has to multiply
// what was summed by f.  Weights are 2^(*c s - *from) afterwards, `shift` powers below one at the maximum; where it is
// far `lower(c, m)` has to replace scores s by c s - m, and *c is one.
template <typename Fall, typename Lower>
__device__ __forceinline__ void follow(float top, float shift, float lag, Maximum* at, float* c, float* from, Fall fall,
                                       Lower lower) {
    const float new_m = fmaxf(at->m, top * *c + (at->far ? 0.0f : shift));
    if (__any(new_m - at->m > lag)) {
        fall(__builtin_amdgcn_exp2f(at->m - (new_m == -INFINITY ? 0.0f : new_m)));
        const bool large = __any(fabsf(new_m) > kLargeScore && fabsf(new_m) < INFINITY);
        at->m = large && !at->far ? new_m - shift : new_m;
        at->far = at->far || large;
    }
    *from = at->m == -INFINITY ? 0.0f : at->m;
    if (at->far) {
        const float m = fmaxf(at->m, score_of(top, *c)), base = m == -INFINITY ? 0.0f : m;
        fall(__builtin_amdgcn_exp2f(at->m - base));
        at->m = m;
        lower(*c, base);
        *c = 1.0f, *from = shift;
    }
}
// For results that are joined: the maximum's part in the sums, and the power of two that is left to them.
__device__ __forceinline__ float left_of(const Maximum& at, float shift) { return at.far ? shift : 0.0f; }

union Words8 {
    uint32_t w[4];
    bf8_t v;
};

// Two codes (byte SEL of w) at their scale as bfloat16, the lower one low.
template <int SEL>
__device__ __forceinline__ uint32_t pair_of(uint32_t w, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}
// Eight codes the same way.
__device__ __forceinline__ bf8_t codes_to_bf(uint32_t w, float scale) {
    Words8 o;
    o.w[0] = pair_of<0>(w, scale);
    o.w[1] = pair_of<1>(w, scale);
    o.w[2] = pair_of<2>(w, scale);
    o.w[3] = pair_of<3>(w, scale);
    return o.v;
}
// Byte `at` of w as the scale that it stands for.
__device__ __forceinline__ float scale_of(uint32_t w, int at) {
    return __uint_as_float((w >> (8 * at) & 0xffu) << 23);
}

// Eight values as bfloat16: their upper halves, and what these leave.
__device__ __forceinline__ void split8(const float* x, bf8_t* hi, bf8_t* lo) {
    Words8 h, l;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t a = __float_as_uint(x[2 * i]), b = __float_as_uint(x[2 * i + 1]);
        h.w[i] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        const float ra = x[2 * i] - __uint_as_float(a & 0xffff0000u);
        const float rb = x[2 * i + 1] - __uint_as_float(b & 0xffff0000u);
        const bf2_t r = {(__bf16)ra, (__bf16)rb};
        l.w[i] = __builtin_bit_cast(uint32_t, r);
    }
    *hi = h.v;
    *lo = l.v;
}
__device__ __forceinline__ bf8_t round8(const float* x) {
    Words8 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf2_t r = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
        o.w[i] = __builtin_bit_cast(uint32_t, r);
    }
    return o.v;
}

// Eight codes at their scale as 16-bit floats, eight values as these, and the product of such or of bfloat16.
__device__ __forceinline__ uint4 codes_to_f16(uint32_t w, float scale) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3)));
}
__device__ __forceinline__ Words8 half8(const float* x) {
    Words8 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const half2_t r = __builtin_convertvector((float2_t{x[2 * i], x[2 * i + 1]}), half2_t);
        o.w[i] = __builtin_bit_cast(uint32_t, r);
    }
    return o;
}
template <bool F16>
__device__ __forceinline__ float16_t product(const Words8& a, const Words8& b, float16_t c) {
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, a), __builtin_bit_cast(half8_t, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
}

// What brings a row's query, `top` its largest value, to the size that it has as a factor of the first product:
// 2^up and the scale's sign (zero for one of zero); and what the scores are multiplied by then, not negative.
struct QueryScale {
    int up;
    float sign, c;
};
__device__ __forceinline__ QueryScale query_scale(const KvAttend& k, float top) {
    uint32_t frac;
    const int e = min(127, max(-90, exponent_of(top, &frac) - 1));  // 2^e <= top < 2^(e + 1)
    const float size = fabsf(k.scale);  // its fraction and exponent are those of the smallest floats too
    const int ec = __builtin_amdgcn_frexp_expf(size);
    // c is no less than 2^-126, so that it is not zero beside a masked score's infinity: for a scale so small beside
    // large keys the query gives way, and all of it for a scale of zero
    const int up = min(kQueryExp - e, ec + 125);
    const float c = __builtin_ldexpf(__builtin_amdgcn_frexp_mantf(size) * kLog2e, ec - up);
    return {up, size == 0.0f ? 0.0f : k.scale < 0.0f ? -1.0f : 1.0f, fminf(fmaxf(c, 1.17549435e-38f), 3.4e38f)};
}
// Values of a query as factors of the first product (PIECES of them); *scale as above.
template <int PIECES, int N>
__device__ __forceinline__ void query_pieces(const KvAttend& k, const float (&x)[N][8], float top,
                                             bf8_t (&q)[PIECES][N], float* scale) {
    const QueryScale by = query_scale(k, top);
    const float f = pow2f(by.up / 2), f2 = by.sign * pow2f(by.up - by.up / 2);  // 2^-131 is no float's least power
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = x[i][j] * f * f2;
        if constexpr (PIECES == 1)
            q[0][i] = round8(y);
        else
            split8(y, &q[0][i], &q[1][i]);
    }
    *scale = by.c;
}

// Few rows: 16 columns of rows, one key head, one chunk of tokens.  Each of four or eight waves takes
// every fourth or eighth step of 64 tokens, with its own running maxima, and they are joined at the
// end.  A wave reads the codes straight into registers; nothing is shared, so there is no barrier in the loop
// and what hides the latency is the other waves of the SIMD.
//
// Tokens: key row n of tile t holds token 4 n + t of the step, lane quarter g a quarter of its dims.  A lane
// of quarter g then has the scores of tokens [16 g, + 16), four in a row from the four tiles.  Of the
// values it reads those tokens' dims [D/16 n, + D/16): row n of the second product's tile t is dim D/16 n + t.
// The instructions that convert take two dims of a token, those that multiply want two tokens of a dim: a byte
// permute a pair turns them, two dims at a time, which keeps the factors' registers few.
//
// What bounds it is memory where there are many workgroups: 64 sequences of 1-16384 tokens 90 us, 4.3 TB/s, of 8192
// each 116 us, 4.9 TB/s; two of 131072 58 us, 4.9 TB/s (a large copy: 4.9).  A step of 64 tokens has 350 vector and 48
// matrix instructions a wave, about half of the time that its 8.7 KB take.  It was 112 and 105 us with registers
// spilled at three waves a SIMD: heads of 128 have three with bfloat16 rows, two with 16-bit floats (whose queries take
// 16 registers more).  One sequence of 1000 tokens 10 us: dependent loads, two steps a wave, and code met for
// the first time.
template <int D, int PIECES, int WAVES>
__global__ __launch_bounds__(WAVES * 64, D == 256 ? 1 : WAVES == 8 || (D == 128 && PIECES == 2) ? 2 : 3) void kv4_rows_kernel(KvAttend k) {
    constexpr int KD = D / 4, KS = KD / 8;  // dims of a lane's keys; steps of the first product
    constexpr int VD = D / 16;              // dims of a lane's values
    constexpr int KE = D == 256 ? 2 : 1;    // scales of a lane's dims of a key
    __shared__ __align__(16) float so[WAVES][16][D + 4];
    __shared__ float sm[WAVES][16], sl[WAVES][16];
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const KvArgs& a = k.a;
    if (blockIdx.x == 0) kv_check_begin(a);
    const uint32_t heads = a.c.heads, n_chunks = (uint32_t)k.shape.n_chunks;
    const int head = (int)(blockIdx.x % heads);
    // chunks slowest: workgroups go to the XCDs in turn, and first chunks, which every row group
    // has, must not all meet one of them; last chunks first, which only long sequences have
    const uint32_t rest = blockIdx.x / heads;
    uint32_t chunk, unit;
    if (const uint32_t each = k.shape.each) {
        // row groups that sequences of `each` rows have, then, of all chunks, those that are empty if they do
        const uint32_t per = (each + 15) / 16, n_seqs = (uint32_t)a.s.n_seqs, all = n_seqs * per;
        const bool had = rest < all * n_chunks;
        const uint32_t r = had ? rest : rest - all * n_chunks, of = had ? all : n_seqs, u = r % of;
        const uint32_t s = had ? u / per : u;
        chunk = n_chunks - 1 - r / of;
        const auto first = [&](uint32_t i) { return (uint32_t)((uint64_t)i * each / 16) + i; };
        unit = first(s) + (had ? u - s * per : per);
        if (!had && unit >= first(s + 1)) return;
    } else {
        const uint32_t units = (uint32_t)k.shape.units;
        chunk = n_chunks - 1 - rest / units;
        unit = (uint32_t)((uint64_t)(rest % units) * k.shape.spread % units);
    }
    RowGroup rg;
    if (!row_group<16>(k, unit, &rg)) return;
    const int64_t last_row = min((int64_t)rg.n_rows, rg.row0 + 16) - 1;
    const int32_t most = wave_one(row_of(k, rg, head, last_row).last);  // the last position any row sees
    const int32_t least = wave_one(row_of(k, rg, head, rg.row0).last);  // all rows see up to here
    const int lb = a.log_block, block = 1 << lb;
    const int64_t start = chunk * k.shape.chunk, end_all = (int64_t)most + 1;
    if (chunk > 0 && start >= end_all) return;
    const int32_t x1 = (int32_t)min(end_all, start + k.shape.chunk);

    Pages pages = {a.s.table + rg.q.s * a.s.table_stride, (uint32_t)max(most, 0) >> lb,
                   (uint32_t)a.c.n_blocks, 0};
    const uint32_t page_size = heads * (uint32_t)(D / 2) << lb, exp_size = heads * (uint32_t)(D / 32) << lb;
    const int k_slot = (((n >> 2) * 16) & (block - 1)) + (n & 3) * 4, v_slot = (g * 16) & (block - 1);
    const uint32_t k_at = (((uint32_t)head << lb) + k_slot) * (D / 2) + g * (KD / 2);
    const uint32_t v_at = (((uint32_t)head << lb) + v_slot) * (D / 2) + n * (VD / 2);
    const uint32_t ke_at = (((uint32_t)head * (D / 32) + g * KD / 32) << lb) + k_slot;
    const uint32_t ve_at = (((uint32_t)head * (D / 32) + n * VD / 32) << lb) + v_slot;
    uint32_t kw[4][KS], vw[16][VD > 8 ? 2 : 1], ke[KE];
    uint4 ve;
    uint32_t k_entry = 0, v_entry = 0;
    auto find = [&](int32_t x) {
        k_entry = pages.entry((uint32_t)(x + (n >> 2) * 16) >> lb);
        v_entry = pages.entry((uint32_t)(x + g * 16) >> lb);
    };
    auto load_keys = [&]() {
        const uint64_t page = pages.page(k_entry);
        const uint8_t* const p = a.c.k_code + (page * page_size + k_at);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if constexpr (KS == 2) {
                const uint2 w = *reinterpret_cast<const uint2*>(p + t * (D / 2));
                kw[t][0] = w.x, kw[t][1] = w.y;
            } else {
#pragma unroll
                for (int c = 0; c < KS / 4; ++c) {
                    const uint4 w = *reinterpret_cast<const uint4*>(p + t * (D / 2) + c * 16);
                    kw[t][4 * c] = w.x, kw[t][4 * c + 1] = w.y, kw[t][4 * c + 2] = w.z, kw[t][4 * c + 3] = w.w;
                }
            }
        }
        const int8_t* const e = a.c.k_exp + (page * exp_size + ke_at);
#pragma unroll
        for (int i = 0; i < KE; ++i) ke[i] = *reinterpret_cast<const uint32_t*>(e + (i << lb));
    };
    auto load_values = [&]() {
        const uint64_t page = pages.page(v_entry);
        const uint8_t* const p = a.c.v_code + (page * page_size + v_at);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            if constexpr (VD == 4) {
                vw[j][0] = *reinterpret_cast<const uint16_t*>(p + j * (D / 2));
            } else if constexpr (VD == 8) {
                vw[j][0] = *reinterpret_cast<const uint32_t*>(p + j * (D / 2));
            } else {
                const uint2 w = *reinterpret_cast<const uint2*>(p + j * (D / 2));
                vw[j][0] = w.x, vw[j][1] = w.y;
            }
        }
        ve = *reinterpret_cast<const uint4*>(a.c.v_exp + (page * exp_size + ve_at));
    };
    const Row row = row_of(k, rg, head, rg.row0 + n);
    int32_t x = (int32_t)start + wave * kStep;
    const int32_t stride = WAVES * kStep;
    uint4 raw[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) raw[i] = load8_16bit(k.q, row.token, row.head, g * KD + i * 8);
    if (x < x1) {
        find(x);
        load_keys();
        load_values();
        if (x + stride < x1) find(x + stride);
    }
    bf8_t q[PIECES][KS];
    float c;
    {
        float y[KS][8], top = 0.0f;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            to_float8(k.q, raw[i], y[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(y[i][j]));
        }
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        query_pieces<PIECES>(k, y, top, q, &c);
    }
    float4_t acc[VD];
    Maximum at;
    float l = 0.0f;
#pragma unroll
    for (int t = 0; t < VD; ++t) acc[t] = float4_t{0, 0, 0, 0};

    for (; x < x1; x += stride) {
        float s[16];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            float4_t z = {0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const bf8_t f = codes_to_bf(kw[t][i], scale_of(ke[i * KE / KS], t));
#pragma unroll
                for (int p = 0; p < PIECES; ++p)
                    z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, q[p][i], z, 0, 0, 0);
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) s[4 * r + t] = z[r];
        }
        const bool more = x + stride < x1;
        if (more) load_keys();
        if (x + kStep - 1 > least) {  // some row does not see some token of the step
            const int seen = row.last - x - g * 16;
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = i > seen ? -INFINITY : s[i];
            // places past the end may hold anything: a scale of one makes their values finite
            const int held = most - x - g * 16;
            uint32_t e[4] = {ve.x, ve.y, ve.z, ve.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t keep = (uint32_t)(((uint64_t)1 << (8 * min(4, max(0, held + 1 - 4 * i)))) - 1);
                e[i] = (e[i] & keep) | (0x7f7f7f7fu & ~keep);
            }
            ve = make_uint4(e[0], e[1], e[2], e[3]);
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
        top = fmaxf(top, __shfl_xor(top, 16, kWave));
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        float by = c, from;
        follow(top, kBelow, kSlack, &at, &by, &from,
               [&](float fall) {
#pragma unroll
                   for (int t = 0; t < VD; ++t) acc[t] *= fall;
                   l *= fall;
               },
               [&](float scale, float base) {
#pragma unroll
                   for (int i = 0; i < 16; ++i) s[i] = below_maximum(s[i], scale, base);
               });
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], by, -from));
            l += s[i];
        }
        const uint32_t e[4] = {ve.x, ve.y, ve.z, ve.w};
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            bf8_t hi, lo;
            split8(s + 8 * half, &hi, &lo);
            float scale[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) scale[j] = scale_of(e[2 * half + j / 4], j % 4);
            // two dims at a time: of each token a byte, of two tokens' bytes each dim's pair
            const auto dims = [&](auto sel, int word, int d) {
                Words8 f[2];
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const uint32_t ta = pair_of<decltype(sel)::value>(vw[8 * half + j][word], scale[j]);
                    const uint32_t tb = pair_of<decltype(sel)::value>(vw[8 * half + j + 1][word], scale[j + 1]);
                    f[0].w[j / 2] = __builtin_amdgcn_perm(tb, ta, 0x05040100u);
                    f[1].w[j / 2] = __builtin_amdgcn_perm(tb, ta, 0x07060302u);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    acc[d + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i].v, hi, acc[d + i], 0, 0, 0);
                    acc[d + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[i].v, lo, acc[d + i], 0, 0, 0);
                }
            };
#pragma unroll
            for (int word = 0; word < (VD > 8 ? 2 : 1); ++word) {
                dims(std::integral_constant<int, 0>(), word, 8 * word);
                dims(std::integral_constant<int, 1>(), word, 8 * word + 2);
                if constexpr (VD >= 8) {
                    dims(std::integral_constant<int, 2>(), word, 8 * word + 4);
                    dims(std::integral_constant<int, 3>(), word, 8 * word + 6);
                }
            }
        }
        if (more) {
            load_values();
            if (x + 2 * (int64_t)stride < x1) find(x + 2 * stride);
        }
    }
    if (pages.bad()) raise_status(a.status, MP_EINVAL);

    // the waves' results of a row joined; a lane has dims [4 VD g, + 4 VD)
    l += __shfl_xor(l, 16, kWave);
    l += __shfl_xor(l, 32, kWave);
    if (g == 0) {
        sm[wave][n] = at.far ? at.m : at.m - kBelow;
        sl[wave][n] = l;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int t = 0; t < VD; t += 4)
            *reinterpret_cast<float4_t*>(&so[wave][n][(4 * g + r) * VD + t]) =
                float4_t{acc[t][r], acc[t + 1][r], acc[t + 2][r], acc[t + 3][r]};
    __syncthreads();
    if (WAVES > 4 && threadIdx.x >= 256) return;
    const int col = threadIdx.x >> 4, d0 = (threadIdx.x & 15) * (D / 16);
    float top = sm[0][col];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) top = fmaxf(top, sm[w][col]);
    const float base = top == -INFINITY ? 0.0f : top;
    float total = 0.0f, o[D / 16];
#pragma unroll
    for (int i = 0; i < D / 16; ++i) o[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const float f = __builtin_amdgcn_exp2f(sm[w][col] - base);
        total += sl[w][col] * f;
#pragma unroll
        for (int i = 0; i < D / 16; i += 4) {
            const float4_t y = *reinterpret_cast<const float4_t*>(&so[w][col][d0 + i]);
#pragma unroll
            for (int z = 0; z < 4; ++z) o[i + z] += y[z] * f;
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
        if (d0 == 0) part_out.sums[index * n_chunks + chunk] = float4_t{top, total * pow2f((int)kBelow), kBelow, 0};
    } else {
        // a row that sees nothing: weights and sums are zero
        const float norm = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) o[i] *= norm;
        constexpr int kOnce = D / 16 >= 8 ? 8 : 4;
#pragma unroll
        for (int i = 0; i < D / 16; i += kOnce) store_16bit<kOnce>(k.out, r.token, r.head, d0 + i, o + i);
        if (k.lse && d0 == 0)
            k.lse[index] = total > 0.0f ? (base + log2f(total * pow2f((int)kBelow))) * kLn2
                                        : total == 0.0f ? -INFINITY : total;
    }
}

// The result of a wave of 32 rows, a column each: lane half h has dims 4 h + [0, 4) of every eight.  Weights
// lie `shift` powers below 2^m.
template <int D>
__device__ __forceinline__ void store_rows(const KvAttend& k, const Row& row, uint32_t chunk,
                                           const float16_t (&acc)[D / 32], float m, float l, float shift, int h) {
    const float total = l + __shfl_xor(l, 32, kWave);
    if (!row.live) return;
    const uint32_t n_chunks = (uint32_t)k.shape.n_chunks;
    // a row that sees nothing: weights and sums are zero
    const float norm = total > 0.0f ? 1.0f / total : total == 0.0f ? 0.0f : total;
    const int64_t index = row.token * (int64_t)k.group * k.a.c.heads + row.head;
    const Partials part_out = partials(k);
    const bool whole = n_chunks == 1;
    const float f = whole ? norm : 1.0f;
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
        const float sum = total * pow2f((int)shift);
        if (!whole)
            part_out.sums[index * n_chunks + chunk] = float4_t{m, sum, shift, 0};
        else if (k.lse)
            k.lse[index] = sum > 0.0f ? (m + log2f(sum)) * kLn2 : sum == 0.0f ? -INFINITY : sum;
    }
}

// Many rows: four waves of 32 rows, one key head, one chunk of tokens, in tiles of 64 tokens whose
// codes the workgroup turns into bfloat16 once, in LDS, for all 128 rows.  Two tiles' room: while one
// is computed the next one's codes, already in registers, are converted into the other and the
// loads of the one after are on their way, so a tile costs one barrier.
//
// Both arrays lie by token, in 16-byte pieces exchanged by the token's low bits, so that the lanes of a
// read meet different banks.  Keys are read along their dims, row n of 32 being token n with bits 2 and 3
// exchanged: a lane's scores are those of eight consecutive tokens, as the second product takes
// them.  Values are read by the transposing loads, 16 lanes of which take four tokens' 16 dims and have
// one dim of the four each.
template <int D>
struct Tile4 {
    uint4 k[64][D / 8];
    uint4 v[64][D / 8];
};
template <int D>
__device__ __forceinline__ int k4_key(int token) {
    return D == 64 ? token >> 1 & 7 : token & 15;
}
template <int D>
__device__ __forceinline__ int v4_key(int token) {
    return D == 64 ? (token >> 1 & 1) << 2 : (token & 3) << 2;
}

// Measured, 333, 127 and 18 rows after 19678, 7516 and 1097 tokens, 4 heads of 64, 7 query heads each, 16-bit floats:
// 98-105 us and the join, 520-560 TFLOP/s.  A tile's softmax takes a wave about 900 cycles of vector instructions (512 of
// them exponentials), its products of heads of 64 512; counted, vector instructions take 64% of the time of the SIMDs
// that work, matrix ones 29%, and compute units stand idle for a quarter of the launch: 800 workgroups of unlike
// lengths for 768 places.  Four sequences of 2048 tokens, 700 new, 32 query heads over 8, bfloat16: heads of 64
// 61 us, of 128 104 us, of 256 312 us; 16-bit floats 66, 113 and 418.
//
// F16, rows of 16-bit floats: the tile as 16-bit floats, so that one instruction holds a query's and a
// weight's 11 bits.  A group of codes that these cannot hold exactly (scales outside 2^-23..2^13, codes not all zero)
// marks its tile, and the workgroup takes a marked tile as bfloat16, with queries and weights in two pieces.  (All tiles
// in two pieces: 143 us, with the join, instead of 112 for the rows above.)  Weights of 16-bit floats lie around 2^10,
// where those have most bits; beside values of scales past 2^13 they would leave the range of the sums, so a workgroup
// that meets such values takes that tile and all after it as bfloat16, weights 24 powers below one.
// Heads of 256 have no registers for both: all their tiles are taken so.
// Heads of 64 have three waves a SIMD (168 registers, three spilled beside the loop); unasked the compiler takes more.
template <int D, bool F16>
__global__ __launch_bounds__(256, D == 256 ? 1 : D == 64 && F16 ? 3 : 2) void kv4_tiles_kernel(KvAttend k) {
    constexpr int KS = D / 16, DT = D / 32, GROUPS = D / 32;
    constexpr int UNITS = 128 * GROUPS / 256;  // groups of 32 dims that a thread moves in a tile, keys first
    constexpr bool kPieces = F16 && D == 256;  // every tile
    constexpr bool kHalves = F16 && !kPieces;  // tiles as 16-bit floats, whose weights reach 2^14, but for marked ones
    constexpr float kShift = kHalves ? -10.0f : kBelow, kLag = kHalves ? 4.0f : kSlack;
    extern __shared__ __align__(16) char lds_raw[];
    Tile4<D>* const lds = reinterpret_cast<Tile4<D>*>(lds_raw);
    __shared__ int32_t marked[2];  // the first token of the last marked tile of each room
    __shared__ int32_t met_large;  // values of a marked tile had a scale past 2^13
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
    const int32_t most = wave_one(row_of(k, rg, head, min((int64_t)rg.n_rows, rg.row0 + 128) - 1).last);
    const int64_t start = chunk * k.shape.chunk;
    if (chunk > 0 && start > most) return;
    const int32_t x0 = (int32_t)start;
    const int32_t x1 = (int32_t)min((int64_t)most + 1, start + k.shape.chunk);

    // this wave's rows: the last position that any sees, and the last that all see
    const int64_t wave_row0 = rg.row0 + 32 * wave;
    const bool awake = wave_row0 < rg.n_rows;
    const int32_t wave_most =
        wave_one(awake ? row_of(k, rg, head, min((int64_t)rg.n_rows, wave_row0 + 32) - 1).last : -1);
    const int32_t wave_least = wave_one(awake ? row_of(k, rg, head, wave_row0).last : -1);
    const Row row = row_of(k, rg, head, wave_row0 + n);

    Words8 q[KS];    // bfloat16 factors, or 16-bit floats, the row's largest from 2^15 on (so these lose no bits)
    float c, c_odd;  // what scores are multiplied by, and those of marked tiles
    {
        uint4 raw[KS];
#pragma unroll
        for (int i = 0; i < KS; ++i) raw[i] = load8_16bit(k.q, row.token, row.head, i * 16 + h * 8);
        if constexpr (F16) {
            half2_t peak = {};
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                q[i].w[0] = raw[i].x, q[i].w[1] = raw[i].y, q[i].w[2] = raw[i].z, q[i].w[3] = raw[i].w;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    peak = __builtin_elementwise_max(peak, __builtin_bit_cast(half2_t, q[i].w[j] & 0x7fff7fffu));
            }
            float top = fmaxf((float)peak[0], (float)peak[1]);
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            // a row of less than 2^-15 stays below 2^15: two factors of such floats are enough
            const QueryScale by = query_scale(k, fminf(fmaxf(top, 0x1p-15f), 65504.0f));
            const int up = by.up + kKeyDown, most_up = min(up, 15);
            const _Float16 f = (_Float16)pow2f(most_up), f2 = (_Float16)(by.sign * pow2f(up - most_up));
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    half2_t x = __builtin_bit_cast(half2_t, q[i].w[j]);
                    x = x * half2_t{f, f} * half2_t{f2, f2};
                    q[i].w[j] = __builtin_bit_cast(uint32_t, x);
                }
            c_odd = by.c;
            c = fmaxf(c_odd * pow2f(-kKeyDown), 1.17549435e-38f);
        } else {
            float y[KS][8], top = 0.0f;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                to_float8(k.q, raw[i], y[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(y[i][j]));
            }
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            bf8_t f[1][KS];
            query_pieces<1>(k, y, top, f, &c);
#pragma unroll
            for (int i = 0; i < KS; ++i) q[i].v = f[0][i];
            c_odd = c;
        }
    }
    // 8 values of the query as a marked tile takes them: two pieces, exact
    const auto odd_query = [&](int i, bf8_t* hi, bf8_t* lo) {
        float y[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t w = q[i].w[j];
            asm volatile("" : "+v"(w));  // made here each time: kept through the loop it would take registers
            pair_to_float(false, w, y + 2 * j);
        }
        split8(y, hi, lo);
    };
    float16_t acc[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = float16_t{};
    Maximum at;
    float l = 0.0f;

    // unit u of a thread: 32 dims of a token's keys or values; table entries are read a tile ahead
    const int lb = a.log_block, block = 1 << lb;
    const uint32_t page_size = heads * (uint32_t)(D / 2) << lb, exp_size = heads * (uint32_t)(D / 32) << lb;
    Pages pages = {a.s.table + rg.q.s * a.s.table_stride, (uint32_t)max(most, 0) >> lb,
                   (uint32_t)a.c.n_blocks, 0};
    const auto is_v = [&](int u) { return u * 256 + tid >= 64 * GROUPS; };
    const auto token_of = [&](int u) { return ((u * 256 + tid) / GROUPS) & 63; };
    const int group = tid % GROUPS;
    uint4 codes[UNITS];
    uint32_t exps[UNITS], entry[UNITS];
    auto find = [&](int32_t x) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) entry[u] = pages.entry((uint32_t)(x + token_of(u)) >> lb);
    };
    auto load = [&]() {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const uint64_t page = pages.page(entry[u]);
            const uint32_t slot = token_of(u) & (block - 1);
            const uint8_t* const from = is_v(u) ? a.c.v_code : a.c.k_code;
            const int8_t* const exp = is_v(u) ? a.c.v_exp : a.c.k_exp;
            codes[u] = *reinterpret_cast<const uint4*>(
                from + (page * page_size + (((uint32_t)head << lb) + slot) * (D / 2) + group * 16));
            exps[u] = (uint8_t)exp[page * exp_size + ((((uint32_t)head * GROUPS + group) << lb) + slot)];
        }
    };
    // the loaded codes (of the tile at x) in LDS; places past the end may hold anything: a scale of one
    // makes their values finite
    auto put = [&](int buf, int32_t x, auto as_f16) {
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int token = token_of(u);
            const uint32_t e = x + token > most ? 127u : exps[u];
            // keys as bfloat16 beside queries of 16-bit floats: these are 2^19 times what bfloat16 ones are
            const uint32_t down = F16 && !decltype(as_f16)::value && !is_v(u) ? kKeyDown : 0;
            const float scale = __uint_as_float((max(e, down) - down) << 23);
            uint4* const to = is_v(u) ? lds[buf].v[token] : lds[buf].k[token];
            const int key = is_v(u) ? v4_key<D>(token) : k4_key<D>(token);
            const uint32_t w[4] = {codes[u].x, codes[u].y, codes[u].z, codes[u].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint4 f;
                if constexpr (decltype(as_f16)::value)
                    f = codes_to_f16(w[i], scale);
                else
                    f = __builtin_bit_cast(uint4, codes_to_bf(w[i], scale));
                to[(group * 4 + i) ^ key] = f;
            }
            if constexpr (decltype(as_f16)::value)
                if (e - 104u > 36u && ((w[0] | w[1] | w[2] | w[3]) & 0x77777777u) != 0) marked[buf] = x;
            if constexpr (kHalves && !decltype(as_f16)::value)
                if (is_v(u) && e > 140u && ((w[0] | w[1] | w[2] | w[3]) & 0x77777777u) != 0) met_large = 1;
        }
    };
    using No = std::false_type;
    using AsF16 = std::integral_constant<bool, kHalves>;
    const int k_token = (n & 0x13) | (n & 4) << 1 | (n & 8) >> 1;
    const int v_token = 8 * h + (lane >> 2 & 3), v_dim = (n & 16) + (lane & 3) * 4;

    int buf = 0;
    if (AsF16::value) {
        if (tid < 2) marked[tid] = -1;
        if (tid == 0) met_large = 0;
        __syncthreads();
    }
    if (x0 < x1) {
        find(x0);
        load();
        find(x0 + 64);
        put(0, x0, AsF16());
    }
    bool large = false;    // the same for the workgroup
    float shift = kShift;  // of its weights below one
    // a tile: its scores, weights and products, as 16-bit floats or (ODD) as a marked one
    const auto tile = [&](int32_t x, auto odd) {
        constexpr bool ODD = decltype(odd)::value;
        const float below = ODD ? shift : kShift, lag = ODD && large ? kSlack : kLag;
        float16_t s[2] = {float16_t{}, float16_t{}};
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            bf8_t hi = {}, lo = {};
            if constexpr (ODD) odd_query(i, &hi, &lo);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int token = t * 32 + k_token;
                Words8 f;
                f.v = __builtin_bit_cast(bf8_t, lds[buf].k[token][(i * 2 + h) ^ k4_key<D>(token)]);
                if constexpr (ODD) {
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, hi, s[t], 0, 0, 0);
                    s[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, lo, s[t], 0, 0, 0);
                } else {
                    s[t] = product<F16>(f, q[i], s[t]);
                }
            }
        }
        // register r of product t is token 32 t + 16 (r / 8) + 8 h + r % 8
        if (x + 63 > wave_least) {
            const int seen = row.last - x - h * 8;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[t][r] = t * 32 + (r >> 3) * 16 + (r & 7) > seen ? -INFINITY : s[t][r];
        }
        float by = ODD ? c_odd : c;
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 32; ++r) top = fmaxf(top, s[r / 16][r % 16]);
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        float from;
        follow(top, below, lag, &at, &by, &from,
               [&](float fall) {
#pragma unroll
                   for (int t = 0; t < DT; ++t) acc[t] *= fall;
                   l *= fall;
               },
               [&](float scale, float base) {
#pragma unroll
                   for (int r = 0; r < 32; ++r) s[r / 16][r % 16] = below_maximum(s[r / 16][r % 16], scale, base);
               });
        const auto weights = [&](int i, Words8* w) {
            float e[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][i % 2 * 8 + r], by, -from));
                l += e[r];
            }
            if constexpr (ODD)
                split8(e, &w[0].v, &w[1].v);
            else if constexpr (F16)
                w[0] = half8(e);
            else
                w[0].v = round8(e);
        };
        Words8 w[4], pieces[2];
        if constexpr (!ODD)
#pragma unroll
            for (int i = 0; i < 4; ++i) weights(i, &w[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (ODD) weights(i, pieces);
#pragma unroll
            for (int t = 0; t < DT; ++t) {
                union {
                    short4_t s[2];
                    Words8 f;
                } f;
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const int token = i * 16 + 4 * z + v_token, d = t * 32 + v_dim;
                    auto* const from8 = reinterpret_cast<short4_t*>(&lds[buf].v[token][(d >> 3) ^ v4_key<D>(token)]) + (d >> 2 & 1);
                    f.s[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) short4_t*)from8);
                }
                if constexpr (ODD) {
                    acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.f.v, pieces[0].v, acc[t], 0, 0, 0);
                    acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.f.v, pieces[1].v, acc[t], 0, 0, 0);
                } else {
                    acc[t] = product<F16>(f.f, w[i], acc[t]);
                }
            }
        }
    };
    for (int32_t x = x0;;) {
        // left at a marked tile, so that what it takes is no part of the loop's registers
        for (; x < x1; x += 64, buf ^= 1) {
            if (x + 64 < x1) {
                load();
                find(x + 128);
            }
            __syncthreads();  // the tile is whole; the other one is read no more
            if (AsF16::value && (large || wave_one(marked[buf]) == x)) break;  // the same for the workgroup
            if (x <= wave_most) tile(x, std::integral_constant<bool, kPieces>());
            if (x + 64 < x1) put(buf ^ 1, x + 64, AsF16());
        }
        if (!AsF16::value || x >= x1) break;
        // the tile once more, then the next one's codes
        find(x);
        load();
        put(buf, x, No());
        __syncthreads();
        if (!large && wave_one(met_large) != 0) {  // not written again before the next tile's barrier
            constexpr float kFall = 0x1p-34f;
            static_assert(!kHalves || kBelow - kShift == 34.0f);
            large = true;
            shift = kBelow;
            if (at.far) {  // sums go with the shift
#pragma unroll
                for (int t = 0; t < DT; ++t) acc[t] *= kFall;
                l *= kFall;
            }
        }
        if (x <= wave_most) tile(x, AsF16());
        if (x + 64 < x1) {
            find(x + 64);
            load();
            find(x + 128);
            put(buf ^ 1, x + 64, AsF16());
        }
        x += 64;
        buf ^= 1;
    }
    if (pages.bad()) raise_status(a.status, MP_EINVAL);
    store_rows<D>(k, row, chunk, acc, at.m, l, left_of(at, shift), h);
}

// Many bfloat16 rows, heads of 128: two teams of four waves, 32 rows each wave, over one key head and one chunk
// of tokens in tiles of 64.  Of a SIMD's two waves one is of each team, and the teams take turns: while one
// is at its matrix products (the last tile's second one, this tile's first) the other is at its softmax; a
// barrier ends a turn.
//
// A team's half of the conversion and of the loads for the next tiles goes between its matrix
// instructions: in the turn of the first product of tile i the keys of tile i + 1 and the values of tile i are
// put into LDS, loaded in the turn before, and keys i + 2 and values i + 1 are loaded.  With team 0 at tile i in
// turn 2 i and team 1 in turn 2 i + 1, keys i are read in these two turns and values i in the next two: each
// is whole the turn before, and two tiles' room is enough for both.
//
// Measured, prompts of 228-4096 tokens, 32 query heads over 8: 257-268 us, 860-900 TFLOP/s; four of 4096 tokens 567-608 us,
// 900-970 TFLOP/s (tiles, beside 257 and 573: 267 and 603).  Counted, matrix instructions take 45% of a SIMD's time,
// vector ones 59%, the LDS is active for 35%: the turns overlap little of the two.  Without the priority of the products
// 274 us.  Keys left as codes in LDS, read in a quarter of its time and converted by each wave: 285 us, as the
// conversions meet the other team's softmax.
__global__ __launch_bounds__(512, 2) void kv4_pair_kernel(KvAttend k) {
    constexpr int D = 128, KS = D / 16, DT = D / 32, GROUPS = D / 32;
    extern __shared__ __align__(16) char lds_raw[];
    Tile4<D>* const lds = reinterpret_cast<Tile4<D>*>(lds_raw);
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
    const int32_t most = wave_one(row_of(k, rg, head, min((int64_t)rg.n_rows, rg.row0 + 256) - 1).last);
    const int64_t start = chunk * k.shape.chunk;
    if (chunk > 0 && start > most) return;
    const int32_t x0 = (int32_t)start;
    const int32_t x1 = (int32_t)min((int64_t)most + 1, start + k.shape.chunk);
    const int32_t tiles = (x1 - x0 + 63) >> 6;  // 0 where no row sees anything

    // this wave's rows, and the last position that all of them see
    const int64_t wave_row0 = rg.row0 + 32 * wave;
    const bool awake = wave_row0 < rg.n_rows;  // has rows
    const int32_t wave_least = wave_one(row_of(k, rg, head, wave_row0).last);
    const Row row = row_of(k, rg, head, wave_row0 + n);

    // a thread moves 16 dims of a token's keys (r 0) and of its values (r 1); table entries are read a
    // tile ahead of the loads, keys a tile ahead of values
    const int lb = a.log_block, block = 1 << lb;
    const uint32_t page_size = heads * (uint32_t)(D / 2) << lb, exp_size = heads * (uint32_t)GROUPS << lb;
    Pages pages = {a.s.table + rg.q.s * a.s.table_stride, (uint32_t)max(most, 0) >> lb,
                   (uint32_t)a.c.n_blocks, 0};
    const int token = team * 32 + tid / 8, piece = tid % 8 * 2;
    const uint32_t slot = token & (block - 1);
    const uint32_t code_at = (((uint32_t)head << lb) + slot) * (D / 2) + piece * 4;
    const uint32_t exp_at = (((uint32_t)head * GROUPS + piece / 4) << lb) + slot;
    uint2 codes[2] = {};
    uint32_t exps[2] = {}, entry[2] = {};
    auto tile_of = [&](int r, int v_tile) { return v_tile + 1 - r; };
    auto find = [&](int r, int v_tile) {
        entry[r] = pages.entry((uint32_t)(x0 + tile_of(r, v_tile) * 64 + token) >> lb);
    };
    auto load = [&](int r) {
        const uint64_t page = pages.page(entry[r]);
        codes[r] = *reinterpret_cast<const uint2*>((r ? a.c.v_code : a.c.k_code) + page * page_size + code_at);
        exps[r] = (uint8_t)(r ? a.c.v_exp : a.c.k_exp)[page * exp_size + exp_at];
    };
    // places past the end may hold anything: a scale of one makes their values finite
    auto put = [&](int r, int v_tile, int half) {
        const int tile = tile_of(r, v_tile);
        const uint32_t e = x0 + tile * 64 + token > most ? 127u : exps[r];
        uint4* const to = r ? lds[tile & 1].v[token] : lds[tile & 1].k[token];
        to[(piece + half) ^ (r ? v4_key<D>(token) : k4_key<D>(token))] =
            __builtin_bit_cast(uint4, codes_to_bf(half ? codes[r].y : codes[r].x, __uint_as_float(e << 23)));
    };
    if (tiles > 0) {
        find(0, -1);  // keys 0
        load(0);
        find(0, 0), find(1, 0);  // keys 1, values 0
    }
    bf8_t q[1][KS];
    float c;
    {
        uint4 raw[KS];
#pragma unroll
        for (int i = 0; i < KS; ++i) raw[i] = load8_16bit(k.q, row.token, row.head, i * 16 + h * 8);
        float y[KS][8], top = 0.0f;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            to_float8(k.q, raw[i], y[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(y[i][j]));
        }
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        query_pieces<1>(k, y, top, q, &c);
    }
    float16_t acc[DT], s[2];
#pragma unroll
    for (int t = 0; t < DT; ++t) acc[t] = float16_t{};
    s[0] = s[1] = float16_t{};
    bf8_t w[4] = {};
    Maximum at;
    float l = 0.0f;

    auto turn = [&]() {
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
        __builtin_amdgcn_sched_barrier(0);
    };
    // Piece `p` of a team's moving of data in the turn of tile i's first product: four pieces put keys
    // i + 1 and values i, the others load the ones after.
    constexpr int kPieces = 8;
    auto move = [&](int p, int i) {
        if (p < 4)
            put(p / 2, i, p % 2);
        else if (p < 6)
            load(p - 4);
        else
            find(p - 6, i + 2);
    };
    // Factors from LDS: keys of instruction step i, product t; values of step i, dims t.
    const int k_token = (n & 0x13) | (n & 4) << 1 | (n & 8) >> 1, k_mine = h ^ k4_key<D>(k_token);
    const int v_token = 8 * h + (lane >> 2 & 3), v_dim = (n & 16) + (lane & 3) * 4;
    auto k_factor = [&](int tile, int i, int t) {
        return __builtin_bit_cast(bf8_t, lds[tile & 1].k[t * 32 + k_token][k_mine ^ (i * 2)]);
    };
    auto v_factor = [&](int tile, int i, int t) {
        union {
            short4_t s[2];
            bf8_t v;
        } f;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
            // the low bits of the token that exchange the pieces are a lane's own
            const uint4* const at = &lds[tile & 1].v[i * 16 + 4 * z + v_token][((t * 32 + v_dim) >> 3) ^ v4_key<D>(v_token)];
            f.s[z] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) short4_t*)(reinterpret_cast<const short4_t*>(at) + (v_dim >> 2 & 1)));
        }
        return f.v;
    };
    // The second product of tile i - 1 (SECOND) and the first of tile i (FIRST), factors read kAhead
    // instructions ahead of their use: left to itself the compiler reads each just before.
    auto products = [&](auto second, auto first_too, int i) {
        constexpr int kSecond = second() ? 4 * DT : 0, kAll = kSecond + (first_too() ? 2 * KS : 0);
        constexpr int kAhead = 6;
        __builtin_amdgcn_s_setprio(1);  // the other wave's vector instructions fill what these leave
        bf8_t f[kAhead];
        auto factor = [&](int j) {
            return j < kSecond ? v_factor(i - 1, j / DT, j % DT) : k_factor(i, (j - kSecond) / 2, (j - kSecond) % 2);
        };
#pragma unroll
        for (int j = 0; j < kAhead; ++j) f[j] = factor(j);
        __builtin_amdgcn_sched_barrier(0);
        if (first_too()) s[0] = s[1] = float16_t{};
#pragma unroll
        for (int j = 0; j < kAll; ++j) {
            const bf8_t use = f[j % kAhead];
            if (j < kSecond) {
                acc[j % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(use, w[j / DT], acc[j % DT], 0, 0, 0);
            } else {
                const int z = j - kSecond;
                s[z % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(use, q[0][z / 2], s[z % 2], 0, 0, 0);
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
        put(0, -1, 0), put(0, -1, 1);
        load(0), load(1);
        find(0, 1), find(1, 1);
    }
    turn();
    if (team) turn();
    if (!awake) {  // only moves data
        for (int tile = 0; tile < tiles; ++tile) {
            for (int p = 0; p < kPieces; ++p) move(p, tile);
            turn();
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
        // register r of product t is token 32 t + 16 (r / 8) + 8 h + r % 8
        if (x + 63 > wave_least) {
            const int seen = row.last - x - h * 8;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[t][r] = t * 32 + (r >> 3) * 16 + (r & 7) > seen ? -INFINITY : s[t][r];
        }
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 32; ++r) top = fmaxf(top, s[r / 16][r % 16]);
        {
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
            top = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
        }
        float by = c, from;
        follow(top, kBelow, kSlack, &at, &by, &from,
               [&](float fall) {
#pragma unroll
                   for (int t = 0; t < DT; ++t) acc[t] *= fall;
                   l *= fall;
               },
               [&](float scale, float base) {
#pragma unroll
                   for (int r = 0; r < 32; ++r) s[r / 16][r % 16] = below_maximum(s[r / 16][r % 16], scale, base);
               });
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float e[8], sum = 0.0f;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][i % 2 * 8 + r], by, -from));
                sum += e[r];
            }
            l += sum;
            w[i] = round8(e);
        }
        turn();
        products(Yes{}, Yes{}, tile + 1);  // the last one's scores are of no tile
    }
    if (!team) turn();
    if (pages.bad()) raise_status(a.status, MP_EINVAL);
    store_rows<D>(k, row, chunk, acc, at.m, l, left_of(at, kBelow), h);
}

template <int D, int PIECES>
hipError_t launch_d(const KvAttend& k, hipStream_t st) {
    const KvAttendShape& sh = k.shape;
    const dim3 grid((uint32_t)(sh.units * k.a.c.heads * sh.n_chunks));
    constexpr int kLds = 2 * sizeof(Tile4<D>);
    if (sh.form == KvForm::pair) {  // bfloat16 rows, heads of 128
        kv4_pair_kernel<<<grid, 512, 2 * sizeof(Tile4<128>), st>>>(k);
    } else if (sh.form == KvForm::tiles) {
        if (kLds > 65536)
            if (hipError_t e = hipFuncSetAttribute((const void*)kv4_tiles_kernel<D, PIECES == 2>,
                                                   hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
                e != hipSuccess)
                return e;
        kv4_tiles_kernel<D, PIECES == 2><<<grid, 256, kLds, st>>>(k);
    } else if (D < 256 && grid.x <= 256) {  // a compute unit for every workgroup
        if constexpr (D < 256) kv4_rows_kernel<D, PIECES, 8><<<grid, 512, 0, st>>>(k);
    } else {
        kv4_rows_kernel<D, PIECES, 4><<<grid, 256, 0, st>>>(k);
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_attend(const KvAttend& k, hipStream_t st) {
    const bool two = k.q.dtype == MP_F16;
    switch (k.a.c.dim) {
        case 64: return two ? launch_d<64, 2>(k, st) : launch_d<64, 1>(k, st);
        case 128: return two ? launch_d<128, 2>(k, st) : launch_d<128, 1>(k, st);
        default: return two ? launch_d<256, 2>(k, st) : launch_d<256, 1>(k, st);
    }
}

}  // namespace mp
