// The 4-bit key/value cache written and read back.
//
// A token's codes depend on nothing but its own values: each 32 dims of a head have their
// scale.  So both operators are copies with a conversion, bound by memory where there are
// many tokens and by a chain of loads (bounds, length, table, values) where there are few.
// A wave takes a token: a lane has eight dims of keys and of values, four lanes a scale, and the
// heads of a token go over the lanes in turn.
#include "kv.hpp"

namespace mp {

namespace {

constexpr int kOnce = 2;  // pieces of a lane whose loads are on their way together

// A token of a call: its place in its block, and the block.
struct KvPlace {
    int64_t page;
    int32_t slot;
};

// The place of row `token`; false (and a data error) where there is none.
__device__ __forceinline__ bool kv_place(const KvArgs& a, int64_t token, KvPlace* p) {
    int64_t i;
    const KvSeq q = kv_find(a, token, [&](int64_t b, int64_t) { return b; }, &i);
    if (!q.ok || i < 0 || i >= q.n) return false;
    const int32_t pos = q.length - q.n + (int32_t)i;
    if (q.length < q.n) {  // more rows than tokens
        raise_status(a.status, MP_EINVAL);
        return false;
    }
    const int32_t page = a.s.table[q.s * a.s.table_stride + (pos >> a.log_block)];
    if (page < 0 || page >= a.c.n_blocks) {
        raise_status(a.status, MP_EINVAL);
        return false;
    }
    p->page = page;
    p->slot = pos & ((1 << a.log_block) - 1);
    return true;
}

// The least e in [kLeastExp, kMostExp] with top <= 7 * 2^e (7 = 7/8 * 2^3).
__device__ __forceinline__ int scale_exponent4(float top) {
    uint32_t frac;
    const int x = exponent_of(top, &frac);
    return min(kMostExp, max(kLeastExp, x - 3 + (frac > 0x600000u)));
}

// Eight values of a lane, four lanes a scale, to codes; *exp as it is held.  Values that are not
// finite: infinities as the largest value, NaN as zero; neither counts for the scale.
__device__ __forceinline__ uint32_t encode8(float* x, int* exp, bool* finite) {
    float top = 0.0f;
    bool all = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float y = fabsf(x[j]);
        all = all && y < INFINITY;
        top = fmaxf(top, y);
    }
    if (!all) {
        top = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (fabsf(x[j]) < INFINITY) top = fmaxf(top, fabsf(x[j]));
            if (x[j] != x[j]) x[j] = 0.0f;
        }
    }
    *finite = all;
    top = fmaxf(top, __shfl_xor(top, 1, kWave));
    top = fmaxf(top, __shfl_xor(top, 2, kWave));
    const int e = scale_exponent4(top);
    *exp = e + 127;
    // the instruction divides by the scale, rounds to nearest even and holds what is beyond 6 to it
    const float scale = pow2f(e);
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    return w;
}

__device__ __forceinline__ void decode8(uint32_t w, int exp, float* x) {
    const float scale = __uint_as_float((uint32_t)exp << 23);
    const float2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
    const float2_t b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const float2_t c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
    const float2_t d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = c[0], x[5] = c[1], x[6] = d[0], x[7] = d[1];
}

// Where eight dims of (page, head, slot) lie: their codes' word, their scale's byte.
struct Places {
    int64_t word, exp;
};
__device__ __forceinline__ Places places(const KvArgs& a, const KvPlace& p, int head, int d) {
    const int64_t row = p.page * a.c.heads + head;
    Places at;
    at.word = ((row << a.log_block) + p.slot) * (a.c.dim / 8) + d / 8;
    at.exp = ((row * (a.c.dim / 32) + d / 32) << a.log_block) + p.slot;
    return at;
}

// 16 prompts of 1-4096 tokens, 8 heads of 128, 16-bit rows: 27 us, 4.2 TB/s; a token each of 256 sequences 5 us.
__global__ __launch_bounds__(256) void kv4_write_kernel(KvArgs a, KvRows k, KvRows v) {
    if (blockIdx.x == 0) kv_check_begin(a);
    const int64_t token = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (token >= a.s.n_tokens) return;
    const int lane = threadIdx.x & 63, vecs = a.c.dim / 8, items = a.c.heads * vecs;
    KvPlace p;
    if (!kv_place(a, token, &p)) return;
    bool finite = true;
    // all lanes of a scale's four are in or out: items is a multiple of 8
    for (int i0 = lane; i0 < items; i0 += kOnce * kWave) {
        Raw8 kr[kOnce], vr[kOnce];
#pragma unroll
        for (int j = 0; j < kOnce; ++j) {
            const int i = i0 + j * kWave, head = i / vecs, d = i % vecs * 8;
            if (i < items) kr[j] = load_raw8(k, token, head, d), vr[j] = load_raw8(v, token, head, d);
        }
#pragma unroll
        for (int j = 0; j < kOnce; ++j) {
            const int i = i0 + j * kWave, head = i / vecs, d = i % vecs * 8;
            if (i >= items) break;
            const Places at = places(a, p, head, d);
            float x[8];
            int exp;
            bool fine;
            raw8_to_float(k, kr[j], x);
            reinterpret_cast<uint32_t*>(a.c.k_code)[at.word] = encode8(x, &exp, &fine);
            finite = finite && fine;
            if (d % 32 == 0) a.c.k_exp[at.exp] = (int8_t)exp;
            raw8_to_float(v, vr[j], x);
            reinterpret_cast<uint32_t*>(a.c.v_code)[at.word] = encode8(x, &exp, &fine);
            finite = finite && fine;
            if (d % 32 == 0) a.c.v_exp[at.exp] = (int8_t)exp;
        }
    }
    if (!finite) raise_status(a.status, MP_EINVAL);
}

// The same tokens read back: 21 us, 5.3 TB/s (the codes of the call before are in the caches); 33 tokens each of 256
// sequences 9.3-9.6 us, 4.3 TB/s: 41 MB, nearly all of them results.
__global__ __launch_bounds__(256) void kv4_read_kernel(KvArgs a, KvRows k, KvRows v) {
    if (blockIdx.x == 0) kv_check_begin(a);
    const int64_t token = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (token >= a.s.n_tokens) return;
    const int lane = threadIdx.x & 63, vecs = a.c.dim / 8, items = a.c.heads * vecs;
    KvPlace p;
    if (!kv_place(a, token, &p)) return;
    for (int i0 = lane; i0 < items; i0 += kOnce * kWave) {
        uint32_t kw[kOnce], vw[kOnce];
        int ke[kOnce], ve[kOnce];
#pragma unroll
        for (int j = 0; j < kOnce; ++j) {
            const int i = i0 + j * kWave;
            if (i >= items) break;
            const Places at = places(a, p, i / vecs, i % vecs * 8);
            kw[j] = reinterpret_cast<const uint32_t*>(a.c.k_code)[at.word];
            vw[j] = reinterpret_cast<const uint32_t*>(a.c.v_code)[at.word];
            ke[j] = (uint8_t)a.c.k_exp[at.exp], ve[j] = (uint8_t)a.c.v_exp[at.exp];
        }
#pragma unroll
        for (int j = 0; j < kOnce; ++j) {
            const int i = i0 + j * kWave, head = i / vecs, d = i % vecs * 8;
            if (i >= items) break;
            float x[8];
            decode8(kw[j], ke[j], x);
            store8(k, token, head, d, x);
            decode8(vw[j], ve[j], x);
            store8(v, token, head, d, x);
        }
    }
}

}  // namespace

int64_t kv4_move_groups(const KvArgs& a) { return (a.s.n_tokens + 3) / 4; }

hipError_t launch_kv4_write(const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t st) {
    const dim3 grid((uint32_t)kv4_move_groups(a));
    if (grid.x == 0) return hipSuccess;
    kv4_write_kernel<<<grid, 256, 0, st>>>(a, k, v);
    return hipGetLastError();
}

hipError_t launch_kv4_read(const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t st) {
    const dim3 grid((uint32_t)kv4_move_groups(a));
    if (grid.x == 0) return hipSuccess;
    kv4_read_kernel<<<grid, 256, 0, st>>>(a, k, v);
    return hipGetLastError();
}

}  // namespace mp
