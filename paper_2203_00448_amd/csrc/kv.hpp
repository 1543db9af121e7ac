// The 8-bit key/value cache: arguments of its kernels and their common device code.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <type_traits>

#include "memoplan.h"
#include "mp_device.hpp"

namespace mp {

// Rows of a call, with what the host found out about their alignment.
struct KvRows {
    char* data;
    int64_t token_stride, head_stride;  // elements
    int32_t dtype;
    int32_t wide;  // data and strides are multiples of 16 bytes
};

struct KvArgs {
    mp_kv_cache c;
    mp_kv_seqs s;
    int32_t log_block;
    int32_t* status;
};

// Whether a launch of so many workgroups is possible: fewer than 2^32 threads.
inline bool grid_ok(int64_t workgroups, int threads) { return workgroups <= (((int64_t)1 << 32) - 1) / threads; }

// Workgroups (of 256 threads) of a write or a read.
int64_t kv_write_groups(const KvArgs& a);
int64_t kv_read_groups(const KvArgs& a);
hipError_t launch_kv_write(const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t st);
hipError_t launch_kv_read(const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t st);

// What a call of mp_kv_attend launches (kv_attend.hip).
enum class KvForm { rows, tiles, pair };
struct KvAttendShape {
    bool ok;
    KvForm form;
    int32_t rows;      // rows (query, head) of a workgroup
    int64_t units;     // row groups over all sequences, an upper bound
    int64_t chunk;     // tokens (of the sequence, or of its listed blocks) of a workgroup
    int64_t n_chunks;
    bool ordered;      // row groups of tiles by what they see
    size_t workspace;
};

struct KvAttend {
    KvArgs a;
    KvRows q, out;
    float scale;
    int32_t group;          // query heads of a key head
    const int32_t* blocks;  // or null
    int32_t keep;
    float* lse;
    void* ws;
    KvAttendShape shape;
};

KvAttendShape kv_attend_shape(const mp_kv_cache& c, const mp_kv_seqs& s, int32_t q_heads,
                              int64_t keep);
hipError_t launch_kv_attend(const KvAttend& a, hipStream_t st);

struct KvSelect {
    KvArgs a;
    KvRows q;
    int32_t group;
    int32_t keep, first, recent;
    int32_t* out;
    float* scores;  // [token][head][score_stride], or in LDS
    int64_t score_stride;
    int32_t tokens;  // of a workgroup
    int64_t units;   // groups of so many tokens over all sequences, an upper bound
};

// What a call of mp_kv_select launches (kv_select.hip).
struct KvSelectShape {
    bool ok;
    bool global;  // scores in the workspace
    int32_t tokens;
    int64_t units, score_stride;
    size_t workspace;
};

KvSelectShape kv_select_shape(const mp_kv_cache& c, const mp_kv_seqs& s, int32_t q_heads);
hipError_t launch_kv_select(const KvSelect& a, hipStream_t st);

// ---- device code

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef uint32_t uint4_t __attribute__((ext_vector_type(4)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef float float4_t __attribute__((ext_vector_type(4)));
typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int kLeastExp = -100, kMostExp = 120;  // of a block's scale

// 2^e for e in [-126, 127].
__device__ __forceinline__ float pow2f(int e) { return __int_as_float((e + 127) << 23); }

// x with top = m * 2^x, 1/2 <= m < 1, for a normal top; the fraction bits of m in *frac.
__device__ __forceinline__ int exponent_of(float top, uint32_t* frac) {
    const uint32_t b = __float_as_uint(top);
    *frac = b & 0x7fffffu;
    return (int)(b >> 23) - 126;
}

// The least e in [kLeastExp, kMostExp] with top <= 448 * 2^e (448 = 7/8 * 2^9) or, int8,
// top <= 127 * 2^e (127 = 127/128 * 2^7); top finite, not negative.  A top below the normal
// range falls to kLeastExp like zero.
template <bool INT8>
__device__ __forceinline__ int scale_exponent(float top) {
    uint32_t frac;
    const int x = exponent_of(top, &frac);
    const int e = INT8 ? x - 7 + (frac > 0x7e0000u) : x - 9 + (frac > 0x600000u);
    return min(kMostExp, max(kLeastExp, e));
}

// x (already scaled) to its code, nearest even.  |x| is at most the largest code.
template <bool INT8>
__device__ __forceinline__ uint32_t encode(float x) {
    if (INT8) return (uint32_t)(int)__builtin_rintf(x) & 0xffu;
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, x, 0, false) & 0xffu;
}
template <bool INT8>
__device__ __forceinline__ float decode(uint32_t code) {
    if (INT8) return (float)(int)(int8_t)code;
    return __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
}

// Eight codes (two words) as eight 16-bit floats, exactly.
template <bool INT8>
__device__ __forceinline__ half8_t codes_to_half(uint32_t a, uint32_t b) {
    union {
        half2_t h[4];
        half8_t v;
    } o;
    if (INT8) {
        // byte + 128 put below the exponent of 1024, whose steps are 1: 1152 + code
        const half2_t bias = {(_Float16)1152.0f, (_Float16)1152.0f};
        const uint32_t x = a ^ 0x80808080u, y = b ^ 0x80808080u;
        const uint32_t w[4] = {__builtin_amdgcn_perm(0x64646464u, x, 0x04010400u),
                               __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u),
                               __builtin_amdgcn_perm(0x64646464u, y, 0x04010400u),
                               __builtin_amdgcn_perm(0x64646464u, y, 0x04030402u)};
#pragma unroll
        for (int i = 0; i < 4; ++i) o.h[i] = __builtin_bit_cast(half2_t, w[i]) - bias;
    } else {
        o.h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false);
        o.h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
        o.h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false);
        o.h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
    }
    return o.v;
}

__device__ __forceinline__ float half_to_float(uint32_t bits) {
    return (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}
__device__ __forceinline__ uint32_t float_to_half(float x) {
    return __builtin_bit_cast(uint16_t, (_Float16)x);
}
__device__ __forceinline__ uint32_t float_to_bf16(float x) {
    return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// Eight consecutive elements of a row, at a multiple of eight, as they lie in memory: loads only,
// so that a caller has several on their way before the first is converted.
struct Raw8 {
    uint32_t w[8];  // 32-bit elements; wide 16-bit ones in pairs in the first four; narrow ones each
};
__device__ __forceinline__ Raw8 load_raw8(const KvRows& r, int64_t token, int64_t head, int d) {
    const int64_t at = token * r.token_stride + head * r.head_stride + d;
    Raw8 x = {};
    if (r.dtype == MP_F32) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(r.data) + at;
        if (r.wide) {
            *reinterpret_cast<uint4_t*>(x.w) = *reinterpret_cast<const uint4_t*>(p);
            *reinterpret_cast<uint4_t*>(x.w + 4) = *reinterpret_cast<const uint4_t*>(p + 4);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) x.w[i] = p[i];
        }
        return x;
    }
    const uint16_t* p = reinterpret_cast<const uint16_t*>(r.data) + at;
    if (r.wide) {
        *reinterpret_cast<uint4_t*>(x.w) = *reinterpret_cast<const uint4_t*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x.w[i] = p[i];
    }
    return x;
}

// Two 16-bit elements as floats.
__device__ __forceinline__ void pair_to_float(bool bf16, uint32_t w, float* x) {
    x[0] = bf16 ? __uint_as_float(w << 16) : half_to_float(w & 0xffffu);
    x[1] = bf16 ? __uint_as_float(w & 0xffff0000u) : half_to_float(w >> 16);
}
__device__ __forceinline__ void raw8_to_float(const KvRows& r, const Raw8& raw, float* x) {
    if (r.dtype == MP_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(raw.w[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = r.wide ? raw.w[i] : raw.w[2 * i] | raw.w[2 * i + 1] << 16;
        pair_to_float(r.dtype == MP_BF16, w, x + 2 * i);
    }
}

// The same of rows of a 16-bit type, packed.
__device__ __forceinline__ uint4 load8_16bit(const KvRows& r, int64_t token, int64_t head, int d) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(r.data) + token * r.token_stride + head * r.head_stride + d;
    if (r.wide) return *reinterpret_cast<const uint4*>(p);
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)p[2 * i] | (uint32_t)p[2 * i + 1] << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void to_float8(const KvRows& r, uint4 w, float* x) {
    const bool bf16 = r.dtype == MP_BF16;
    pair_to_float(bf16, w.x, x);
    pair_to_float(bf16, w.y, x + 2);
    pair_to_float(bf16, w.z, x + 4);
    pair_to_float(bf16, w.w, x + 6);
}

// The same place written, each value rounded once; where the stores are wide, past the caches, which
// have the codes to hold: 8 sequences of 1-16384 tokens read back in 69 us, 73 through them; with
// codes that the caches hold from an earlier call 52 us, 74 through them.
__device__ __forceinline__ void store8(const KvRows& r, int64_t token, int64_t head, int d,
                                       const float* x) {
    const int64_t at = token * r.token_stride + head * r.head_stride + d;
    if (r.dtype == MP_F32) {
        float* p = reinterpret_cast<float*>(r.data) + at;
        if (r.wide) {
            __builtin_nontemporal_store(*reinterpret_cast<const float4_t*>(x), reinterpret_cast<float4_t*>(p));
            __builtin_nontemporal_store(*reinterpret_cast<const float4_t*>(x + 4), reinterpret_cast<float4_t*>(p) + 1);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = x[i];
        }
        return;
    }
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        w[i] = r.dtype == MP_BF16
                   ? float_to_bf16(x[2 * i]) | float_to_bf16(x[2 * i + 1]) << 16
                   : float_to_half(x[2 * i]) | float_to_half(x[2 * i + 1]) << 16;
    uint16_t* p = reinterpret_cast<uint16_t*>(r.data) + at;
    if (r.wide) {
        __builtin_nontemporal_store(uint4_t{w[0], w[1], w[2], w[3]}, reinterpret_cast<uint4_t*>(p));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[2 * i] = (uint16_t)w[i];
            p[2 * i + 1] = (uint16_t)(w[i] >> 16);
        }
    }
}

// N (four or eight, at a multiple of it) elements of rows of a 16-bit type written the same way.
template <int N>
__device__ __forceinline__ void store_16bit(const KvRows& r, int64_t token, int64_t head, int d, const float* x) {
    const bool bf16 = r.dtype == MP_BF16;
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const uint32_t b = float_to_bf16(x[2 * i]) | float_to_bf16(x[2 * i + 1]) << 16;
        const uint32_t h = float_to_half(x[2 * i]) | float_to_half(x[2 * i + 1]) << 16;
        w[i] = bf16 ? b : h;
    }
    uint16_t* p = reinterpret_cast<uint16_t*>(r.data) + token * r.token_stride + head * r.head_stride + d;
    if (r.wide) {
        if constexpr (N == 8)
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else
            *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        return;
    }
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        p[2 * i] = (uint16_t)w[i];
        p[2 * i + 1] = (uint16_t)(w[i] >> 16);
    }
}

// A sequence of a call: its rows [begin, begin + n) and its tokens.
struct KvSeq {
    int32_t s, length, n;
    int64_t begin;
    bool ok;
};

// The whole of begin[] checked, by the first workgroup of a launch.
__device__ __forceinline__ void kv_check_begin(const KvArgs& a) {
    if (!a.s.begin) return;
    bool bad = a.s.begin[0] != 0 || a.s.begin[a.s.n_seqs] != a.s.n_tokens;
    for (int64_t i = threadIdx.x; i < a.s.n_seqs; i += blockDim.x)
        bad |= a.s.begin[i + 1] < a.s.begin[i];
    if (bad) raise_status(a.status, MP_EINVAL);
}

// Rows [b, e) of sequence s, as begin[] gave them.
__device__ __forceinline__ KvSeq kv_seq(const KvArgs& a, int64_t s, int64_t b, int64_t e) {
    KvSeq q;
    q.s = (int32_t)s;
    q.length = a.s.length[s];
    q.begin = b;
    q.n = (int32_t)(e - b);
    q.ok = b >= 0 && e >= b && e <= a.s.n_tokens && (!a.s.begin || e - b <= a.s.most_new) &&
           q.length >= 0 && q.length <= a.s.longest;
    if (!q.ok) raise_status(a.status, MP_EINVAL);
    return q;
}

// What all lanes of the wave have alike, said so: scalar registers hold it.
__device__ __forceinline__ int32_t wave_one(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t wave_one(int64_t x) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)x);
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | lo);
}
__device__ __forceinline__ KvSeq wave_one(KvSeq q) {
    q.s = wave_one(q.s);
    q.length = wave_one(q.length);
    q.n = wave_one(q.n);
    q.begin = wave_one(q.begin);
    q.ok = wave_one((int32_t)q.ok) != 0;
    return q;
}

// The last sequence whose key(begin[s], s) is at most u, where keys never fall with s (s itself
// without begin), and u less its key; the whole wave searches, 64 keys a turn, and keeps what
// it read of begin[].  Any values there give a sequence in range.
template <typename Key>
__device__ __forceinline__ KvSeq kv_find(const KvArgs& a, int64_t u, Key key, int64_t* rest) {
    if (!a.s.begin) {
        *rest = 0;
        return wave_one(kv_seq(a, u, u, u + 1));
    }
    const int lane = threadIdx.x & (kWave - 1);
    int64_t lo = 0, hi = a.s.n_seqs, b = 0, e = 0;
    int count = kWave;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
        b = at <= hi ? a.s.begin[at] : 0;
        const uint64_t below = __ballot(at < hi && key(b, at) <= u);
        count = below == ~0ull ? kWave : __ffsll((unsigned long long)~below) - 1;
        if (step == 1 && count < kWave) {  // this turn read the sequence's rows and the next one's
            const int i = max(0, count - 1);
            e = __shfl(b, i + 1, kWave);
            b = __shfl(b, i, kWave);
            *rest = wave_one(u - key(b, lo + i));
            return wave_one(kv_seq(a, lo + i, b, e));
        }
        lo += (int64_t)max(0, count - 1) * step;
        hi = min(hi, lo + step);
    }
    b = a.s.begin[lo];
    *rest = wave_one(u - key(b, lo));
    return wave_one(kv_seq(a, lo, b, a.s.begin[lo + 1]));
}

}  // namespace mp
