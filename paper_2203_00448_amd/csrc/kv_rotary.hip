// Rotary positions: pairs of elements of queries and keys turned by angles that grow with the
// token's position.
//
// A copy with a few operations an element, bound by memory where there are many tokens and by the launch where
// there are few.  The angle is a product in 64 bits, brought below an eighth of a turn in 64 bits, whose sine and
// cosine are then sums of a few terms in 32: one a token and pair, made by the workgroup in LDS for all its
// heads.
#include "kv.hpp"

namespace mp {

namespace {

constexpr int kMaxDim = 4096;

struct Rotary {
    const int32_t* position;
    const double* freq;
    KvRows q, k, q_out, k_out;
    int64_t n_tokens;
    int32_t q_heads, heads;  // of queries; of both
    int32_t dim, turned, tokens;  // tokens of a workgroup
    int32_t q_copy, k_copy;  // whether the elements that are not turned have to be copied
    int32_t log_lanes;       // threads of a head
    float magnitude, sign;
    float by_heads;          // 1 / heads
};

// sin and cos of x in [-pi/4, pi/4] from their series: what is left out is below 2^-29 of one.
__device__ __forceinline__ void small_sin_cos(float x, float* s, float* c) {
    const float z = x * x;
    float p = 1.0f / 362880;
    p = __builtin_fmaf(p, z, -1.0f / 5040);
    p = __builtin_fmaf(p, z, 1.0f / 120);
    p = __builtin_fmaf(p, z, -1.0f / 6);
    *s = __builtin_fmaf(p * z, x, x);
    float r = -1.0f / 3628800;
    r = __builtin_fmaf(r, z, 1.0f / 40320);
    r = __builtin_fmaf(r, z, -1.0f / 720);
    r = __builtin_fmaf(r, z, 1.0f / 24);
    r = __builtin_fmaf(r, z, -0.5f);
    *c = __builtin_fmaf(r, z, 1.0f);
}

__device__ __forceinline__ float2_t sin_cos(int32_t position, double freq) {
    constexpr double kHi = 1.5707963267948966, kLo = 6.123233995736766e-17;  // pi / 2
    const double angle = (double)position * freq;
    const double turns = __builtin_rint(angle * 0.6366197723675814);
    const float x = (float)__builtin_fma(-turns, kLo, __builtin_fma(-turns, kHi, angle));
    const int quarter = (int)(turns - 4.0 * __builtin_floor(turns * 0.25)) & 3;
    float s, c;
    small_sin_cos(x, &s, &c);
    const float a = quarter & 1 ? c : s, b = quarter & 1 ? s : c;
    return float2_t{quarter & 2 ? -a : a, quarter == 1 || quarter == 2 ? -b : b};
}

__device__ __forceinline__ float load_one(const KvRows& r, int64_t at) {
    if (r.dtype == MP_F32) return reinterpret_cast<const float*>(r.data)[at];
    const uint16_t x = reinterpret_cast<const uint16_t*>(r.data)[at];
    return r.dtype == MP_BF16 ? __uint_as_float((uint32_t)x << 16) : half_to_float(x);
}
__device__ __forceinline__ void store_one(const KvRows& r, int64_t at, float x) {
    if (r.dtype == MP_F32)
        reinterpret_cast<float*>(r.data)[at] = x;
    else
        reinterpret_cast<uint16_t*>(r.data)[at] =
            (uint16_t)(r.dtype == MP_BF16 ? float_to_bf16(x) : float_to_half(x));
}

template <int BYTES, int N>
__device__ __forceinline__ void load_vec(const KvRows& r, int64_t at, float (&x)[N]) {
    if constexpr (BYTES == 4) {
        const float4_t w = *reinterpret_cast<const float4_t*>(r.data + at * 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = w[i];
    } else {
        const uint4_t w = *reinterpret_cast<const uint4_t*>(r.data + at * 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) pair_to_float(r.dtype == MP_BF16, w[i], x + 2 * i);
    }
}
template <int BYTES, int N>
__device__ __forceinline__ void store_vec(const KvRows& r, int64_t at, const float (&x)[N]) {
    if constexpr (BYTES == 4) {
        *reinterpret_cast<float4_t*>(r.data + at * 4) = float4_t{x[0], x[1], x[2], x[3]};
    } else {
        uint4_t w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = r.dtype == MP_BF16 ? float_to_bf16(x[2 * i]) | float_to_bf16(x[2 * i + 1]) << 16
                                      : float_to_half(x[2 * i]) | float_to_half(x[2 * i + 1]) << 16;
        *reinterpret_cast<uint4_t*>(r.data + at * 2) = w;
    }
}

// BYTES of an element; WIDE: 16 bytes at a time, with `turned` and `dim` in whole pieces of them (of
// `turned / 2` where PAIRS is not set).  A thread keeps its place in a head and goes through the (token, head)
// pairs of the workgroup.
//
// 16384 tokens of 40 heads of 128, 16-bit: 69 us, 4.9 TB/s (a large copy: 4.9).  8191 of 27 heads of 96 in 32 bits
// 32 us, 5.3 TB/s on inputs that the caches hold, 46 us cold; 64 tokens of 40 heads 4.6 us traced.
template <int BYTES, bool PAIRS, bool WIDE>
__global__ __launch_bounds__(256) void kv_rotary_kernel(Rotary a) {
    constexpr int V = WIDE ? 16 / BYTES : 1;
    extern __shared__ __align__(16) float lds[];
    const int pairs = a.turned / 2, tid = threadIdx.x;
    const int64_t token0 = (int64_t)blockIdx.x * a.tokens;
    const int tokens = (int)min((int64_t)a.tokens, a.n_tokens - token0);
    float* const cosines = lds;
    float* const sines = lds + a.tokens * pairs;
    for (int i = tid; i < tokens * pairs; i += 256) {
        const int t = i / pairs, pair = i - t * pairs;
        const float2_t sc = sin_cos(a.position[token0 + t], a.freq[pair]);
        cosines[i] = sc[1] * a.magnitude;
        sines[i] = sc[0] * a.magnitude * a.sign;
    }
    __syncthreads();
    // pieces of a head: turned ones, then the others
    const int turned_pieces = PAIRS ? (WIDE ? a.turned / V : pairs) : pairs / V;
    const int pieces = turned_pieces + (a.dim - a.turned) / V;
    const int lanes = 1 << a.log_lanes, side = 256 >> a.log_lanes;
    const int all = tokens * a.heads;
    for (int u = tid >> a.log_lanes; u < all; u += side) {
        const int t = (int)(((float)u + 0.5f) * a.by_heads), head = u - t * a.heads;
        const bool is_k = head >= a.q_heads;
        const KvRows& in = is_k ? a.k : a.q;
        const KvRows& out = is_k ? a.k_out : a.q_out;
        const int own = is_k ? head - a.q_heads : head;
        const int64_t from = (token0 + t) * in.token_stride + own * in.head_stride;
        const int64_t to = (token0 + t) * out.token_stride + own * out.head_stride;
        const float* const cs = cosines + t * pairs;
        const float* const sn = sines + t * pairs;
        for (int piece = tid & (lanes - 1); piece < pieces; piece += lanes) {
            if (piece >= turned_pieces) {
                if (!(is_k ? a.k_copy : a.q_copy)) continue;
                const int d = a.turned + (piece - turned_pieces) * V;
                if constexpr (WIDE)
                    *reinterpret_cast<uint4_t*>(out.data + (to + d) * BYTES) =
                        *reinterpret_cast<const uint4_t*>(in.data + (from + d) * BYTES);
                else if constexpr (BYTES == 4)
                    reinterpret_cast<uint32_t*>(out.data)[to + d] = reinterpret_cast<const uint32_t*>(in.data)[from + d];
                else
                    reinterpret_cast<uint16_t*>(out.data)[to + d] = reinterpret_cast<const uint16_t*>(in.data)[from + d];
                continue;
            }
            if constexpr (!WIDE) {
                const int d = PAIRS ? 2 * piece : piece, e = PAIRS ? d + 1 : d + pairs;
                const float x = load_one(in, from + d), y = load_one(in, from + e);
                const float c = cs[piece], s = sn[piece];
                store_one(out, to + d, x * c - y * s);
                store_one(out, to + e, x * s + y * c);
            } else if constexpr (PAIRS) {
                float x[V];
                load_vec<BYTES>(in, from + piece * V, x);
#pragma unroll
                for (int i = 0; i < V; i += 2) {
                    const float c = cs[piece * (V / 2) + i / 2], s = sn[piece * (V / 2) + i / 2];
                    const float p = x[i], q = x[i + 1];
                    x[i] = p * c - q * s;
                    x[i + 1] = p * s + q * c;
                }
                store_vec<BYTES>(out, to + piece * V, x);
            } else {
                float x[V], y[V];
                load_vec<BYTES>(in, from + piece * V, x);
                load_vec<BYTES>(in, from + pairs + piece * V, y);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float c = cs[piece * V + i], s = sn[piece * V + i];
                    const float p = x[i], q = y[i];
                    x[i] = p * c - q * s;
                    y[i] = p * s + q * c;
                }
                store_vec<BYTES>(out, to + piece * V, x);
                store_vec<BYTES>(out, to + pairs + piece * V, y);
            }
        }
    }
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Rows of `tokens` x `heads`; strides that keep every element's offset within 64 bits.
bool rows_ok(const mp_kv_rows* r, int64_t tokens, int64_t heads, KvRows* out) {
    if (!r || (!r->data && tokens > 0)) return false;
    if (r->dtype != MP_BF16 && r->dtype != MP_F16 && r->dtype != MP_F32) return false;
    const int64_t most = (int64_t)1 << 58;
    if (r->token_stride < 0 || r->head_stride < 0 || r->head_stride > most / heads) return false;
    if (tokens > 0 && r->token_stride > most / tokens) return false;
    const size_t size = r->dtype == MP_F32 ? 4 : 2;
    if (!aligned(r->data, size)) return false;
    *out = {static_cast<char*>(r->data), r->token_stride, r->head_stride, r->dtype,
            aligned(r->data, 16) && r->token_stride * size % 16 == 0 && r->head_stride * size % 16 == 0};
    return true;
}

// Whether no two elements of rows that a call writes share a place: one axis lies within a step
// of the other.
bool rows_apart(const KvRows& r, int64_t tokens, int64_t heads, int64_t dim) {
    const bool tokens_outside = r.token_stride >= r.head_stride;
    const int64_t inner = tokens_outside ? r.head_stride : r.token_stride;
    const int64_t outer = tokens_outside ? r.token_stride : r.head_stride;
    const int64_t n_inner = tokens_outside ? heads : tokens, n_outer = tokens_outside ? tokens : heads;
    if (n_inner > 1 && inner < dim) return false;
    const int64_t extent = n_inner > 1 ? (n_inner - 1) * inner + dim : dim;
    return n_outer <= 1 || outer >= extent;
}

bool same_rows(const KvRows& a, const KvRows& b) {
    return a.data == b.data && a.token_stride == b.token_stride && a.head_stride == b.head_stride;
}

template <int BYTES, bool PAIRS>
void launch(const Rotary& a, bool wide, dim3 grid, size_t room, hipStream_t st) {
    if (wide)
        kv_rotary_kernel<BYTES, PAIRS, true><<<grid, 256, room, st>>>(a);
    else
        kv_rotary_kernel<BYTES, PAIRS, false><<<grid, 256, room, st>>>(a);
}

}  // namespace

}  // namespace mp

using namespace mp;

extern "C" int32_t mp_rotate(const int32_t* position, int64_t n_tokens, const double* freq, int32_t turned,
                             int32_t layout, float magnitude, int32_t inverse, int32_t dim,
                             const mp_kv_rows* q, int32_t q_heads, const mp_kv_rows* q_out,
                             const mp_kv_rows* k, int32_t k_heads, const mp_kv_rows* k_out, void* stream) {
    Rotary a = {};
    if (n_tokens < 0 || n_tokens > ((int64_t)1 << 30) || dim < 2 || dim > kMaxDim || turned < 2 ||
        turned > dim || turned % 2 != 0 || (layout != MP_ROTARY_HALVES && layout != MP_ROTARY_PAIRS) ||
        q_heads < 1 || q_heads > (1 << 16) || k_heads < 0 || k_heads > (1 << 16))
        return MP_EINVAL;
    if ((!position && n_tokens > 0) || !aligned(position, 4) || !freq || !aligned(freq, 8)) return MP_EINVAL;
    if (!rows_ok(q, n_tokens, q_heads, &a.q) || !rows_ok(q_out, n_tokens, q_heads, &a.q_out) ||
        a.q.dtype != a.q_out.dtype || !rows_apart(a.q_out, n_tokens, q_heads, dim))
        return MP_EINVAL;
    if (k_heads > 0) {
        if (!rows_ok(k, n_tokens, k_heads, &a.k) || !rows_ok(k_out, n_tokens, k_heads, &a.k_out) ||
            a.k.dtype != a.q.dtype || a.k_out.dtype != a.q.dtype || !rows_apart(a.k_out, n_tokens, k_heads, dim))
            return MP_EINVAL;
    } else {
        a.k = a.q, a.k_out = a.q_out;
    }
    if (n_tokens == 0) return MP_OK;
    a.position = position, a.freq = freq, a.n_tokens = n_tokens;
    a.q_heads = q_heads, a.heads = q_heads + k_heads, a.dim = dim, a.turned = turned;
    a.q_copy = !same_rows(a.q, a.q_out), a.k_copy = !same_rows(a.k, a.k_out);
    a.magnitude = magnitude, a.sign = inverse ? -1.0f : 1.0f, a.by_heads = 1.0f / a.heads;
    const bool pairs = layout == MP_ROTARY_PAIRS, f32 = a.q.dtype == MP_F32;
    const int v = f32 ? 4 : 8;
    const bool wide = a.q.wide && a.q_out.wide && a.k.wide && a.k_out.wide && dim % v == 0 &&
                      (pairs ? turned : turned / 2) % v == 0;
    const int per = wide ? v : 1;
    const int pieces = (pairs ? (wide ? turned / v : turned / 2) : turned / 2 / per) + (dim - turned) / per;
    while ((1 << a.log_lanes) < pieces && a.log_lanes < 8) ++a.log_lanes;
    // tokens of a workgroup: a few thousand pieces, but a workgroup for every place of the device first;
    // their angles fit 32 KiB
    int64_t tokens = 4096 / ((int64_t)a.heads << a.log_lanes);
    if (tokens > n_tokens / 2048) tokens = n_tokens / 2048;
    if (tokens > 4096 / (turned / 2)) tokens = 4096 / (turned / 2);
    a.tokens = tokens < 1 ? 1 : (int32_t)tokens;
    const int64_t groups = (n_tokens + a.tokens - 1) / a.tokens;
    if (!grid_ok(groups, 256)) return MP_EINVAL;
    const dim3 grid((uint32_t)groups);
    const size_t room = (size_t)a.tokens * turned * 4;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (f32)
        pairs ? launch<4, true>(a, wide, grid, room, st) : launch<4, false>(a, wide, grid, room, st);
    else
        pairs ? launch<2, true>(a, wide, grid, room, st) : launch<2, false>(a, wide, grid, room, st);
    return hipGetLastError() == hipSuccess ? MP_OK : MP_EDEVICE;
}
