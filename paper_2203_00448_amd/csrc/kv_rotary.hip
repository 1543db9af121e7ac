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
    // Pieces of a head: those that are turned, all of 16 bytes, with the single pairs, with the single others.
    int32_t turned_pieces, wide, pairs_to, pieces;
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

// VB bytes of elements, 16 or one element's, as words; a piece of 16 bytes lies anywhere where WHOLE is not set (its
// elements are aligned, the load and the store need no more).
template <int VB>
struct Piece {
    uint32_t w[(VB + 3) / 4];
};
typedef uint32_t any4_t __attribute__((ext_vector_type(4), aligned(2)));
template <int VB, bool WHOLE>
__device__ __forceinline__ Piece<VB> load_piece(const char* p) {
    Piece<VB> x;
    if constexpr (VB == 16) {
        const uint4_t w = WHOLE ? *reinterpret_cast<const uint4_t*>(p) : (uint4_t)*reinterpret_cast<const any4_t*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) x.w[i] = w[i];
    } else if constexpr (VB == 4) {
        x.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        x.w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
    return x;
}
template <int VB, bool WHOLE>
__device__ __forceinline__ void store_piece(char* p, const Piece<VB>& x) {
    if constexpr (VB == 16) {
        const uint4_t w = {x.w[0], x.w[1], x.w[2], x.w[3]};
        if constexpr (WHOLE)
            *reinterpret_cast<uint4_t*>(p) = w;
        else
            *reinterpret_cast<any4_t*>(p) = w;
    } else if constexpr (VB == 4) {
        *reinterpret_cast<uint32_t*>(p) = x.w[0];
    } else {
        *reinterpret_cast<uint16_t*>(p) = (uint16_t)x.w[0];
    }
}
// As the type DTYPE is known to the compiler: conversions take a third of the instructions otherwise.
template <int DTYPE, int VB>
__device__ __forceinline__ void to_floats(const Piece<VB>& p, float* x) {
#pragma unroll
    for (int i = 0; i < (VB + 3) / 4; ++i) {
        if constexpr (DTYPE == MP_F32)
            x[i] = __uint_as_float(p.w[i]);
        else if constexpr (VB >= 4)
            pair_to_float(DTYPE == MP_BF16, p.w[i], x + 2 * i);
        else
            x[0] = DTYPE == MP_BF16 ? __uint_as_float(p.w[0] << 16) : half_to_float(p.w[0]);
    }
}
template <int DTYPE, int VB>
__device__ __forceinline__ Piece<VB> from_floats(const float* x) {
    typedef __bf16 bf2_t __attribute__((ext_vector_type(2)));
    Piece<VB> p;
#pragma unroll
    for (int i = 0; i < (VB + 3) / 4; ++i) {
        if constexpr (DTYPE == MP_F32)
            p.w[i] = __float_as_uint(x[i]);
        else if constexpr (VB < 4)
            p.w[0] = DTYPE == MP_BF16 ? float_to_bf16(x[0]) : float_to_half(x[0]);
        else if constexpr (DTYPE == MP_BF16)
            p.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((float2_t{x[2 * i], x[2 * i + 1]}), bf2_t));
        else
            p.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((float2_t{x[2 * i], x[2 * i + 1]}), half2_t));
    }
    return p;
}

// With roundings that do not depend on the place in a piece: to 32 bits, and from there.  (The empty statements keep the
// compiler from one instruction for a sum and its rounding to 16 bits, which it takes here and not there.)
__device__ __forceinline__ void turned_pair(float p, float q, float c, float s, float* x, float* y) {
    float a = __builtin_fmaf(p, c, -(q * s)), b = __builtin_fmaf(p, s, q * c);
    asm("" : "+v"(a));
    asm("" : "+v"(b));
    *x = a, *y = b;
}

// 16 bytes at a time, V elements.  WHOLE: rows lie at multiples of 16 bytes, `dim` and `turned` are whole pieces of them
// (`turned / 2` where PAIRS is not set).  Otherwise pieces lie anywhere, and the last one of the turned elements and of
// the others begins earlier, in the one before, where outputs are not their inputs: both write the same.  Of rows turned
// in place, whose elements may be written before the other piece reads them, and of fewer than V elements, what is left
// goes one by one.  A thread keeps its place in a head and goes through the (token, head) pairs of the workgroup.
//
// 16384 tokens of 40 heads of 128, 16-bit: 69 us, 4.9 TB/s (a large copy: 4.9).  8191 of 27 heads of 96, 64
// turned, in 32 bits 29 us, 5.9 TB/s on inputs that the caches hold, 39 us cold (32 and 46 with loads of their own for
// the lanes that turn nothing); 64 tokens of 40 heads 4 us traced.  Not whole, 16-bit, 16384 tokens of 40 heads, halves:
// of 66 31 us (100 by single elements, 35 with what is left of a head by them), 50 turned of 128 88 (228, 144).
template <int DTYPE, bool PAIRS, bool WHOLE>
__global__ __launch_bounds__(256) void kv_rotary_kernel(Rotary a) {
    constexpr int BYTES = DTYPE == MP_F32 ? 4 : 2, V = 16 / BYTES;
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
    const int turned_pieces = a.turned_pieces, wide = a.wide, pieces = WHOLE ? wide : a.pieces;
    const int each = PAIRS ? a.turned : pairs, rest = a.dim - a.turned;
    const int lanes = 1 << a.log_lanes, side = 256 >> a.log_lanes;
    const int all = tokens * a.heads;
    for (int u = tid >> a.log_lanes; u < all; u += side) {
        const int t = (int)(((float)u + 0.5f) * a.by_heads), head = u - t * a.heads;
        const bool is_k = head >= a.q_heads;
        // field by field: of a struct that a lane chooses the fields are loaded again for every head (46 us cold became 59)
        const int64_t index = is_k ? head - a.q_heads : head, token = token0 + t;
        const char* const from = (is_k ? a.k.data : a.q.data) + (token * (is_k ? a.k.token_stride : a.q.token_stride) +
                                                                 index * (is_k ? a.k.head_stride : a.q.head_stride)) * BYTES;
        char* const to = (is_k ? a.k_out.data : a.q_out.data) +
                         (token * (is_k ? a.k_out.token_stride : a.q_out.token_stride) +
                          index * (is_k ? a.k_out.head_stride : a.q_out.head_stride)) * BYTES;
        const float* const cs = cosines + t * pairs;
        const float* const sn = sines + t * pairs;
        for (int piece = tid & (lanes - 1); piece < pieces; piece += lanes) {
            if (!WHOLE && piece >= wide) {
                const bool turn = piece < a.pairs_to;
                if (!turn && !(is_k ? a.k_copy : a.q_copy)) continue;
                const int pair = turned_pieces * (PAIRS ? V / 2 : V) + piece - wide;
                const int d = !turn ? a.dim - (pieces - piece) : PAIRS ? 2 * pair : pair;
                Piece<BYTES> first = load_piece<BYTES, true>(from + d * BYTES);
                if (turn) {
                    const int e = PAIRS ? d + 1 : d + pairs;
                    const float c = cs[pair], s = sn[pair];
                    float p, q;
                    to_floats<DTYPE, BYTES>(load_piece<BYTES, true>(from + e * BYTES), &q);
                    to_floats<DTYPE, BYTES>(first, &p);
                    float x, y;
                    turned_pair(p, q, c, s, &x, &y);
                    store_piece<BYTES, true>(to + e * BYTES, from_floats<DTYPE, BYTES>(&y));
                    first = from_floats<DTYPE, BYTES>(&x);
                }
                store_piece<BYTES, true>(to + d * BYTES, first);
                continue;
            }
            const bool turn = piece < turned_pieces;
            if (!turn && !(is_k ? a.k_copy : a.q_copy)) continue;
            if constexpr (PAIRS) {  // one load of all lanes, whether they turn it or not
                const int at = (turn ? piece : piece - turned_pieces) * V, end = (turn ? each : rest) - V;
                const int d = (turn ? 0 : a.turned) + (WHOLE ? at : min(at, end));
                Piece<16> own = load_piece<16, WHOLE>(from + d * BYTES);
                if (turn) {
                    float x[V];
                    to_floats<DTYPE, 16>(own, x);
#pragma unroll
                    for (int i = 0; i < V; i += 2) {
                        const float c = cs[(d + i) / 2], s = sn[(d + i) / 2];
                        turned_pair(x[i], x[i + 1], c, s, &x[i], &x[i + 1]);
                    }
                    own = from_floats<DTYPE, 16>(x);
                }
                store_piece<16, WHOLE>(to + d * BYTES, own);
            } else if (!turn) {
                const int at = (piece - turned_pieces) * V, d = a.turned + (WHOLE ? at : min(at, rest - V));
                store_piece<16, WHOLE>(to + d * BYTES, load_piece<16, WHOLE>(from + d * BYTES));
            } else {
                const int d = WHOLE ? piece * V : min(piece * V, each - V), e = d + pairs;
                float x[V], y[V];
                to_floats<DTYPE, 16>(load_piece<16, WHOLE>(from + d * BYTES), x);
                to_floats<DTYPE, 16>(load_piece<16, WHOLE>(from + e * BYTES), y);
#pragma unroll
                for (int i = 0; i < V; ++i) turned_pair(x[i], y[i], cs[d + i], sn[d + i], &x[i], &y[i]);
                store_piece<16, WHOLE>(to + d * BYTES, from_floats<DTYPE, 16>(x));
                store_piece<16, WHOLE>(to + e * BYTES, from_floats<DTYPE, 16>(y));
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

// Whether rows are the same places.  An axis of one has no stride.
bool same_rows(const KvRows& a, const KvRows& b, int64_t tokens, int64_t heads) {
    return a.data == b.data && (tokens <= 1 || a.token_stride == b.token_stride) &&
           (heads <= 1 || a.head_stride == b.head_stride);
}

template <int DTYPE>
void launch(const Rotary& a, bool pairs, bool whole, dim3 grid, size_t room, hipStream_t st) {
    if (pairs)
        whole ? kv_rotary_kernel<DTYPE, true, true><<<grid, 256, room, st>>>(a)
              : kv_rotary_kernel<DTYPE, true, false><<<grid, 256, room, st>>>(a);
    else
        whole ? kv_rotary_kernel<DTYPE, false, true><<<grid, 256, room, st>>>(a)
              : kv_rotary_kernel<DTYPE, false, false><<<grid, 256, room, st>>>(a);
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
    a.q_copy = !same_rows(a.q, a.q_out, n_tokens, q_heads);
    a.k_copy = k_heads > 0 ? !same_rows(a.k, a.k_out, n_tokens, k_heads) : a.q_copy;
    a.magnitude = magnitude, a.sign = inverse ? -1.0f : 1.0f, a.by_heads = 1.0f / a.heads;
    const bool pairs = layout == MP_ROTARY_PAIRS, f32 = a.q.dtype == MP_F32;
    const int v = f32 ? 4 : 8, each = pairs ? turned : turned / 2;
    const int rest = a.q_copy || a.k_copy ? dim - turned : 0;
    const bool whole = a.q.wide && a.q_out.wide && a.k.wide && a.k_out.wide && dim % v == 0 && each % v == 0;
    const bool twice = a.q_copy && a.k_copy;  // a last piece may begin in the one before
    a.turned_pieces = twice && each >= v ? (each + v - 1) / v : each / v;
    a.wide = a.turned_pieces + (twice && rest >= v ? (rest + v - 1) / v : rest / v);
    a.pairs_to = a.wide + (twice && each >= v ? 0 : each % v / (pairs ? 2 : 1));
    a.pieces = a.pairs_to + (twice && rest >= v ? 0 : rest % v);
    while ((1 << a.log_lanes) < a.pieces && a.log_lanes < 8) ++a.log_lanes;
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
    switch (a.q.dtype) {
        case MP_BF16: launch<MP_BF16>(a, pairs, whole, grid, room, st); break;
        case MP_F16: launch<MP_F16>(a, pairs, whole, grid, room, st); break;
        default: launch<MP_F32>(a, pairs, whole, grid, room, st);
    }
    return hipGetLastError() == hipSuccess ? MP_OK : MP_EDEVICE;
}
