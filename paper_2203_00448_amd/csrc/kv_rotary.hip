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

// VB bytes (an element at least) of elements of BYTES each, as words, as floats and back.
template <int VB>
struct Piece {
    uint32_t w[(VB + 3) / 4];
};
template <int VB>
__device__ __forceinline__ Piece<VB> load_piece(const char* p) {
    Piece<VB> x;
    if constexpr (VB == 16)
        *reinterpret_cast<uint4_t*>(x.w) = *reinterpret_cast<const uint4_t*>(p);
    else if constexpr (VB == 8)
        *reinterpret_cast<uint2*>(x.w) = *reinterpret_cast<const uint2*>(p);
    else if constexpr (VB == 4)
        x.w[0] = *reinterpret_cast<const uint32_t*>(p);
    else
        x.w[0] = *reinterpret_cast<const uint16_t*>(p);
    return x;
}
template <int VB>
__device__ __forceinline__ void store_piece(char* p, const Piece<VB>& x) {
    if constexpr (VB == 16)
        *reinterpret_cast<uint4_t*>(p) = *reinterpret_cast<const uint4_t*>(x.w);
    else if constexpr (VB == 8)
        *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(x.w);
    else if constexpr (VB == 4)
        *reinterpret_cast<uint32_t*>(p) = x.w[0];
    else
        *reinterpret_cast<uint16_t*>(p) = (uint16_t)x.w[0];
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

// VB bytes at a time, V elements, with `dim` and `turned` in whole pieces of them (`turned / 2`
// where PAIRS is not set; a single element of a pair has the other one beside it).  A thread keeps its place in a
// head and goes through the (token, head) pairs of the workgroup.
//
// 16384 tokens of 40 heads of 128, 16-bit: 69 us, 4.9 TB/s (a large copy: 4.9).  8191 of 27 heads of 96, 64
// turned, in 32 bits 29 us, 5.9 TB/s on inputs that the caches hold, 39 us cold (32 and 46 with loads of their own for
// the lanes that turn nothing); 64 tokens of 40 heads 4.6 us traced.
template <int DTYPE, bool PAIRS, int VB>
__global__ __launch_bounds__(256) void kv_rotary_kernel(Rotary a) {
    constexpr int BYTES = DTYPE == MP_F32 ? 4 : 2, V = VB / BYTES;
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
    // pieces of a head: turned ones (with PAIRS and single elements, one for two), then the others
    const int turned_pieces = PAIRS && V > 1 ? a.turned / V : pairs / V;
    const int pieces = turned_pieces + (a.dim - a.turned) / V;
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
            const bool turn = piece < turned_pieces;
            if (!turn && !(is_k ? a.k_copy : a.q_copy)) continue;
            if constexpr (PAIRS && V > 1) {  // one load of all lanes, whether they turn it or not
                const int d = piece * V;
                Piece<VB> own = load_piece<VB>(from + d * BYTES);
                if (turn) {
                    float x[V];
                    to_floats<DTYPE, VB>(own, x);
#pragma unroll
                    for (int i = 0; i < V; i += 2) {
                        const float c = cs[(d + i) / 2], s = sn[(d + i) / 2], p = x[i], q = x[i + 1];
                        x[i] = p * c - q * s;
                        x[i + 1] = p * s + q * c;
                    }
                    own = from_floats<DTYPE, VB>(x);
                }
                store_piece<VB>(to + d * BYTES, own);
            } else if (!turn) {
                const int d = a.turned + (piece - turned_pieces) * V;
                store_piece<VB>(to + d * BYTES, load_piece<VB>(from + d * BYTES));
            } else {
                const int d = PAIRS ? 2 * piece : piece * V, e = PAIRS ? d + 1 : d + pairs;
                float x[V], y[V];
                to_floats<DTYPE, VB>(load_piece<VB>(from + d * BYTES), x);
                to_floats<DTYPE, VB>(load_piece<VB>(from + e * BYTES), y);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float c = cs[piece * V + i], s = sn[piece * V + i], p = x[i], q = y[i];
                    x[i] = p * c - q * s;
                    y[i] = p * s + q * c;
                }
                store_piece<VB>(to + d * BYTES, from_floats<DTYPE, VB>(x));
                store_piece<VB>(to + e * BYTES, from_floats<DTYPE, VB>(y));
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

// The most bytes, a power of two up to 16, that divide a row's place and strides.
int alignment(const KvRows& r) {
    const uintptr_t size = r.dtype == MP_F32 ? 4 : 2;
    const uintptr_t all = reinterpret_cast<uintptr_t>(r.data) | r.token_stride * size | r.head_stride * size | 16;
    return (int)(all & -all);
}

template <int DTYPE, bool PAIRS>
void launch(const Rotary& a, int vb, dim3 grid, size_t room, hipStream_t st) {
    if (vb == 16)
        kv_rotary_kernel<DTYPE, PAIRS, 16><<<grid, 256, room, st>>>(a);
    else if (vb == 8)
        kv_rotary_kernel<DTYPE, PAIRS, 8><<<grid, 256, room, st>>>(a);
    else if (vb == 4)
        kv_rotary_kernel<DTYPE, PAIRS, 4><<<grid, 256, room, st>>>(a);
    else
        kv_rotary_kernel<DTYPE, PAIRS, DTYPE == MP_F32 ? 4 : 2><<<grid, 256, room, st>>>(a);
}

template <int DTYPE>
void launch(const Rotary& a, bool pairs, int vb, dim3 grid, size_t room, hipStream_t st) {
    pairs ? launch<DTYPE, true>(a, vb, grid, room, st) : launch<DTYPE, false>(a, vb, grid, room, st);
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
    // the widest pieces that everything is whole ones of.  16-bit, by these and by elements: 32534 tokens of 9 heads
    // of 96, 76 turned in pairs (8 bytes) 34 and 78 us; 16384 of 40 heads of 66 in pairs (4 bytes) 95 and 128.
    const int size = f32 ? 4 : 2, whole = pairs ? turned : turned / 2;
    int vb = alignment(a.q);
    for (const KvRows* r : {&a.q_out, &a.k, &a.k_out}) vb = alignment(*r) < vb ? alignment(*r) : vb;
    while (vb > size && (dim % (vb / size) != 0 || whole % (vb / size) != 0)) vb /= 2;
    const int v = vb / size;
    const int pieces = (pairs && v > 1 ? turned / v : turned / 2 / v) + (dim - turned) / v;
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
    switch (a.q.dtype) {
        case MP_BF16: launch<MP_BF16>(a, pairs, vb, grid, room, st); break;
        case MP_F16: launch<MP_F16>(a, pairs, vb, grid, room, st); break;
        default: launch<MP_F32>(a, pairs, vb, grid, room, st);
    }
    return hipGetLastError() == hipSuccess ? MP_OK : MP_EDEVICE;
}
