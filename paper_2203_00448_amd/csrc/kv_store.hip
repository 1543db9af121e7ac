// The 8-bit key/value cache written and read back.
//
// Both are copies with a conversion: a value is read once and a byte written, or the
// other way round, so memory bounds them where there are many tokens and the launch
// where there are few.  A workgroup takes one head of one touched block.  The block is
// put together in LDS, keys by token and values by dim as they lie in memory, because
// values change their order on the way (the attention reads them along the tokens).
#include "kv.hpp"
#include "internal.hpp"

namespace mp {

namespace {

constexpr int kMaxDim = 256, kMaxBlock = 64;

// A piece of a sequence within one block: the call's tokens [lo, hi) of block `blk`.
struct KvPiece {
    int32_t page;
    int32_t first;  // place of the first token in the block
    int32_t count;
    int64_t token;  // row of the first token
};

// Piece `u` of the launch.  Sequence s has the pieces from (begin[s] >> log_block) + 2 s on: n
// tokens touch at most (n >> log_block) + 2 blocks, so no two sequences share one.
__device__ __forceinline__ bool kv_piece(const KvArgs& a, int64_t u, KvPiece* p) {
    const int lb = a.log_block;
    int64_t s = u, j = 0;
    if (a.s.begin) {
        s = kv_find(a.s.n_seqs, u, [&](int64_t i) { return (a.s.begin[i] >> lb) + 2 * i; });
        j = u - ((a.s.begin[s] >> lb) + 2 * s);
    }
    const KvSeq q = kv_seq(a, s);
    if (!q.ok || j < 0 || q.n == 0) return false;
    const int32_t start = q.length - q.n;
    if (start < 0) {  // more rows than tokens
        raise_status(a.status, MP_EINVAL);
        return false;
    }
    const int64_t blk = (start >> lb) + j;
    const int64_t lo = max((int64_t)start, blk << lb), hi = min((int64_t)q.length, (blk + 1) << lb);
    if (lo >= hi) return false;
    p->page = a.s.table[s * a.s.table_stride + blk];
    if (p->page < 0 || p->page >= a.c.n_blocks) {
        raise_status(a.status, MP_EINVAL);
        return false;
    }
    p->first = (int32_t)(lo - (blk << lb));
    p->count = (int32_t)(hi - lo);
    p->token = q.begin + lo - start;
    return true;
}

template <int THREADS>
__device__ __forceinline__ float block_max(float x, float* scratch) {
    return THREADS == kWave ? wave_reduce(x, OpMax<float>())
                            : block_reduce<THREADS>(x, OpMax<float>(), scratch);
}

// One head of one block.  THREADS = 64 is the form for one token of each sequence (its 2 dim
// values fit the wave), 256 the form for any number.
//
// The first pass over the values finds the scale, and they stay in registers for the
// second.  Codes that the block holds already are read only where they change (the scale
// grew), where a mean is due (the block became full) or, in the form for many tokens,
// always, so that rows of values are written whole.
template <bool INT8, int THREADS>
__global__ __launch_bounds__(THREADS) void kv_write_kernel(KvArgs a, KvRows k, KvRows v) {
    constexpr int kItems = THREADS == kWave ? 1 : kMaxDim * kMaxBlock / 8 / THREADS;
    __shared__ __align__(16) uint8_t sk[kMaxDim * kMaxBlock];
    __shared__ __align__(16) uint8_t sv[kMaxDim * kMaxBlock];
    __shared__ float scratch[THREADS / kWave];
    const int tid = threadIdx.x, dim = a.c.dim, block = 1 << a.log_block;
    if (blockIdx.x == 0) kv_check_begin(a);
    const int64_t u = blockIdx.x / a.c.heads;
    const int head = blockIdx.x % a.c.heads;
    KvPiece p;
    if (!kv_piece(a, u, &p)) return;
    if (THREADS == kWave && p.count > 1) return;  // no sequence of that form has more
    const int vecs = dim / 8, items = p.count * vecs;
    const int64_t at = (int64_t)p.page * a.c.heads + head;
    uint8_t* const k_code = a.c.k_code + at * block * dim;
    uint8_t* const v_code = a.c.v_code + at * block * dim;

    float kx[kItems][8], vx[kItems][8];
    float k_top = 0.0f, v_top = 0.0f;
    bool finite = true;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = tid + i * THREADS;
        if (item < items) {
            const int row = item / vecs, d = item % vecs * 8;
            load8(k, p.token + row, head, d, kx[i]);
            load8(v, p.token + row, head, d, vx[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float ka = fabsf(kx[i][j]), va = fabsf(vx[i][j]);
                if (ka < INFINITY) k_top = fmaxf(k_top, ka);
                if (va < INFINITY) v_top = fmaxf(v_top, va);
                finite = finite && ka < INFINITY && va < INFINITY;
            }
        }
    }
    if (!finite) raise_status(a.status, MP_EINVAL);
    const bool held = p.first > 0, full = p.first + p.count == block;
    const int k_was = held ? a.c.k_exp[at] : kLeastExp, v_was = held ? a.c.v_exp[at] : kLeastExp;
    k_top = block_max<THREADS>(k_top, scratch);
    v_top = block_max<THREADS>(v_top, scratch);
    const int ke = max(k_was, scale_exponent<INT8>(k_top));
    const int ve = max(v_was, scale_exponent<INT8>(v_top));
    const bool k_grew = held && ke > k_was, v_grew = held && ve > v_was;
    const bool k_held = held && (THREADS > kWave || k_grew || full);
    const bool v_whole = THREADS > kWave || v_grew;  // rows of values are written whole

    // new codes
    const float limit = INT8 ? 127.0f : 448.0f, kf = pow2f(-ke), vf = pow2f(-ve);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = tid + i * THREADS;
        if (item < items) {
            const int row = p.first + item / vecs, d = item % vecs * 8;
            uint32_t w[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // infinities to the largest code, NaN to zero
                const float x = kx[i][j] * kf, y = vx[i][j] * vf;
                const float xc = x != x ? 0.0f : fminf(limit, fmaxf(-limit, x));
                const float yc = y != y ? 0.0f : fminf(limit, fmaxf(-limit, y));
                w[j / 4] |= encode<INT8>(xc) << (8 * (j % 4));
                sv[(d + j) * block + row] = (uint8_t)encode<INT8>(yc);
            }
            *reinterpret_cast<uint2*>(sk + row * dim + d) = make_uint2(w[0], w[1]);
        }
    }
    // held codes, at the new scale; places past the sequence get zeros
    if (k_held) {
        const float f = pow2f(max(-126, k_was - ke));
        for (int i = tid; i < p.first * dim / 4; i += THREADS) {
            uint32_t w = reinterpret_cast<const uint32_t*>(k_code)[i];
            if (k_grew) {
                uint32_t o = 0;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    o |= encode<INT8>(decode<INT8>(w >> (8 * j) & 0xffu) * f) << (8 * j);
                w = o;
            }
            reinterpret_cast<uint32_t*>(sk)[i] = w;
        }
    }
    if (v_whole) {
        const float f = pow2f(max(-126, v_was - ve));
        for (int i = tid; i < dim * block / 4; i += THREADS) {
            const int t = i * 4 & (block - 1);
            uint32_t w = 0;
            if (t < p.first) w = reinterpret_cast<const uint32_t*>(v_code)[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = t + j;
                if (row >= p.first && row < p.first + p.count) continue;
                uint32_t code = row < p.first ? w >> (8 * j) & 0xffu : 0;
                if (v_grew) code = encode<INT8>(decode<INT8>(code) * f);
                sv[i * 4 + j] = (uint8_t)code;
            }
        }
    }
    __syncthreads();

    const int from = k_grew ? 0 : p.first;
    for (int i = from * dim / 8 + tid; i < (p.first + p.count) * dim / 8; i += THREADS)
        reinterpret_cast<uint2*>(k_code)[i] = reinterpret_cast<const uint2*>(sk)[i];
    if (v_whole) {
        for (int i = tid; i < dim * block / 16; i += THREADS)
            reinterpret_cast<uint4*>(v_code)[i] = reinterpret_cast<const uint4*>(sv)[i];
    } else {
        for (int i = tid; i < dim * p.count; i += THREADS) {
            const int d = i / p.count, row = p.first + i % p.count;
            v_code[d * block + row] = sv[d * block + row];
        }
    }
    if (tid == 0) {
        a.c.k_exp[at] = (int8_t)ke;
        a.c.v_exp[at] = (int8_t)ve;
    }
    if (!full) return;
    // the mean of the keys: at most 64 codes, whole multiples of 2^-9 below 2^15: exact in any order
    constexpr int kDims = (kMaxDim + THREADS - 1) / THREADS;
    float sum[kDims], top = 0.0f;
#pragma unroll
    for (int i = 0; i < kDims; ++i) {
        const int d = tid + i * THREADS;
        sum[i] = 0.0f;
        if (d < dim)
            for (int t = 0; t < block; ++t) sum[i] += decode<INT8>(sk[t * dim + d]);
        top = fmaxf(top, fabsf(sum[i]));
    }
    top = block_max<THREADS>(top, scratch);
    const int e = top > 0.0f ? scale_exponent<true>(top) : -15;
#pragma unroll
    for (int i = 0; i < kDims; ++i) {
        const int d = tid + i * THREADS;
        if (d < dim) a.c.mean_code[at * dim + d] = (int8_t)encode<true>(sum[i] * pow2f(-e));
    }
    if (tid == 0) a.c.mean_exp[at] = (int8_t)(ke + e - a.log_block);
}

// One head of one block's tokens back to rows.  The values' bytes turn in LDS; a row of it
// is four bytes longer than a block's so that the threads that read along the dims meet
// different banks.
template <bool INT8>
__global__ __launch_bounds__(256) void kv_read_kernel(KvArgs a, KvRows k, KvRows v) {
    __shared__ __align__(16) uint8_t sv[kMaxDim * (kMaxBlock + 4)];
    const int tid = threadIdx.x, dim = a.c.dim, block = 1 << a.log_block;
    if (blockIdx.x == 0) kv_check_begin(a);
    const int64_t u = blockIdx.x / a.c.heads;
    const int head = blockIdx.x % a.c.heads;
    KvPiece p;
    if (!kv_piece(a, u, &p)) return;
    const int vecs = dim / 8, items = p.count * vecs;
    const int64_t at = (int64_t)p.page * a.c.heads + head;
    const uint8_t* const k_code = a.c.k_code + at * block * dim;
    const uint8_t* const v_code = a.c.v_code + at * block * dim;
    const float kf = pow2f(a.c.k_exp[at]), vf = pow2f(a.c.v_exp[at]);
    for (int i = tid; i < dim * block / 16; i += 256) {
        const uint4 w = reinterpret_cast<const uint4*>(v_code)[i];
        const int d = i * 16 >> a.log_block, t = i * 16 & (block - 1);
        uint32_t* o = reinterpret_cast<uint32_t*>(sv + d * (block + 4) + t);
        o[0] = w.x, o[1] = w.y, o[2] = w.z, o[3] = w.w;
    }
    __syncthreads();
    for (int item = tid; item < items; item += 256) {
        const int row = item / vecs, d = item % vecs * 8, t = p.first + row;
        const uint2 w = *reinterpret_cast<const uint2*>(k_code + t * dim + d);
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            x[j] = decode<INT8>((j < 4 ? w.x : w.y) >> (8 * (j % 4)) & 0xffu) * kf;
        store8(k, p.token + row, head, d, x);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = decode<INT8>(sv[(d + j) * (block + 4) + t]) * vf;
        store8(v, p.token + row, head, d, x);
    }
}

int64_t pieces(const KvArgs& a) {
    return a.s.begin ? (a.s.n_tokens >> a.log_block) + 2 * a.s.n_seqs : a.s.n_seqs;
}

}  // namespace

hipError_t launch_kv_write(const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t st) {
    const dim3 grid((uint32_t)(pieces(a) * a.c.heads));
    if (grid.x == 0) return hipSuccess;
    if (a.s.begin) {
        if (a.c.kind == MP_KV_INT8)
            kv_write_kernel<true, 256><<<grid, 256, 0, st>>>(a, k, v);
        else
            kv_write_kernel<false, 256><<<grid, 256, 0, st>>>(a, k, v);
    } else {
        if (a.c.kind == MP_KV_INT8)
            kv_write_kernel<true, 64><<<grid, 64, 0, st>>>(a, k, v);
        else
            kv_write_kernel<false, 64><<<grid, 64, 0, st>>>(a, k, v);
    }
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t st) {
    const dim3 grid((uint32_t)(pieces(a) * a.c.heads));
    if (grid.x == 0) return hipSuccess;
    if (a.c.kind == MP_KV_INT8)
        kv_read_kernel<true><<<grid, 256, 0, st>>>(a, k, v);
    else
        kv_read_kernel<false><<<grid, 256, 0, st>>>(a, k, v);
    return hipGetLastError();
}

}  // namespace mp
