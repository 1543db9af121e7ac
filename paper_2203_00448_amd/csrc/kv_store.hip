// The 8-bit key/value cache written and read back.
//
// Both are copies with a conversion: a value is read once and a byte written, or the
// other way round, so memory bounds them where there are many tokens and the launch
// where there are few.  A workgroup takes one head of one touched block.  The block is
// put together in LDS, keys by token and values by dim as they lie in memory, because
// values change their order on the way (the attention reads them along the tokens).
#include "kv.hpp"

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
    int64_t j;
    const KvSeq q = kv_find(a, u, [&](int64_t b, int64_t i) { return (b >> lb) + 2 * i; }, &j);
    if (!q.ok || j < 0 || q.n == 0) return false;
    const int32_t start = q.length - q.n;
    if (start < 0) {  // more rows than tokens
        raise_status(a.status, MP_EINVAL);
        return false;
    }
    const int64_t blk = (start >> lb) + j;
    const int64_t lo = max((int64_t)start, blk << lb), hi = min((int64_t)q.length, (blk + 1) << lb);
    if (lo >= hi) return false;
    p->page = a.s.table[q.s * a.s.table_stride + blk];
    if (p->page < 0 || p->page >= a.c.n_blocks) {
        raise_status(a.status, MP_EINVAL);
        return false;
    }
    p->first = (int32_t)(lo - (blk << lb));
    p->count = (int32_t)(hi - lo);
    p->token = q.begin + lo - start;
    return true;
}

// Four scaled values as four codes, the first lowest.
template <bool INT8>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    if (INT8) {
        const uint32_t x = (uint32_t)(int)__builtin_rintf(a), y = (uint32_t)(int)__builtin_rintf(b);
        const uint32_t z = (uint32_t)(int)__builtin_rintf(c), w = (uint32_t)(int)__builtin_rintf(d);
        // the low bytes of two words each
        const uint32_t lo = __builtin_amdgcn_perm(y, x, 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(w, z, 0x0c0c0400u);
        return lo | hi << 16;
    }
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// Four held codes at a scale 1 / f times as large.
template <bool INT8>
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float f) {
    return encode4<INT8>(decode<INT8>(w & 0xffu) * f, decode<INT8>(w >> 8 & 0xffu) * f,
                         decode<INT8>(w >> 16 & 0xffu) * f, decode<INT8>(w >> 24) * f);
}

// The largest of a and of b over the workgroup.
__device__ __forceinline__ void block_max2(float* a, float* b, float (*scratch)[2]) {
    *a = wave_reduce(*a, OpMax<float>());
    *b = wave_reduce(*b, OpMax<float>());
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (lane == 0) scratch[wave][0] = *a, scratch[wave][1] = *b;
    __syncthreads();
    *a = fmaxf(fmaxf(scratch[0][0], scratch[1][0]), fmaxf(scratch[2][0], scratch[3][0]));
    *b = fmaxf(fmaxf(scratch[0][1], scratch[1][1]), fmaxf(scratch[2][1], scratch[3][1]));
}

// One head of one block.  ITEMS of a thread's places are 0 in the form for one token of each
// sequence (ONE), else what four places and eight dims a thread leave.
//
// The first pass over the values finds the scale, and they stay in registers for the
// second: a thread has eight dims of four consecutive places of the block (ONE: of one), so
// that it has whole words of both arrays, whose bytes go by dim and by token.  Codes that the
// block holds already are read only where they change (the scale grew), where a mean is due
// (the block became full) or, in the form for many tokens, always, so that rows of values
// are written whole.  All of a thread's loads are on their way before the first is converted: 16
// prompts of 1-4096 tokens, 8 heads of 128, 37 us (3.7 TB/s), 43 with a wait for each.
template <bool INT8, int ITEMS>
__global__ __launch_bounds__(256) void kv_write_kernel(KvArgs a, KvRows k, KvRows v) {
    constexpr bool ONE = ITEMS == 0;
    constexpr int kItems = ONE ? 1 : ITEMS, kRows = ONE ? 1 : 4;
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ float scratch[4][2];
    __shared__ float4_t sums[256];
    const int tid = threadIdx.x, dim = a.c.dim, block = 1 << a.log_block;
    uint8_t* const sk = lds;                // [token][dim]
    uint8_t* const sv = lds + dim * block;  // [dim][token], rows four bytes longer: other banks
    const int v_row = block + 4;
    if (blockIdx.x == 0) kv_check_begin(a);
    const uint32_t heads = a.c.heads;
    const int64_t u = blockIdx.x / heads;
    const int head = blockIdx.x % heads;
    KvPiece p;
    if (!kv_piece(a, u, &p)) return;
    const int vecs = dim / 8;
    const int64_t at = (int64_t)p.page * heads + head;
    uint8_t* const k_code = a.c.k_code + at * block * dim;
    uint8_t* const v_code = a.c.v_code + at * block * dim;
    const bool held = p.first > 0, full = p.first + p.count == block;
    const int k_was = held ? a.c.k_exp[at] : kLeastExp, v_was = held ? a.c.v_exp[at] : kLeastExp;

    // places of item i: four from 4 * (item / vecs) on (ONE: the token's), those that are the call's
    const int items = ONE ? vecs : block / 4 * vecs;
    auto place = [&](int item, int r) { return ONE ? p.first : item / vecs * 4 + r; };
    auto is_new = [&](int item, int r) {
        const int t = place(item, r) - p.first;
        return item < items && t >= 0 && t < p.count;
    };
    float kx[kItems][kRows][8], vx[kItems][kRows][8];
    float k_top = 0.0f, v_top = 0.0f;
    // all loads before the first conversion; places that are not the call's as zeros
    Raw8 k_raw[kItems][kRows], v_raw[kItems][kRows];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = tid + i * 256, d = item % vecs * 8;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            k_raw[i][r] = v_raw[i][r] = Raw8{};
            if (is_new(item, r)) {
                k_raw[i][r] = load_raw8(k, p.token + place(item, r) - p.first, head, d);
                v_raw[i][r] = load_raw8(v, p.token + place(item, r) - p.first, head, d);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i)
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            raw8_to_float(k, k_raw[i][r], kx[i][r]);
            raw8_to_float(v, v_raw[i][r], vx[i][r]);
        }
    bool finite = true;
#pragma unroll
    for (int i = 0; i < kItems; ++i)
#pragma unroll
        for (int r = 0; r < kRows; ++r)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float ka = fabsf(kx[i][r][j]), va = fabsf(vx[i][r][j]);
                finite = finite && ka < INFINITY && va < INFINITY;
                k_top = fmaxf(k_top, ka);
                v_top = fmaxf(v_top, va);
            }
    if (!finite) {
        // infinities as the largest value, NaN as zero; neither counts for the scale
        raise_status(a.status, MP_EINVAL);
        k_top = v_top = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
            for (int r = 0; r < kRows; ++r)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float ka = kx[i][r][j], va = vx[i][r][j];
                    if (fabsf(ka) < INFINITY) k_top = fmaxf(k_top, fabsf(ka));
                    if (fabsf(va) < INFINITY) v_top = fmaxf(v_top, fabsf(va));
                    if (ka != ka) kx[i][r][j] = 0.0f;
                    if (va != va) vx[i][r][j] = 0.0f;
                }
    }
    block_max2(&k_top, &v_top, scratch);
    const int ke = max(k_was, scale_exponent<INT8>(k_top));
    const int ve = max(v_was, scale_exponent<INT8>(v_top));
    const bool k_grew = held && ke > k_was, v_grew = held && ve > v_was;
    const bool k_held = held && (!ONE || k_grew || full);
    const bool v_whole = !ONE || v_grew;  // rows of values are written whole

    // new codes; a value past the largest one (not finite, or beyond the largest scale) is held to it
    const float limit = INT8 ? 127.0f : 448.0f, kf = pow2f(-ke), vf = pow2f(-ve);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = tid + i * 256, d = item % vecs * 8;
        if (item >= items) continue;
        bool all = !ONE;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            all = all && is_new(item, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                kx[i][r][j] = __builtin_amdgcn_fmed3f(kx[i][r][j] * kf, -limit, limit);
                vx[i][r][j] = __builtin_amdgcn_fmed3f(vx[i][r][j] * vf, -limit, limit);
            }
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (!is_new(item, r)) continue;
            const float* x = kx[i][r];
            *reinterpret_cast<uint2*>(sk + place(item, r) * dim + d) = make_uint2(
                encode4<INT8>(x[0], x[1], x[2], x[3]), encode4<INT8>(x[4], x[5], x[6], x[7]));
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint8_t* const to = sv + (d + j) * v_row + place(item, 0);
            if (kRows == 4) {
                const uint32_t w = encode4<INT8>(vx[i][0][j], vx[i][1 % kRows][j], vx[i][2 % kRows][j],
                                                 vx[i][3 % kRows][j]);
                if (all) {
                    *reinterpret_cast<uint32_t*>(to) = w;
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (is_new(item, r)) to[r] = (uint8_t)(w >> (8 * r));
                }
            } else {
                to[0] = (uint8_t)encode<INT8>(vx[i][0][j]);
            }
        }
    }
    // held codes, at the new scale; places past the sequence get zeros
    if (k_held) {
        const float f = pow2f(max(-126, k_was - ke));
        for (int i = tid; i < p.first * dim / 4; i += 256) {
            uint32_t w = reinterpret_cast<const uint32_t*>(k_code)[i];
            if (k_grew) w = rescale4<INT8>(w, f);
            reinterpret_cast<uint32_t*>(sk)[i] = w;
        }
    }
    if (v_whole && (held || !full)) {
        const float f = pow2f(max(-126, v_was - ve));
        for (int i = tid; i < dim * block / 4; i += 256) {
            const int t = i * 4 & (block - 1);
            if (t >= p.first && t + 4 <= p.first + p.count) continue;
            uint32_t w = 0;
            if (t < p.first) {
                w = reinterpret_cast<const uint32_t*>(v_code)[i];
                if (v_grew) w = rescale4<INT8>(w, f);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = t + j;
                uint8_t* const to = sv + (i * 4 >> a.log_block) * v_row + row;
                if (row < p.first) *to = (uint8_t)(w >> (8 * j));
                if (row >= p.first + p.count) *to = 0;
            }
        }
    }
    __syncthreads();

    const int from = k_grew ? 0 : p.first;
    for (int i = from * dim / 16 + tid; i < (p.first + p.count) * dim / 16; i += 256)
        reinterpret_cast<uint4*>(k_code)[i] = reinterpret_cast<const uint4*>(sk)[i];
    if (v_whole) {
        for (int i = tid; i < dim * block / 16; i += 256) {
            const uint32_t* const w = reinterpret_cast<const uint32_t*>(
                sv + (i * 16 >> a.log_block) * v_row + (i * 16 & (block - 1)));
            reinterpret_cast<uint4*>(v_code)[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    } else {
        for (int d = tid; d < dim; d += 256) v_code[d * block + p.first] = sv[d * v_row + p.first];
    }
    if (tid == 0) {
        a.c.k_exp[at] = (int8_t)ke;
        a.c.v_exp[at] = (int8_t)ve;
    }
    if (!full) return;
    // the mean of the keys: at most 64 codes, whole multiples of 2^-9 below 2^15: exact in any order
    // four dims a thread, of some of the tokens
    const int fours = dim / 4, slices = 256 / fours, four = tid % fours, slice = tid / fours;
    float4_t part = {0, 0, 0, 0};
    for (int r = slice; r < block; r += slices) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(sk + r * dim + four * 4);
#pragma unroll
        for (int j = 0; j < 4; ++j) part[j] += decode<INT8>(w >> (8 * j) & 0xffu);
    }
    sums[tid] = part;
    __syncthreads();
    float sum = 0.0f, unused = 0.0f;
    if (tid < dim)
        for (int r = 0; r < slices; ++r) sum += reinterpret_cast<const float*>(sums + r * fours)[tid];
    float top = fabsf(sum);
    block_max2(&top, &unused, scratch);
    const int e = top > 0.0f ? scale_exponent<true>(top) : -15;
    if (tid < dim) a.c.mean_code[at * dim + tid] = (int8_t)encode<true>(sum * pow2f(-e));
    if (tid == 0) a.c.mean_exp[at] = (int8_t)(ke + e - a.log_block);
}

// A block's tokens back to rows, `per` key heads one after the other.  The values' bytes turn
// in LDS; a row of it is four bytes longer than a block's so that the threads that read
// along the dims meet different banks.  8 sequences of 1-16384 tokens, 8 heads of 128: 69 us, 4.4 TB/s.
template <bool INT8>
__global__ __launch_bounds__(256) void kv_read_kernel(KvArgs a, KvRows k, KvRows v, int32_t per) {
    extern __shared__ __align__(16) uint8_t sv[];
    const int tid = threadIdx.x, dim = a.c.dim, lb = a.log_block, block = 1 << lb;
    if (blockIdx.x == 0) kv_check_begin(a);
    const uint32_t heads = a.c.heads, parts = (heads + per - 1) / per;
    const int64_t u = blockIdx.x / parts;
    const int head0 = blockIdx.x % parts * per, head1 = min((int)heads, head0 + per);
    KvPiece p;
    if (!kv_piece(a, u, &p)) return;
    const int vecs = dim / 8, items = p.count * vecs, size = dim << lb;
    const int64_t at = (int64_t)p.page * heads;
    constexpr int kLoads = kMaxDim * kMaxBlock / 16 / 256;
    uint4 w[kLoads];
    auto load = [&](int head) {
        const uint4* const from = reinterpret_cast<const uint4*>(a.c.v_code + (at + head) * size);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            if (tid + i * 256 < size / 16) w[i] = from[tid + i * 256];
    };
    load(head0);
    for (int head = head0; head < head1; ++head) {
        const uint8_t* const k_code = a.c.k_code + (at + head) * size;
        const float kf = pow2f(a.c.k_exp[at + head]), vf = pow2f(a.c.v_exp[at + head]);
        if (head > head0) __syncthreads();
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int b = (tid + i * 256) * 16;
            if (b < size) {
                uint32_t* o = reinterpret_cast<uint32_t*>(sv + (b >> lb) * (block + 4) + (b & (block - 1)));
                o[0] = w[i].x, o[1] = w[i].y, o[2] = w[i].z, o[3] = w[i].w;
            }
        }
        if (head + 1 < head1) load(head + 1);
        __syncthreads();
        for (int item = tid; item < items; item += 256) {
            const int row = item / vecs, d = item % vecs * 8, t = p.first + row;
            const uint2 c = *reinterpret_cast<const uint2*>(k_code + t * dim + d);
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                x[j] = decode<INT8>((j < 4 ? c.x : c.y) >> (8 * (j % 4)) & 0xffu) * kf;
            store8(k, p.token + row, head, d, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = decode<INT8>(sv[(d + j) * (block + 4) + t]) * vf;
            store8(v, p.token + row, head, d, x);
        }
    }
}

int64_t pieces(const KvArgs& a) {
    return a.s.begin ? (a.s.n_tokens >> a.log_block) + 2 * a.s.n_seqs : a.s.n_seqs;
}

// Heads that a workgroup reads: as many as leave 2048 workgroups, which the device holds at once.
int64_t heads_of(const KvArgs& a) {
    const int64_t per = pieces(a) * a.c.heads / 2048;
    return per < 1 ? 1 : per > a.c.heads ? a.c.heads : per > 8 ? 8 : per;
}

}  // namespace

int64_t kv_write_groups(const KvArgs& a) { return pieces(a) * a.c.heads; }

int64_t kv_read_groups(const KvArgs& a) {
    const int64_t per = heads_of(a);
    return pieces(a) * ((a.c.heads + per - 1) / per);
}

hipError_t launch_kv_write(const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t st) {
    const dim3 grid((uint32_t)kv_write_groups(a));
    if (grid.x == 0) return hipSuccess;
    const size_t room = (size_t)a.c.dim * ((2 << a.log_block) + 4);
    const bool i8 = a.c.kind == MP_KV_INT8;
    const int items = !a.s.begin ? 0 : (a.c.dim << a.log_block) / 32 <= 256 ? 1 : 2;
    if (items == 0)
        (i8 ? kv_write_kernel<true, 0> : kv_write_kernel<false, 0>)<<<grid, 256, room, st>>>(a, k, v);
    else if (items == 1)
        (i8 ? kv_write_kernel<true, 1> : kv_write_kernel<false, 1>)<<<grid, 256, room, st>>>(a, k, v);
    else
        (i8 ? kv_write_kernel<true, 2> : kv_write_kernel<false, 2>)<<<grid, 256, room, st>>>(a, k, v);
    return hipGetLastError();
}

hipError_t launch_kv_read(const KvArgs& a, const KvRows& k, const KvRows& v, hipStream_t st) {
    const dim3 grid((uint32_t)kv_read_groups(a));
    if (grid.x == 0) return hipSuccess;
    const int64_t per = heads_of(a);
    const size_t room = (size_t)a.c.dim * ((1 << a.log_block) + 4);
    if (a.c.kind == MP_KV_INT8)
        kv_read_kernel<true><<<grid, 256, room, st>>>(a, k, v, (int32_t)per);
    else
        kv_read_kernel<false><<<grid, 256, room, st>>>(a, k, v, (int32_t)per);
    return hipGetLastError();
}

}  // namespace mp
