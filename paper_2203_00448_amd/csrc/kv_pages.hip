// Blocks given to sequences and taken back: tables, lengths, bounds, positions and slots of a step, on
// the device.
//
// Two sums run over the sequences (tokens, blocks); what hangs on them is one store a token, a
// block, a sequence.  One workgroup has the sums, whose inputs it reads twice, so that nothing is changed where
// an argument is wrong or the pool is short; a second launch has the stores, a thread a token (or, taking
// back, a workgroup a sequence).
#include "kv.hpp"

namespace mp {

namespace {

constexpr int kThreads = 1024, kItems = 8;  // of the workgroup that sums; sequences of a thread at once
constexpr int64_t kMaxCount = (int64_t)1 << 30;

struct Pages {
    const int32_t* ids;
    int32_t* ids_out;  // release
    int64_t n_ids;
    const int64_t* used;
    int32_t* table;
    int64_t table_stride, table_width;
    int32_t log_block;
    const int32_t* length;
    const int32_t* more;   // extend
    const uint8_t* done;   // release
    int64_t n_seqs, n_tokens;
    int32_t* length_out;
    int64_t* used_out;
    int64_t* begin_out;
    int32_t* position_out;
    int64_t* slot_out;
    int64_t* first;  // workspace: of each sequence its first block's place in ids, and the end; then the tokens
    int32_t* status;
};

struct Need {
    int64_t tokens, blocks;
    int32_t length;  // afterwards
    bool ok;
};

template <bool EXTEND>
__device__ __forceinline__ Need need_of(const Pages& p, int64_t s) {
    Need n = {0, 0, 0, true};
    const int64_t t = ((int64_t)1 << p.log_block) - 1, room = p.table_width << p.log_block;
    const int64_t length = p.length[s];
    n.ok = length >= 0 && length <= room;
    n.length = (int32_t)length;
    if (EXTEND) {
        const int64_t more = p.more[s];
        n.ok = n.ok && more >= 0 && length + more <= room && length + more <= INT32_MAX;
        n.tokens = more;
        n.blocks = ((length + more + t) >> p.log_block) - ((length + t) >> p.log_block);
        n.length = (int32_t)(length + more);
    } else if (p.done[s]) {
        n.blocks = (length + t) >> p.log_block;
        n.length = 0;
    }
    if (!n.ok) n.tokens = n.blocks = 0;
    return n;
}

template <bool EXTEND>
__global__ __launch_bounds__(kThreads) void kv_pages_sum_kernel(Pages p) {
    __shared__ int64_t scratch[kThreads / 64];
    __shared__ int32_t bad_scratch[kThreads / 64];
    const int tid = threadIdx.x;
    const int64_t used = *p.used;
    Need mine[kItems];
    int64_t tokens = 0, blocks = 0;
    bool ok = true;
    const int64_t step = kThreads * kItems;
    auto load = [&](int64_t s0) {
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int64_t s = s0 + tid * kItems + i;
            mine[i] = s < p.n_seqs ? need_of<EXTEND>(p, s) : Need{0, 0, 0, true};
        }
    };
    for (int64_t s0 = 0; s0 < p.n_seqs; s0 += step) {
        load(s0);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            tokens += mine[i].tokens;
            blocks += mine[i].blocks;
            ok = ok && mine[i].ok;
        }
    }
    int32_t code = ok && used >= 0 && used <= p.n_ids ? MP_OK : MP_EINVAL;
    code = block_reduce<kThreads>(code, OpMin<int32_t>(), bad_scratch);
    tokens = block_reduce<kThreads>(tokens, OpAdd<int64_t>(), scratch);
    blocks = block_reduce<kThreads>(blocks, OpAdd<int64_t>(), scratch);
    if (code == MP_OK && EXTEND && (tokens > p.n_tokens || blocks > p.n_ids - used)) code = MP_ENOSPC;
    if (code == MP_OK && !EXTEND && blocks > used) code = MP_EINVAL;
    const bool fine = code == MP_OK;
    if (tid == 0) {
        raise_status(p.status, code);
        *p.used_out = fine ? (EXTEND ? used + blocks : used - blocks) : used;
        p.first[p.n_seqs + 1] = fine ? tokens : 0;
    }
    int64_t token_at = 0, block_at = EXTEND ? used : used - blocks;
    for (int64_t s0 = 0; s0 < p.n_seqs; s0 += step) {
        if (p.n_seqs > step) load(s0);
        int64_t my_tokens = 0, my_blocks = 0, all_tokens, all_blocks;
#pragma unroll
        for (int i = 0; i < kItems; ++i) my_tokens += mine[i].tokens, my_blocks += mine[i].blocks;
        int64_t t = token_at + block_exclusive_sum<kThreads>(my_tokens, &all_tokens, scratch);
        int64_t b = block_at + block_exclusive_sum<kThreads>(my_blocks, &all_blocks, scratch);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int64_t s = s0 + tid * kItems + i;
            if (s >= p.n_seqs) continue;
            if (EXTEND) p.begin_out[s] = fine ? t : 0;
            p.first[s] = fine ? b : 0;
            if (fine)
                p.length_out[s] = mine[i].length;
            else if (p.length_out != p.length)
                p.length_out[s] = p.length[s];
            t += mine[i].tokens;
            b += mine[i].blocks;
        }
        token_at += all_tokens;
        block_at += all_blocks;
    }
    if (tid == 0) {
        if (EXTEND) p.begin_out[p.n_seqs] = fine ? token_at : 0;
        p.first[p.n_seqs] = fine ? block_at : 0;
    }
}

// The last sequence whose begin is at most `row`, which lies in [begin[0], begin[n_seqs]); the wave's rows
// are consecutive.  The wave looks at 64 bounds at once, first for its first row, then for all.
__device__ __forceinline__ int64_t sequence_of(const int64_t* begin, int64_t n_seqs, int64_t row, int64_t row0,
                                               int64_t last, int64_t* start) {
    const int lane = threadIdx.x & 63;
    int64_t lo = 0, hi = n_seqs;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kWave - 1) / kWave, at = lo + lane * step;
        const uint64_t below = __ballot(at < hi && begin[min(at, n_seqs)] <= row0);
        const int count = below == ~0ull ? kWave : __ffsll((unsigned long long)~below) - 1;
        lo += (int64_t)max(0, count - 1) * step;
        hi = min(hi, lo + step);
    }
    int64_t s = lo, from = begin[lo];
    for (int64_t base = lo + 1; base < n_seqs; base += kWave) {
        const int64_t b = base + lane < n_seqs ? begin[base + lane] : INT64_MAX;
        int count = 0;  // of these bounds, how many are at most row
#pragma unroll
        for (int bit = 32; bit > 0; bit >>= 1)
            if (__shfl(b, count + bit - 1, kWave) <= row) count += bit;
        if (count == 63 && __shfl(b, 63, kWave) <= row) count = 64;
        const int64_t at = __shfl(b, max(0, count - 1), kWave);
        if (count > 0) s = base + count - 1, from = at;
        if (__shfl(b, 63, kWave) > last) break;
    }
    *start = from;
    return s;
}

__global__ __launch_bounds__(256) void kv_pages_fill_kernel(Pages p) {
    const int64_t total = p.first[p.n_seqs + 1];
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x, row0 = row - (threadIdx.x & 63);
    if (row0 >= total) return;  // whole waves
    const int64_t last = min(total, row0 + kWave) - 1;
    int64_t begin;
    const int64_t s = sequence_of(p.begin_out, p.n_seqs, min(row, last), row0, last, &begin);
    if (row >= total) return;
    const int lb = p.log_block;
    const int64_t held = (int64_t)p.length_out[s] - p.more[s], pos = held + row - begin;
    const int64_t have = (held + ((int64_t)1 << lb) - 1) >> lb, block = pos >> lb, at = pos & ((1 << lb) - 1);
    int32_t* const entry = p.table + s * p.table_stride + block;
    const int32_t id = block >= have ? p.ids[p.first[s] + block - have] : *entry;
    if (id < 0) raise_status(p.status, MP_EINVAL);
    if (block >= have && at == 0) *entry = id;
    if (p.position_out) p.position_out[row] = (int32_t)pos;
    if (p.slot_out) p.slot_out[row] = ((int64_t)id << lb) + at;
}

__global__ __launch_bounds__(256) void kv_pages_free_kernel(Pages p) {
    const int64_t s = blockIdx.x, first = p.first[s], n = p.first[s + 1] - first;
    for (int64_t i = threadIdx.x; i < n; i += 256) {
        const int32_t id = p.table[s * p.table_stride + i];
        if (id < 0) raise_status(p.status, MP_EINVAL);
        p.ids_out[first + i] = id;
    }
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool pages_ok(const Pages& p, int32_t block, const void* ws, size_t ws_bytes) {
    if (p.n_seqs < 0 || p.n_seqs > kMaxCount || p.n_ids < 0 || p.n_ids > kMaxCount) return false;
    if (block != 16 && block != 32 && block != 64) return false;
    if (p.table_width < 0 || p.table_width > kMaxCount || p.table_stride < p.table_width) return false;
    if (p.n_seqs > 0 && p.table_stride > INT64_MAX / 8 / p.n_seqs) return false;
    if (!p.used || !p.used_out || !p.status || (!p.ids && p.n_ids > 0)) return false;
    if (p.n_seqs > 0 && (!p.length || !p.length_out || (!p.table && p.table_width > 0))) return false;
    return ws && aligned(ws, 16) && ws_bytes >= mp_kv_pages_workspace_size(p.n_seqs);
}

int log_of(int32_t block) { return block == 16 ? 4 : block == 32 ? 5 : 6; }

}  // namespace

}  // namespace mp

using namespace mp;

extern "C" size_t mp_kv_pages_workspace_size(int64_t n_seqs) {
    return n_seqs < 0 || n_seqs > kMaxCount ? 0 : ((size_t)n_seqs + 2) * 8;
}

extern "C" int32_t mp_kv_extend(const int32_t* ids, int64_t n_ids, const int64_t* used, int32_t* table,
                                int64_t table_stride, int64_t table_width, int32_t block,
                                const int32_t* length, const int32_t* more, int64_t n_seqs,
                                int64_t n_tokens, int32_t* length_out, int64_t* used_out,
                                int64_t* begin_out, int32_t* position_out, int64_t* slot_out,
                                void* workspace, size_t workspace_bytes, int32_t* status_out,
                                void* stream) {
    Pages p = {};
    p.ids = ids, p.n_ids = n_ids, p.used = used, p.table = table, p.table_stride = table_stride;
    p.table_width = table_width, p.length = length, p.more = more, p.n_seqs = n_seqs, p.n_tokens = n_tokens;
    p.length_out = length_out, p.used_out = used_out, p.begin_out = begin_out, p.position_out = position_out;
    p.slot_out = slot_out, p.first = static_cast<int64_t*>(workspace), p.status = status_out;
    if (!pages_ok(p, block, workspace, workspace_bytes) || !begin_out || (!more && n_seqs > 0)) return MP_EINVAL;
    if (n_tokens < 0 || n_tokens > kMaxCount) return MP_EINVAL;
    p.log_block = log_of(block);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    kv_pages_sum_kernel<true><<<1, kThreads, 0, st>>>(p);
    if (n_tokens > 0) kv_pages_fill_kernel<<<dim3((uint32_t)((n_tokens + 255) / 256)), 256, 0, st>>>(p);
    return hipGetLastError() == hipSuccess ? MP_OK : MP_EDEVICE;
}

extern "C" int32_t mp_kv_release(int32_t* ids, int64_t n_ids, const int64_t* used, const int32_t* table,
                                 int64_t table_stride, int64_t table_width, int32_t block,
                                 const int32_t* length, const uint8_t* done, int64_t n_seqs,
                                 int32_t* length_out, int64_t* used_out, void* workspace,
                                 size_t workspace_bytes, int32_t* status_out, void* stream) {
    Pages p = {};
    p.ids = ids, p.ids_out = ids, p.n_ids = n_ids, p.used = used, p.table = const_cast<int32_t*>(table);
    p.table_stride = table_stride, p.table_width = table_width, p.length = length, p.done = done;
    p.n_seqs = n_seqs, p.length_out = length_out, p.used_out = used_out;
    p.first = static_cast<int64_t*>(workspace), p.status = status_out;
    if (!pages_ok(p, block, workspace, workspace_bytes) || (!done && n_seqs > 0)) return MP_EINVAL;
    if (!grid_ok(n_seqs, 256)) return MP_EINVAL;
    p.log_block = log_of(block);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    kv_pages_sum_kernel<false><<<1, kThreads, 0, st>>>(p);
    if (n_seqs > 0) kv_pages_free_kernel<<<dim3((uint32_t)n_seqs), 256, 0, st>>>(p);
    return hipGetLastError() == hipSuccess ? MP_OK : MP_EDEVICE;
}
