// Blocks given to sequences and taken back: tables, lengths, bounds, positions and slots of a step, on
// the device.
//
// Two sums run over the sequences (tokens, blocks); what hangs on them is one store a token, a
// block, a sequence.  One workgroup has the sums; nothing is changed where an argument is wrong or the pool
// is short, so it knows both totals before it writes.  Where few tokens (or few table entries) follow it
// writes those too; otherwise a second launch does, a wave 256 tokens, a workgroup a sequence.
#include "kv.hpp"

namespace mp {

namespace {

constexpr int kThreads = 1024;       // of the workgroup that sums
// Calls of one launch: sequences (one a thread), new tokens, table entries that a release may read.
constexpr int kOneSeqs = kThreads, kOneTokens = 4096, kOneEntries = 1 << 16;
constexpr int kRun = 4;              // groups of 64 tokens that a wave of the second launch writes
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

// Of a sequence that holds `length` tokens; `with`: those it gets, or whether it ends.
template <bool EXTEND>
__device__ __forceinline__ Need need_of(const Pages& p, int32_t length, int32_t with) {
    Need n = {0, 0, length, true};
    const int64_t t = ((int64_t)1 << p.log_block) - 1, room = p.table_width << p.log_block;
    n.ok = length >= 0 && length <= room;
    if (EXTEND) {
        const int64_t after = (int64_t)length + with;
        n.ok = n.ok && with >= 0 && after <= room && after <= INT32_MAX;
        n.tokens = with;
        n.blocks = ((after + t) >> p.log_block) - ((length + t) >> p.log_block);
        n.length = (int32_t)after;
    } else if (with) {
        n.blocks = (length + t) >> p.log_block;
        n.length = 0;
    }
    if (!n.ok) n.tokens = n.blocks = 0;
    return n;
}

// What a new token of sequence s writes: `offset` tokens after the `held` ones; `first` its first new block's
// place in ids.
__device__ __forceinline__ void place_token(const Pages& p, int32_t s, int32_t row, int32_t held, int32_t offset,
                                            int32_t first) {
    const int lb = p.log_block;
    const int32_t pos = held + offset, have = (int32_t)(((uint32_t)held + (1u << lb) - 1) >> lb);
    const int32_t block = pos >> lb, at = pos & ((1 << lb) - 1);
    int32_t* const entry = p.table + s * p.table_stride + block;
    const int32_t id = block >= have ? p.ids[first + block - have] : *entry;
    if (id < 0) raise_status(p.status, MP_EINVAL);
    if (block >= have && at == 0) *entry = id;
    if (p.position_out) p.position_out[row] = pos;
    if (p.slot_out) p.slot_out[row] = ((int64_t)id << lb) + at;
}

__device__ __forceinline__ void free_blocks(const Pages& p, int64_t s, int64_t first, int64_t n, int lane, int lanes) {
    for (int64_t i = lane; i < n; i += lanes) {
        const int32_t id = p.table[s * p.table_stride + i];
        if (id < 0) raise_status(p.status, MP_EINVAL);
        p.ids_out[first + i] = id;
    }
}

// Sums before a thread's own and over the workgroup, of two numbers at once, and the least code.
struct Sums {
    int64_t a, b, all_a, all_b;
    int32_t code;
};
__device__ __forceinline__ Sums block_sums(int64_t a, int64_t b, int32_t code, int64_t (*scratch)[3]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t up_a = wave_inclusive_sum(a), up_b = wave_inclusive_sum(b);
    const bool bad = __any(code != MP_OK);
    if (lane == 63) scratch[wave][0] = up_a, scratch[wave][1] = up_b, scratch[wave][2] = bad;
    __syncthreads();
    Sums s = {up_a - a, up_b - b, 0, 0, MP_OK};
#pragma unroll 4  // all at once take a hundred registers
    for (int w = 0; w < kThreads / 64; ++w) {
        const int64_t x = scratch[w][0], y = scratch[w][1];
        s.a += w < wave ? x : 0, s.b += w < wave ? y : 0;
        s.all_a += x, s.all_b += y;
        if (scratch[w][2]) s.code = MP_EINVAL;
    }
    return s;
}

// ITEMS sequences of a thread at once; ONE (with one item): the call's only launch.  256 sequences of a token each
// 5 us, and 5 us to take back a tenth of them; 2048 sequences' sums 5 and 4 us.  Latency bounds it: loads, one
// exchange through LDS, stores.
template <bool EXTEND, int ITEMS, bool ONE>
__global__ __launch_bounds__(kThreads) void kv_pages_sum_kernel(Pages p) {
    __shared__ int64_t scratch[2][kThreads / 64][3];
    __shared__ int32_t bounds[ONE ? kOneSeqs + 1 : 1];  // ONE: tokens before each sequence
    __shared__ int64_t firsts[ONE ? kOneSeqs : 1];
    __shared__ int32_t lengths[ONE ? kOneSeqs : 1];     // held before (extend); blocks (release)
    const int tid = threadIdx.x;
    const int64_t used = *p.used;
    int32_t mine[ITEMS], with[ITEMS];  // lengths, and need_of's
    int64_t tokens = 0, blocks = 0;
    int32_t code = used >= 0 && used <= p.n_ids ? MP_OK : MP_EINVAL;
    const int64_t step = kThreads * ITEMS;
    auto load = [&](int64_t s0) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int64_t s = s0 + tid * ITEMS + i;
            const bool some = s < p.n_seqs;
            mine[i] = some ? p.length[s] : 0;
            with[i] = !some ? 0 : EXTEND ? p.more[s] : p.done[s];
        }
    };
    load(0);
    // the first pass: all totals, before anything is written
    for (int64_t s0 = 0;;) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const Need need = need_of<EXTEND>(p, mine[i], with[i]);
            tokens += need.tokens;
            blocks += need.blocks;
            if (!need.ok) code = MP_EINVAL;
        }
        s0 += step;
        if (s0 >= p.n_seqs) break;
        load(s0);
    }
    Sums sums = block_sums(tokens, blocks, code, scratch[0]);
    code = sums.code;
    if (code == MP_OK && EXTEND && (sums.all_a > p.n_tokens || sums.all_b > p.n_ids - used)) code = MP_ENOSPC;
    if (code == MP_OK && !EXTEND && sums.all_b > used) code = MP_EINVAL;
    const bool fine = code == MP_OK;
    const int64_t total = fine ? sums.all_a : 0;
    if (tid == 0) {
        raise_status(p.status, code);
        *p.used_out = !fine ? used : EXTEND ? used + sums.all_b : used - sums.all_b;
        if (EXTEND) p.begin_out[p.n_seqs] = total;
        if (!ONE) {
            p.first[p.n_seqs] = !fine ? 0 : EXTEND ? used + sums.all_b : used;
            p.first[p.n_seqs + 1] = total;
        } else {
            bounds[p.n_seqs] = (int32_t)total;
        }
    }
    int64_t token_at = 0, block_at = EXTEND ? used : used - sums.all_b;
    for (int64_t s0 = 0, turn = 1; s0 < p.n_seqs; s0 += step, ++turn) {
        if (p.n_seqs > step) {  // more than one pass's: this one's again, and its own sums
            load(s0);
            int64_t a = 0, b = 0;
#pragma unroll
            for (int i = 0; i < ITEMS; ++i) {
                const Need need = need_of<EXTEND>(p, mine[i], with[i]);
                a += need.tokens, b += need.blocks;
            }
            __syncthreads();
            sums = block_sums(a, b, MP_OK, scratch[turn & 1]);
        }
        int64_t t = token_at + sums.a, b = block_at + sums.b;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int64_t s = s0 + tid * ITEMS + i;
            if (s >= p.n_seqs) continue;
            const Need need = need_of<EXTEND>(p, mine[i], with[i]);
            if (EXTEND) p.begin_out[s] = fine ? t : 0;
            if (ONE) {
                if (EXTEND) bounds[s] = fine ? (int32_t)t : 0;
                firsts[s] = b;
                lengths[s] = EXTEND ? mine[i] : fine ? (int32_t)need.blocks : 0;
            } else {
                p.first[s] = fine ? b : 0;
            }
            if (fine)
                p.length_out[s] = need.length;
            else if (p.length_out != p.length)
                p.length_out[s] = mine[i];
            t += need.tokens;
            b += need.blocks;
        }
        token_at += sums.all_a;
        block_at += sums.all_b;
    }
    if (!ONE) return;
    __syncthreads();
    if (EXTEND) {
        for (int row = tid; row < total; row += kThreads) {
            int lo = 0, hi = (int)p.n_seqs;  // bounds[lo] <= row < bounds[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (bounds[mid] <= row)
                    lo = mid;
                else
                    hi = mid;
            }
            place_token(p, lo, row, lengths[lo], row - bounds[lo], (int32_t)firsts[lo]);
        }
    } else {
        for (int s = tid >> 6; s < p.n_seqs; s += kThreads / 64)
            free_blocks(p, s, firsts[s], lengths[s], tid & 63, 64);
    }
}

// A wave has kRun groups of 64 consecutive tokens.  It finds the sequence of its first one, 64 bounds a turn, and
// those of the others among the next 64 bounds at a time.  1.4 million tokens of 2048 sequences 12 us, for 17 MB of
// stores: its instructions (14 us with 64-bit places) and a chain of loads, bounds, a sequence's numbers, its ids.
__global__ __launch_bounds__(256) void kv_pages_fill_kernel(Pages p) {
    // sequences, tokens of the call, positions and places in ids are all below 2^31
    const int32_t total = (int32_t)p.first[p.n_seqs + 1], n_seqs = (int32_t)p.n_seqs;
    const auto begin = [&](int32_t s) { return (int32_t)p.begin_out[s]; };
    const int lane = threadIdx.x & 63;
    const int64_t row00 = ((int64_t)blockIdx.x * 4 + (threadIdx.x >> 6)) * (64 * kRun);
    if (row00 >= total) return;  // whole waves
    int32_t row0 = (int32_t)row00, lo = 0, hi = n_seqs;
    while (hi - lo > 1) {
        const int32_t step = (hi - lo + kWave - 1) / kWave;
        const int64_t at = lo + (int64_t)lane * step;
        const uint64_t below = __ballot(at < hi && begin((int32_t)min(at, (int64_t)n_seqs)) <= row0);
        const int count = below == ~0ull ? kWave : __ffsll((unsigned long long)~below) - 1;
        lo += max(0, count - 1) * step;
        hi = min(hi, lo + step);
    }
    int32_t base = lo + 1, from_lo = begin(lo);  // sequence lo begins at from_lo; the bounds from `base` on
    int32_t b = base + lane < n_seqs ? begin(base + lane) : INT32_MAX;
    for (int run = 0; run < kRun && row0 < total; ++run, row0 += 64) {
        const int32_t row = row0 + lane, last = min(total, row0 + 64) - 1, find = min(row, last);
        int32_t s = lo, from = from_lo;
        for (;;) {
            int count = 0;  // of these bounds, how many are at most the lane's row
#pragma unroll
            for (int bit = 32; bit > 0; bit >>= 1)
                if (__shfl(b, count + bit - 1, kWave) <= find) count += bit;
            const int32_t end = __builtin_amdgcn_readlane(b, 63);
            if (count == 63 && end <= find) count = 64;
            const int32_t at = __shfl(b, max(0, count - 1), kWave);
            if (count > 0) s = base + count - 1, from = at;
            if (end > last) break;  // INT32_MAX past the last sequence
            lo = base + 63, from_lo = end, base += kWave;
            b = base + lane < n_seqs ? begin(base + lane) : INT32_MAX;
        }
        if (row < total)
            place_token(p, s, row, p.length_out[s] - p.more[s], row - from, (int32_t)p.first[s]);
    }
}

__global__ __launch_bounds__(256) void kv_pages_free_kernel(Pages p) {
    const int64_t s = blockIdx.x, first = p.first[s];
    free_blocks(p, s, first, p.first[s + 1] - first, threadIdx.x, 256);
}

// Four sequences a thread where one is not enough: a call of 2048 / 8192 / 65536 14 / 29 / 142 us, with one each
// 19 / 39 / 214, with eight 14 / 28 / 210.
template <bool EXTEND>
void launch_sums(const Pages& p, bool one, hipStream_t st) {
    if (one)
        kv_pages_sum_kernel<EXTEND, 1, true><<<1, kThreads, 0, st>>>(p);
    else if (p.n_seqs <= kThreads)
        kv_pages_sum_kernel<EXTEND, 1, false><<<1, kThreads, 0, st>>>(p);
    else
        kv_pages_sum_kernel<EXTEND, 4, false><<<1, kThreads, 0, st>>>(p);
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
    const bool one = n_seqs <= kOneSeqs && n_tokens <= kOneTokens;
    launch_sums<true>(p, one, st);
    const int64_t per = 256 * kRun;
    if (!one && n_tokens > 0) kv_pages_fill_kernel<<<dim3((uint32_t)((n_tokens + per - 1) / per)), 256, 0, st>>>(p);
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
    const bool one = n_seqs <= kOneSeqs && n_seqs * table_width <= kOneEntries;
    launch_sums<false>(p, one, st);
    if (!one) kv_pages_free_kernel<<<dim3((uint32_t)n_seqs), 256, 0, st>>>(p);
    return hipGetLastError() == hipSuccess ? MP_OK : MP_EDEVICE;
}
