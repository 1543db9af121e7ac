// C ABI entry points of the 8-bit key/value cache: host-side argument checks, then
// launches on the caller's stream.  No allocation, no synchronisation.
#include "kv.hpp"

using namespace mp;

namespace {

int32_t launched(hipError_t e) { return e == hipSuccess ? MP_OK : MP_EDEVICE; }

constexpr int64_t kMaxCount = (int64_t)1 << 30;  // sequences, rows of a call, blocks
constexpr int32_t kMaxHeads = 1 << 16;
// Tokens of a sequence: the kernels step through it, and look some steps ahead, in 32 bits.
constexpr int64_t kMostTokens = INT32_MAX - 4096;

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

bool shape_ok(const mp_kv_cache* c) {
    if (!c) return false;
    if (c->n_blocks < 1 || c->n_blocks > kMaxCount || c->heads < 1 || c->heads > kMaxHeads)
        return false;
    if (c->dim != 64 && c->dim != 128 && c->dim != 256) return false;
    if (c->block != 16 && c->block != 32 && c->block != 64) return false;
    return c->kind == MP_KV_E4M3 || c->kind == MP_KV_INT8;
}

bool counts_ok(const mp_kv_cache* c, const mp_kv_seqs* s) {
    if (!s) return false;
    if (s->n_seqs < 0 || s->n_seqs > kMaxCount || s->n_tokens < 0 || s->n_tokens > kMaxCount)
        return false;
    if (s->table_width < 0 || s->table_width > kMaxCount || s->table_stride < s->table_width)
        return false;
    if (s->n_seqs > 0 && s->table_stride > INT64_MAX / 8 / s->n_seqs) return false;
    if (s->most_new < 0 || s->longest < 0 || s->longest > kMostTokens) return false;
    return s->longest <= s->table_width * c->block;
}

bool cache_ok(const mp_kv_cache* c) {
    if (!c->k_code || !c->v_code || !c->k_exp || !c->v_exp || !c->mean_code || !c->mean_exp)
        return false;
    return aligned(c->k_code, 16) && aligned(c->v_code, 16) && aligned(c->mean_code, 8);
}

bool seqs_ok(const mp_kv_seqs* s) {
    if (s->n_seqs == 0) return s->n_tokens == 0;
    if (!s->length || (!s->table && s->table_width > 0)) return false;
    return s->begin || s->n_tokens == s->n_seqs;
}

// Rows of `tokens` x `heads`; strides that keep every element's offset within 64 bits.
bool rows_ok(const mp_kv_rows* r, int64_t tokens, int64_t heads, bool f32, KvRows* out) {
    if (!r || (!r->data && tokens > 0)) return false;
    if (r->dtype != MP_BF16 && r->dtype != MP_F16 && !(f32 && r->dtype == MP_F32)) return false;
    const int64_t most = (int64_t)1 << 58;
    if (r->token_stride < 0 || r->head_stride < 0 || r->head_stride > most / heads) return false;
    if (tokens > 0 && r->token_stride > most / tokens) return false;
    const size_t size = r->dtype == MP_F32 ? 4 : 2;
    if (!aligned(r->data, size)) return false;
    out->data = static_cast<char*>(r->data);
    out->token_stride = r->token_stride;
    out->head_stride = r->head_stride;
    out->dtype = r->dtype;
    out->wide = aligned(r->data, 16) && r->token_stride * size % 16 == 0 &&
                r->head_stride * size % 16 == 0;
    return true;
}

// Whether no two elements of rows that a call writes share a place: one axis lies within a step
// of the other.
bool rows_apart(const mp_kv_rows* r, int64_t tokens, int64_t heads, int64_t dim) {
    const bool tokens_outside = r->token_stride >= r->head_stride;
    const int64_t inner = tokens_outside ? r->head_stride : r->token_stride;
    const int64_t outer = tokens_outside ? r->token_stride : r->head_stride;
    const int64_t n_inner = tokens_outside ? heads : tokens, n_outer = tokens_outside ? tokens : heads;
    if (n_inner > 1 && inner < dim) return false;
    const int64_t extent = n_inner > 1 ? (n_inner - 1) * inner + dim : dim;
    return n_outer <= 1 || outer >= extent;
}

KvArgs args_of(const mp_kv_cache* c, const mp_kv_seqs* s, int32_t* status) {
    KvArgs a = {*c, *s, c->block == 16 ? 4 : c->block == 32 ? 5 : 6, status};
    return a;
}

bool heads_ok(const mp_kv_cache* c, int32_t q_heads) {
    return q_heads >= c->heads && q_heads % c->heads == 0 && q_heads <= kMaxHeads;
}

// Query heads of a key head whose codes fit the scores' LDS.
constexpr int32_t kMaxSelectGroup = 128;

int32_t move_rows(const mp_kv_cache* cache, const mp_kv_seqs* seqs, const mp_kv_rows* k,
                  const mp_kv_rows* v, int32_t* status_out, void* stream, bool write) {
    KvRows kr, vr;
    if (!shape_ok(cache) || !counts_ok(cache, seqs) || !cache_ok(cache) || !seqs_ok(seqs) ||
        !status_out ||
        !rows_ok(k, seqs->n_tokens, cache->heads, true, &kr) ||
        !rows_ok(v, seqs->n_tokens, cache->heads, true, &vr))
        return MP_EINVAL;
    if (!write && (!rows_apart(k, seqs->n_tokens, cache->heads, cache->dim) ||
                   !rows_apart(v, seqs->n_tokens, cache->heads, cache->dim)))
        return MP_EINVAL;
    const KvArgs a = args_of(cache, seqs, status_out);
    if (!grid_ok(write ? kv_write_groups(a) : kv_read_groups(a), 256)) return MP_EINVAL;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return launched(write ? launch_kv_write(a, kr, vr, st) : launch_kv_read(a, kr, vr, st));
}

}  // namespace

extern "C" int32_t mp_kv_write(const mp_kv_cache* cache, const mp_kv_seqs* seqs,
                               const mp_kv_rows* k, const mp_kv_rows* v, int32_t* status_out,
                               void* stream) {
    return move_rows(cache, seqs, k, v, status_out, stream, true);
}

extern "C" int32_t mp_kv_read(const mp_kv_cache* cache, const mp_kv_seqs* seqs,
                              const mp_kv_rows* k_out, const mp_kv_rows* v_out,
                              int32_t* status_out, void* stream) {
    return move_rows(cache, seqs, k_out, v_out, status_out, stream, false);
}

extern "C" int32_t mp_kv_attend(const mp_kv_cache* cache, const mp_kv_seqs* seqs,
                                const mp_kv_rows* q, int32_t q_heads, float scale,
                                const int32_t* blocks, int64_t keep, const mp_kv_rows* out,
                                float* lse_out, void* workspace, size_t workspace_bytes,
                                int32_t* status_out, void* stream) {
    KvAttend k = {};
    if (!shape_ok(cache) || !counts_ok(cache, seqs) || !cache_ok(cache) || !seqs_ok(seqs) ||
        !status_out || !heads_ok(cache, q_heads))
        return MP_EINVAL;
    if (keep < 0 || keep > kMaxCount / 64) return MP_EINVAL;
    if ((blocks != nullptr) != (keep > 0) && seqs->n_tokens > 0) return MP_EINVAL;
    if (!rows_ok(q, seqs->n_tokens, q_heads, false, &k.q) ||
        !rows_ok(out, seqs->n_tokens, q_heads, false, &k.out) || q->dtype != out->dtype ||
        !rows_apart(out, seqs->n_tokens, q_heads, cache->dim))
        return MP_EINVAL;
    k.shape = kv_attend_shape(*cache, *seqs, q_heads, keep);
    if (!k.shape.ok || workspace_bytes < k.shape.workspace || !aligned(workspace, 16) ||
        (k.shape.workspace > 0 && !workspace))
        return MP_EINVAL;
    k.a = args_of(cache, seqs, status_out);
    k.scale = scale;
    k.group = q_heads / cache->heads;
    k.blocks = blocks;
    k.keep = (int32_t)keep;
    k.lse = lse_out;
    k.ws = workspace;
    return launched(launch_kv_attend(k, static_cast<hipStream_t>(stream)));
}

extern "C" int32_t mp_kv_select(const mp_kv_cache* cache, const mp_kv_seqs* seqs,
                                const mp_kv_rows* q, int32_t q_heads, int64_t keep, int64_t first,
                                int64_t recent, int32_t* blocks_out, void* workspace,
                                size_t workspace_bytes, int32_t* status_out, void* stream) {
    KvSelect k = {};
    if (!shape_ok(cache) || !counts_ok(cache, seqs) || !cache_ok(cache) || !seqs_ok(seqs) ||
        !status_out || !heads_ok(cache, q_heads) || q_heads / cache->heads > kMaxSelectGroup)
        return MP_EINVAL;
    if (keep < 1 || keep > kMaxCount / 64 || first < 0 || recent < 1 || first > keep ||
        recent > keep - first || (!blocks_out && seqs->n_tokens > 0))
        return MP_EINVAL;
    if (!rows_ok(q, seqs->n_tokens, q_heads, false, &k.q)) return MP_EINVAL;
    const KvSelectShape sh = kv_select_shape(*cache, *seqs, q_heads);
    if (!sh.ok || workspace_bytes < sh.workspace || (sh.workspace > 0 && !workspace) || !aligned(workspace, 16))
        return MP_EINVAL;
    k.a = args_of(cache, seqs, status_out);
    k.group = q_heads / cache->heads;
    k.keep = (int32_t)keep;
    k.first = (int32_t)first;
    k.recent = (int32_t)recent;
    k.out = blocks_out;
    k.scores = static_cast<float*>(workspace);
    k.score_stride = sh.score_stride;
    k.tokens = sh.tokens;
    k.units = sh.units;
    return launched(launch_kv_select(k, static_cast<hipStream_t>(stream)));
}

extern "C" size_t mp_kv_workspace_size(int32_t op, const mp_kv_cache* cache,
                                       const mp_kv_seqs* seqs, int32_t q_heads, int64_t keep) {
    if (!shape_ok(cache) || !counts_ok(cache, seqs) || !heads_ok(cache, q_heads) || keep < 0 ||
        keep > kMaxCount / 64)
        return 0;
    if (op == MP_OP_KV_ATTEND) {
        const KvAttendShape sh = kv_attend_shape(*cache, *seqs, q_heads, keep);
        return sh.ok ? sh.workspace : 0;
    }
    if (op == MP_OP_KV_SELECT) {
        if (q_heads / cache->heads > kMaxSelectGroup) return 0;
        return kv_select_shape(*cache, *seqs, q_heads).workspace;
    }
    return 0;
}
