// Sanitizer driver for the sizes that the key/value cache's host side computes (test infrastructure):
// built with its sources by tests/test_kv_limit_sanitizers.py with the host pass under
// -fsanitize=address,undefined and run without a GPU.  Counts, lengths and bounds up to the ends of
// what is accepted; and the rule by which row groups are ordered, where a level would leave its bits.
#include <stdint.h>
#include <stdio.h>

#include "kv.hpp"

static int failures = 0;
#define CHECK(c)                                                             \
    do {                                                                     \
        if (!(c)) {                                                          \
            fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c);  \
            ++failures;                                                      \
        }                                                                    \
    } while (0)

int main() {
    int64_t begin = 0;
    const int64_t counts[] = {0, 1, 64, 4096, (int64_t)1 << 20, (int64_t)1 << 28, (int64_t)1 << 30};
    const int64_t lengths[] = {0, 1, 1024, 1 << 20, 1 << 26, 1 << 30, INT32_MAX - 4096};
    const int64_t news[] = {0, 1, 300, (int64_t)1 << 30, (int64_t)1 << 40, INT64_MAX};
    const int32_t heads[] = {1, 8, 1 << 16}, groups[] = {1, 4, 1 << 10, 1 << 16}, dims[] = {64, 128, 256};
    for (int64_t seqs : counts)
        for (int64_t tokens : counts)
            for (int64_t longest : lengths)
                for (int64_t most_new : news)
                    for (int32_t h : heads)
                        for (int32_t g : groups)
                            for (int32_t dim : dims) {
                                mp_kv_cache c = {};
                                c.n_blocks = 16, c.heads = h, c.dim = dim, c.block = 16;
                                mp_kv_seqs s = {};
                                s.table_width = (int64_t)1 << 30;
                                s.table_stride = seqs > 1 ? INT64_MAX / 8 / seqs : s.table_width;
                                if (s.table_stride < s.table_width) s.table_stride = s.table_width;
                                s.n_seqs = seqs, s.n_tokens = tokens, s.most_new = most_new;
                                s.longest = longest;
                                const int32_t q_heads = (int64_t)h * g > (1 << 16) ? h : h * g;
                                for (int64_t keep : {(int64_t)0, (int64_t)1, (int64_t)1 << 24}) {
                                    s.begin = &begin;
                                    (void)mp_kv_workspace_size(MP_OP_KV_ATTEND, &c, &s, q_heads, keep);
                                    (void)mp_kv_workspace_size(MP_OP_KV_SELECT, &c, &s, q_heads, keep);
                                    s.begin = nullptr;
                                    (void)mp_kv_workspace_size(MP_OP_KV_ATTEND, &c, &s, q_heads, keep);
                                    (void)mp_kv_workspace_size(MP_OP_KV_SELECT, &c, &s, q_heads, keep);
                                }
                            }
    // many long sequences of many query heads, in one chunk
    mp_kv_cache c = {};
    c.n_blocks = 16, c.heads = 1, c.dim = 64, c.block = 64;
    mp_kv_seqs s = {};
    s.begin = &begin, s.n_seqs = 8, s.n_tokens = 2048, s.most_new = 2048;
    s.table_width = s.table_stride = 1 << 26;
    for (int32_t group : {1, 16, 64, 256, 1024}) {
        for (int64_t longest : {(int64_t)1 << 16, (int64_t)1 << 24, (int64_t)1 << 27, (int64_t)INT32_MAX - 4096}) {
            s.longest = longest;
            const mp::KvAttendShape sh = mp::kv_attend_shape(c, s, group, 0);
            CHECK(sh.ok && sh.form == mp::KvForm::tiles);
            // its level: the rows before a group, over the group's
            if (sh.ordered) CHECK((unsigned __int128)longest * group / sh.rows < (1u << 30));
            if (sh.n_chunks == 1 && longest <= (1 << 24) && group <= 256) CHECK(sh.ordered);
        }
    }
    if (failures) return 1;
    printf("all checks passed\n");
    return 0;
}
