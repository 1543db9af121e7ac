// Sanitizer driver for the host side of the key/value cache's entry points (test
// infrastructure): built with their sources by tests/test_kv_sanitizers.py with the host
// pass under -fsanitize=address,undefined and run without a GPU.  Workspace queries over
// the whole ranges of their arguments, and calls that the host checks must refuse.
#include <stdint.h>
#include <stdio.h>

#include "memoplan.h"

static int failures = 0;
#define CHECK(c)                                                             \
    do {                                                                     \
        if (!(c)) {                                                          \
            fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c);  \
            ++failures;                                                      \
        }                                                                    \
    } while (0)

int main() {
    alignas(16) static char space[64];
    const int64_t counts[] = {INT64_MIN, -1, 0, 1, 255, 4096, (int64_t)1 << 20, (int64_t)1 << 30,
                              (int64_t)1 << 31, (int64_t)1 << 40, INT64_MAX};
    const int32_t heads[] = {INT32_MIN, -1, 0, 1, 8, 1 << 16, INT32_MAX};
    for (int64_t n : counts)
        for (int64_t tokens : counts)
            for (int64_t width : counts)
                for (int32_t h : heads) {
                    mp_kv_cache c = {};
                    c.n_blocks = 16, c.heads = h, c.dim = 128, c.block = 64;
                    mp_kv_seqs s = {};
                    s.table_stride = s.table_width = width;
                    s.n_seqs = n, s.n_tokens = tokens, s.most_new = tokens;
                    s.longest = width > 0 && width < (1 << 24) ? width * 64 : 0;
                    for (int64_t keep : counts) {
                        (void)mp_kv_workspace_size(MP_OP_KV_ATTEND, &c, &s, h, keep);
                        s.begin = reinterpret_cast<int64_t*>(space);
                        (void)mp_kv_workspace_size(MP_OP_KV_ATTEND, &c, &s, h, keep);
                        (void)mp_kv_workspace_size(MP_OP_KV_SELECT, &c, &s, 8, keep);
                        s.begin = nullptr;
                    }
                }
    int32_t status = 0;
    mp_kv_cache c = {};
    mp_kv_seqs s = {};
    mp_kv_rows r = {};
    CHECK(mp_kv_write(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr) == MP_EINVAL);
    CHECK(mp_kv_write(&c, &s, &r, &r, &status, nullptr) == MP_EINVAL);
    CHECK(mp_kv_read(&c, &s, &r, &r, &status, nullptr) == MP_EINVAL);
    CHECK(mp_kv_attend(&c, &s, &r, 1, 1.0f, nullptr, 0, &r, nullptr, nullptr, 0, &status, nullptr) ==
          MP_EINVAL);
    CHECK(mp_kv_select(&c, &s, &r, 1, 1, 0, 1, nullptr, nullptr, 0, &status, nullptr) == MP_EINVAL);
    uint8_t* const p = reinterpret_cast<uint8_t*>(space);
    int8_t* const e = reinterpret_cast<int8_t*>(space);
    c = {p, p, e, e, e, e, 16, 8, 128, 64, MP_KV_INT8};
    s.n_seqs = 1, s.n_tokens = 1, s.table_stride = s.table_width = 4, s.longest = 256;
    s.table = s.length = reinterpret_cast<int32_t*>(space);
    for (int64_t stride : counts) {
        if (stride >= 0 && stride < ((int64_t)1 << 50)) continue;  // would pass
        r = {space, stride, 128, MP_BF16};
        CHECK(mp_kv_write(&c, &s, &r, &r, &status, nullptr) == MP_EINVAL);
        r = {space, 1024, stride, MP_BF16};
        CHECK(mp_kv_read(&c, &s, &r, &r, &status, nullptr) == MP_EINVAL);
    }
    r = {space, 1024, 128, MP_BF16};
    for (int64_t keep : counts) {
        if (keep > 0 && keep < (1 << 24)) continue;
        CHECK(mp_kv_select(&c, &s, &r, 8, keep, 1, 1, s.table ? const_cast<int32_t*>(s.table) : nullptr,
                           space, 1 << 20, &status, nullptr) == MP_EINVAL);
        CHECK(mp_kv_select(&c, &s, &r, 8, 4, keep == 0 ? -1 : keep, 1, const_cast<int32_t*>(s.table),
                           space, 1 << 20, &status, nullptr) == MP_EINVAL);
        CHECK(mp_kv_attend(&c, &s, &r, 8, 1.0f, s.table, keep, &r, nullptr, space, 1 << 20, &status,
                           nullptr) == MP_EINVAL);
    }
    if (failures) return 1;
    printf("all checks passed\n");
    return 0;
}
