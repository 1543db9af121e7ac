// Sanitizer driver for the host side of the pages' and the rotary positions' entry points (test
// infrastructure): built with their sources by tests/test_kv_more_sanitizers.py with the host pass under
// -fsanitize=address,undefined and run without a GPU.  Calls over the ends of their arguments' ranges, which the
// host checks must refuse.
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
    const int64_t counts[] = {INT64_MIN, -1, 0, 1, 4096, (int64_t)1 << 30, (int64_t)1 << 31, (int64_t)1 << 62, INT64_MAX};
    int32_t* const i32 = reinterpret_cast<int32_t*>(space);
    int64_t* const i64 = reinterpret_cast<int64_t*>(space);
    uint8_t* const u8 = reinterpret_cast<uint8_t*>(space);
    int32_t status = 0;
    for (int64_t n : counts) {
        (void)mp_kv_pages_workspace_size(n);
        for (int64_t m : counts)
            for (int64_t w : counts) {
                // no workspace: refused whatever the counts are
                CHECK(mp_kv_extend(i32, m, i64, i32, w, w, 64, i32, i32, n, m, i32, i64, i64, i32, i64, nullptr, 0, &status,
                                   nullptr) == MP_EINVAL);
                CHECK(mp_kv_extend(i32, n, i64, i32, w, m, 16, i32, i32, w, n, i32, i64, i64, nullptr, nullptr, space, 0,
                                   &status, nullptr) == MP_EINVAL);
                CHECK(mp_kv_release(i32, m, i64, i32, w, w, 32, i32, u8, n, i32, i64, nullptr, 0, &status, nullptr) ==
                      MP_EINVAL);
                CHECK(mp_kv_release(i32, n, i64, i32, w, m, 16, i32, u8, w, i32, i64, space, 0, &status, nullptr) ==
                      MP_EINVAL);
            }
    }
    const int32_t heads[] = {INT32_MIN, -1, 0, 1, 1 << 16, INT32_MAX};
    const double* const freq = reinterpret_cast<const double*>(space);
    for (int64_t n : counts)
        for (int32_t h : heads)
            for (int32_t d : heads)
                for (int64_t stride : counts) {
                    mp_kv_rows r = {space, stride, stride, MP_BF16}, bad = {space, stride, stride, 9};
                    CHECK(mp_rotate(i32, n, freq, d, MP_ROTARY_PAIRS, 1.0f, 0, d, &r, h, &r, &r, h, &bad, nullptr) ==
                              MP_EINVAL ||
                          h == 0);
                    CHECK(mp_rotate(i32, n, freq, 3, MP_ROTARY_HALVES, 1.0f, 1, d, &r, h, &r, nullptr, 0, nullptr, nullptr) ==
                          MP_EINVAL);
                    CHECK(mp_rotate(i32, n, nullptr, 2, MP_ROTARY_HALVES, 1.0f, 1, d, &r, h, &r, nullptr, 0, nullptr,
                                    nullptr) == MP_EINVAL);
                }
    // nothing to do: no launch
    mp_kv_rows r = {nullptr, 128, 64, MP_F32};
    CHECK(mp_rotate(nullptr, 0, freq, 64, MP_ROTARY_HALVES, 1.0f, 0, 64, &r, 2, &r, nullptr, 0, nullptr, nullptr) == MP_OK);
    if (failures == 0) printf("all checks passed\n");
    return failures != 0;
}
