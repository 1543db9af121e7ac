// Sanitizer driver for the sizes that the host side of the key/value cache computes (test infrastructure): built
// with its sources by tests/test_kv4_limit_sanitizers.py with the host pass under
// -fsanitize=address,undefined and run without a GPU.  Counts, lengths and bounds up to the ends of what is
// accepted, for every kind and type of rows; and what the launches rely on.
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
    const int64_t counts[] = {0, 1, 63, 4096, (int64_t)1 << 20, (int64_t)1 << 30};
    const int64_t lengths[] = {0, 1, 1024, 1 << 17, 1 << 26, INT32_MAX - 4096};
    const int64_t news[] = {0, 1, 300, (int64_t)1 << 30, (int64_t)1 << 40, INT64_MAX};
    const int32_t heads[] = {1, 8, 1 << 16}, groups[] = {1, 4, 1 << 10, 1 << 16}, dims[] = {64, 128, 256};
    for (int32_t kind : {MP_KV_E4M3, MP_KV_INT8, MP_KV_E2M1})
        for (int64_t seqs : counts)
            for (int64_t tokens : counts)
                for (int64_t longest : lengths)
                    for (int64_t most_new : news)
                        for (int32_t h : heads)
                            for (int32_t g : groups)
                                for (int32_t dim : dims) {
                                    mp_kv_cache c = {};
                                    c.n_blocks = 16, c.heads = h, c.dim = dim, c.block = 16, c.kind = kind;
                                    mp_kv_seqs s = {};
                                    s.table_width = s.table_stride = (int64_t)1 << 30;
                                    s.n_seqs = seqs, s.n_tokens = tokens, s.most_new = most_new, s.longest = longest;
                                    const int32_t q_heads = (int64_t)h * g > (1 << 16) ? h : h * g;
                                    for (const int64_t* b : {(const int64_t*)&begin, (const int64_t*)nullptr}) {
                                        s.begin = b;
                                        (void)mp_kv_workspace_size(MP_OP_KV_ATTEND, &c, &s, q_heads, 0);
                                        for (int32_t dtype : {MP_BF16, MP_F16}) {
                                            const mp::KvAttendShape sh = mp::kv_attend_shape(c, s, q_heads, 0, dtype);
                                            if (!sh.ok) continue;
                                            // every workgroup's place in 32 bits, chunks that hold the longest sequence
                                            CHECK(sh.units >= 0 && sh.n_chunks >= 1);
                                            CHECK((unsigned __int128)sh.units * h * sh.n_chunks < ((uint64_t)1 << 31));
                                            CHECK(sh.chunk > 0 && sh.chunk * sh.n_chunks >= longest);
                                            // as many rows of every sequence as they have at most
                                            if (sh.each) CHECK(b && most_new <= tokens && tokens == seqs * most_new);
                                            if (sh.each) CHECK((int64_t)sh.each == most_new * (q_heads / h));
                                        }
                                    }
                                }
    if (failures) return 1;
    printf("all checks passed\n");
    return 0;
}
