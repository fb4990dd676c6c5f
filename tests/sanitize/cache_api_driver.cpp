// Drives the entry points of csrc/fa_cache_api.hip through accepted and refused calls under host sanitizers, with stand-ins for
// the launchers; built by tests/test_cache_host.py, which checks the exit status and the line printed at the end.
#include <stdio.h>
#include <stdlib.h>

#include "../../paper_2407_08608_amd/csrc/fa_launch.h"

namespace fa {
int launch_rope(const Rows&, const Rows&, const Rows&, const Rows&, const double*, const int*, int, int, int, int, int, int, float, int,
                bool, int, hipStream_t) { return FA_OK; }
int launch_cache_write(const Rows&, const Rows&, const Cache&, const int*, int, int, int, int, hipStream_t) { return FA_OK; }
int launch_cache_read(const Cache&, void*, void*, int, int, int, int, hipStream_t) { return FA_OK; }
size_t fwd_cache_workspace_bytes(int, int, int, int, int, int, int) { return 64; }
int launch_fwd_cache(const Rows&, const Cache&, const int*, const int*, int, const Rows&, float*, void*, int, int, int, int, int, float,
                     int, hipStream_t) { return FA_OK; }
}  // namespace fa

static int failures = 0;
#define EXPECT(call, want)                                                        \
    do {                                                                          \
        const int got = (call);                                                   \
        if (got != (want)) {                                                      \
            printf("line %d: %s = %d, wanted %d\n", __LINE__, #call, got, want);  \
            ++failures;                                                           \
        }                                                                         \
    } while (0)

int main() {
    void* p = aligned_alloc(256, 4096);
    void* odd = (char*)p + 8;
    const double* f = (const double*)p;
    float* s = (float*)p;
    const int* n = (const int*)p;
    const long long token_major[3] = {4096, 64, 256}, odd_rows[3] = {4096, 64, 260}, huge[3] = {1LL << 62, 1LL << 61, 64};
    EXPECT(fa_rope(p, 0, p, 0, p, 0, p, 0, f, n, 2, 4, 2, 16, 64, 64, 1.f, 0, FA_BF16, 0), FA_OK);
    EXPECT(fa_rope(p, token_major, 0, 0, p, token_major, 0, 0, f, 0, 2, 4, 0, 16, 64, 32, 1.f, 1, FA_F32, 0), FA_OK);
    EXPECT(fa_rope(p, huge, p, huge, p, 0, p, 0, f, n, 2, 4, 2, 16, 64, 64, 1.f, 0, FA_F16, 0), FA_OK);
    EXPECT(fa_rope_bwd(p, odd_rows, p, 0, p, 0, p, 0, f, n, 2, 4, 2, 16, 64, 64, 1.f, 0, FA_BF16, 0), FA_ERR_ALIGN);
    EXPECT(fa_rope_bwd(p, 0, p, 0, p, 0, p, 0, f, n, 0x7fffffff, 0x7fffffff, 0x7fffffff, 0x7fffffff, 64, 64, 1.f, 0, FA_BF16, 0), FA_ERR_SHAPE);
    // the stride of a dimension of size 1 may be anything
    const long long one[3] = {7, -3, 64};
    EXPECT(fa_rope(p, one, 0, 0, p, one, 0, 0, f, n, 1, 1, 0, 16, 64, 64, 1.f, 0, FA_BF16, 0), FA_OK);
    double freq[32];
    float amplitude;
    for (int scaling = FA_ROPE_PLAIN; scaling <= FA_ROPE_BY_PARTS; ++scaling)
        EXPECT(fa_rope_frequencies(freq, scaling % 2 ? &amplitude : 0, 64, 10000.0, scaling, 4.0, 4096.0), FA_OK);
    EXPECT(fa_rope_frequencies(freq, 0, 63, 10000.0, 0, 1.0, 0.0), FA_ERR_SHAPE);
    EXPECT(fa_cache_write(p, 0, p, token_major, p, p, s, s, n, n, 0, 2, 2, 3, 64, 16, 9, 4, FA_F32, FA_FP8_E4M3, 0), FA_OK);
    EXPECT(fa_cache_write(p, 0, p, 0, p, p, 0, 0, n, n, n, 2, 2, 3, 64, 16, 9, 4, FA_BF16, FA_BF16, 0), FA_OK);
    EXPECT(fa_cache_write(p, 0, p, 0, p, p, 0, 0, n, n, n, 2, 2, 3, 64, 16, 9, 0x7fffffff, FA_BF16, FA_BF16, 0), FA_ERR_SHAPE);
    EXPECT(fa_cache_read(p, p, 0, 0, n, n, p, p, 2, 2, 3, 64, 16, 9, 4, FA_F16, FA_F32, 0), FA_OK);
    EXPECT(fa_cache_read(p, odd, 0, 0, n, n, p, p, 2, 2, 3, 64, 16, 9, 4, FA_F16, FA_F32, 0), FA_ERR_ALIGN);
    EXPECT(fa_fwd_cache(p, 0, p, p, s, s, n, n, 0, n, 1, p, 0, s, p, 64, 2, 4, 2, 3, 64, 16, 9, 4, 0, 0.1f, FA_BF16, FA_FP8_E4M3, 0), FA_OK);
    EXPECT(fa_fwd_cache(p, 0, p, p, 0, 0, n, n, 0, 0, 0, p, token_major, s, p, 64, 2, 4, 2, 3, 64, 16, 9, 4, 0x7fffffff, 0.1f, FA_F16, FA_F16, 0), FA_OK);
    EXPECT(fa_fwd_cache(p, 0, p, p, 0, 0, n, n, 0, 0, 0, p, 0, s, p, 63, 2, 4, 2, 3, 64, 16, 9, 4, 0, 0.1f, FA_F16, FA_F16, 0), FA_ERR_WORKSPACE);
    EXPECT(fa_fwd_cache(p, 0, p, p, 0, 0, n, n, 0, 0, 0, p, 0, s, odd, 64, 2, 4, 2, 3, 64, 16, 9, 4, 0, 0.1f, FA_F16, FA_F16, 0), FA_ERR_ALIGN);
    if (fa_fwd_cache_workspace_bytes(2, 4, 2, 3, 64, 100, FA_F16) != 64 || fa_fwd_cache_workspace_bytes(2, 4, 2, 0, 64, 100, FA_F16) != 0) ++failures;
    free(p);
    printf("cache api sanitizer run: %d failures\n", failures);
    return failures ? 1 : 0;
}
