// Drives the entry points of csrc/fa_pages_api.hip through accepted and refused calls under host sanitizers, with stand-ins for
// the launchers; built by tests/test_pages_host.py, which checks the exit status and the line printed at the end.
#include <stdio.h>
#include <stdlib.h>

#include "../../paper_2407_08608_amd/csrc/fa_launch.h"

namespace fa {
int launch_rope_axes(const Rows&, const Rows&, const Rows&, const Rows&, const double*, const int*, const int*, int, int, int, int, int, int,
                     int, float, int, bool, int, hipStream_t) { return FA_OK; }
size_t cache_pages_workspace_bytes(int, int) { return 64; }
int launch_cache_fork(const int*, const int*, const int*, const int*, int*, int*, int*, int*, int*, void*, int, int, int, int, int,
                      hipStream_t) { return FA_OK; }
int launch_cache_extend(int*, const int*, const int*, const int*, int*, void*, int, int, int, int, int, hipStream_t) { return FA_OK; }
int launch_cache_compact(const int*, const int*, int*, int*, int*, int*, void*, int, int, int, int, hipStream_t) { return FA_OK; }
int launch_cache_copy(const Cache&, const int*, const int*, int, int, hipStream_t) { return FA_OK; }
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
    void *p = aligned_alloc(256, 4096), *other = aligned_alloc(256, 4096);
    int *n = (int*)p, *m = (int*)other, *odd = (int*)((char*)p + 2);
    const double* f = (const double*)p;
    const long long token_major[3] = {4096, 64, 256}, huge[3] = {1LL << 62, 1LL << 61, 64};
    EXPECT(fa_rope_axes(p, 0, p, 0, p, 0, p, 0, f, n, n, 3, 2, 4, 2, 16, 64, 64, 1.f, 0, FA_BF16, 0), FA_OK);
    EXPECT(fa_rope_axes_bwd(p, token_major, 0, 0, p, token_major, 0, 0, f, n, n, 0x7fffffff, 2, 4, 0, 16, 64, 32, 1.f, 1, FA_F32, 0), FA_OK);
    EXPECT(fa_rope_axes(p, huge, p, huge, p, 0, p, 0, f, n, n, 1, 2, 4, 2, 16, 64, 64, 1.f, 0, FA_F16, 0), FA_OK);
    EXPECT(fa_rope_axes(p, 0, p, 0, p, 0, p, 0, f, n, n, 0, 2, 4, 2, 16, 64, 64, 1.f, 0, FA_BF16, 0), FA_ERR_SHAPE);
    EXPECT(fa_rope_axes_bwd(p, 0, p, 0, p, 0, p, 0, f, odd, n, 3, 2, 4, 2, 16, 64, 64, 1.f, 0, FA_BF16, 0), FA_ERR_ALIGN);
    EXPECT(fa_rope_axes_bwd(p, 0, p, 0, p, 0, p, 0, f, n, 0, 3, 2, 4, 2, 16, 64, 64, 1.f, 0, FA_BF16, 0), FA_ERR_NULL);
    EXPECT(fa_cache_fork(n, n, n, 0, m, m, n, n, n, p, 64, 3, 4, 16, 9, 5, 0), FA_OK);
    EXPECT(fa_cache_fork(n, n, n, n, m, m, n, n, n, p, 63, 3, 4, 16, 9, 5, 0), FA_ERR_WORKSPACE);
    EXPECT(fa_cache_fork(n, n, n, n, n, m, n, n, n, p, 64, 3, 4, 16, 9, 5, 0), FA_ERR_SHAPE);
    EXPECT(fa_cache_fork(n, n, n, n, m, n, n, n, n, p, 64, 3, 4, 16, 9, 5, 0), FA_ERR_SHAPE);
    EXPECT(fa_cache_fork(n, n, n, n, m, m, n, n, n, p, 64, 1, 0x7fffffff, 1, 0x7fffffff, 1, 0), FA_OK);
    EXPECT(fa_cache_fork(n, n, n, n, m, m, n, n, n, p, 64, 1, 0x7fffffff, 1, 0x7fffffff, 2, 0), FA_ERR_SHAPE);
    EXPECT(fa_cache_fork(n, n, n, n, m, m, n, n, n, p, 64, 1, 1, 0x7fffffff, 9, 0x7fffffff, 0), FA_ERR_SHAPE);
    EXPECT(fa_cache_extend(n, n, 0, 0, n, p, 64, 3, 0x7fffffff / 3, 16, 9, 5, 0), FA_OK);
    EXPECT(fa_cache_extend(n, n, n, odd, n, p, 64, 3, 1, 16, 9, 5, 0), FA_ERR_ALIGN);
    EXPECT(fa_cache_extend(n, n, n, n, n, odd, 64, 3, 1, 16, 9, 5, 0), FA_ERR_ALIGN);
    EXPECT(fa_cache_compact(n, 0, n, n, n, n, p, 64, 3, 0x7fffffff, 9, 5, 0), FA_OK);
    EXPECT(fa_cache_compact(n, 0, n, n, n, 0, p, 64, 3, 1, 9, 5, 0), FA_ERR_NULL);
    EXPECT(fa_cache_copy(p, p, 0, 0, n, n, 0x7fffffff, 2, 64, 16, 9, FA_BF16, 0), FA_OK);
    EXPECT(fa_cache_copy(p, p, p, p, n, n, 3, 2, 256, 16, 9, FA_FP4_E2M1, 0), FA_OK);
    EXPECT(fa_cache_copy(p, p, p, 0, n, n, 3, 2, 256, 16, 9, FA_FP4_E2M1, 0), FA_ERR_NULL);
    EXPECT(fa_cache_copy(p, p, p, p, n, n, 3, 2, 256, 16, 9, FA_F16, 0), FA_ERR_DTYPE);
    EXPECT(fa_cache_copy(p, odd, 0, 0, n, n, 3, 2, 256, 16, 9, FA_F16, 0), FA_ERR_ALIGN);
    if (fa_cache_pages_workspace_bytes(1, 1) != 64 || fa_cache_pages_workspace_bytes(0, 1) != 0) ++failures;
    free(p);
    free(other);
    printf("pages api sanitizer run: %d failures\n", failures);
    return failures != 0;
}
