/* The largest launches of the paged cache's entry points (csrc/paged_api.hip): a launch has less than
 * 2^32 threads, and a call that would need more in any of its kernels is refused before the first.
 * The launchers are stubs, device pointers are fake aligned addresses. Prints "paged limits ok". */
#include <limits.h>
#include <stdint.h>
#include <stdio.h>

#include "mustafar.h"

extern long mf_stub_launches;
static int failures = 0;

static void expect(const char* what, int got, int want) {
    static long before = 0;
    if (got != want || mf_stub_launches != before + (want == MUSTAFAR_OK)) {
        fprintf(stderr, "%s -> %d, expected %d; %ld launches\n", what, got, want, mf_stub_launches - before);
        ++failures;
    }
    before = mf_stub_launches;
}

static void* P(uintptr_t a) { return (void*)a; }

static mustafar_pages_t pages(int B, int H, int d) {
    mustafar_pages_t p;
    if (mustafar_paged_init(&p, P(0x100000), P(0x200000), P(0x300000), P(0x400000), P(0x500000), B, H, d, 64, 100, 40, 0,
                            (int64_t)H * 64 * d, 64 * d, d) != MUSTAFAR_OK)
        ++failures;
    return p;
}

static int attn(const mustafar_pages_t* p, int n_q, int Hq, int max_q, int n_splits) {
    const int64_t row = (int64_t)Hq * p->d;
    return mustafar_paged_attn(P(0x10), row, n_q, Hq, p, P(0x20), 0, 0, 0.f, P(0x30), row, max_q, 4096, n_splits, P(0x40),
                               SIZE_MAX, 0);
}

int main(void) {
    mustafar_pages_t p = pages(64, 8, 128);
    /* chunks beside single tokens: 67 tiles of 256 rows * 8 heads * ranges * 512 threads */
    expect("chunks", attn(&p, 200, 32, 100, 15650), MUSTAFAR_OK);
    expect("chunks, one range more", attn(&p, 200, 32, 100, 15651), MUSTAFAR_EINVAL);
    expect("chunks, the most ranges", attn(&p, 200, 32, 100, 1 << 16), MUSTAFAR_EINVAL);
    /* single tokens: 4352 tiles of 16 rows * 32 heads * ranges * 64 threads */
    p = pages(4096, 32, 128);
    expect("single tokens", attn(&p, 4096, 32, 1, 481), MUSTAFAR_OK);
    expect("single tokens, one range more", attn(&p, 4096, 32, 1, 482), MUSTAFAR_EINVAL);
    /* joining them: 64 threads a row at d = 256 */
    p = pages(3, 8, 256);
    expect("rows", attn(&p, (1 << 21) - 1, 32, 1 << 21, 2), MUSTAFAR_OK);
    expect("rows, one more", attn(&p, 1 << 21, 32, 1 << 21, 2), MUSTAFAR_EINVAL);
    expect("rows of one range", attn(&p, 1 << 21, 32, 1 << 21, 1), MUSTAFAR_OK);
    /* gather: 24 entries and heads * 16 threads a token */
    p = pages(3, 8, 128);
    expect("gather", mustafar_paged_gather(&p, 0, P(0x10), P(0x20), 11184800, 0), MUSTAFAR_OK);
    expect("gather, one more", mustafar_paged_gather(&p, 0, P(0x10), P(0x20), 11184801, 0), MUSTAFAR_EINVAL);
    /* a write takes several launches */
    expect("write", mustafar_paged_write(&p, P(0x10), 1024, P(0x20), 1024, P(0x30), INT_MAX, 0), MUSTAFAR_OK);
    if (failures) return 1;
    printf("paged limits ok\n");
    return 0;
}
