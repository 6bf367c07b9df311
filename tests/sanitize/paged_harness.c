/* Calls every entry point of the paged cache (csrc/paged_api.hip) with valid, invalid and
 * extreme arguments under AddressSanitizer and UndefinedBehaviorSanitizer; the launchers are
 * stubs, device pointers are fake aligned addresses. Prints "paged harness ok" at the end. */
#include <limits.h>
#include <stdint.h>
#include <stdio.h>

#include "mustafar.h"

extern long mf_stub_launches;
static int failures = 0;

#define EXPECT(call, want)                                                                       \
    do {                                                                                         \
        const int got_ = (call);                                                                 \
        if (got_ != (want)) {                                                                    \
            fprintf(stderr, "%s:%d: %s -> %d, expected %d\n", __FILE__, __LINE__, #call, got_,   \
                    (int)(want));                                                                \
            ++failures;                                                                          \
        }                                                                                        \
    } while (0)

static void* P(uintptr_t a) { return (void*)a; }

int main(void) {
    static const int ints[] = {INT_MIN, -1, 0, 1, 8, 16, 64, 128, 256, 1024, 4096, 1 << 19, 1 << 20, INT_MAX};
    static const int64_t strides[] = {INT64_MIN, -8, 0, 8, 128, 8192, 1 << 20, (int64_t)1 << 31, (int64_t)1 << 41, INT64_MAX};
    enum { NI = sizeof ints / sizeof *ints, NS = sizeof strides / sizeof *strides };
    mustafar_pages_t p, x;
    for (int a = 0; a < NI; ++a)
        for (int b = 0; b < NI; ++b)
            for (int c = 0; c < NI; ++c) {
                (void)mustafar_paged_init(&x, P(0x100000), P(0x200000), P(0x300000), P(0x400000), P(0x500000), ints[a],
                                          ints[b], 128, ints[c], ints[a], ints[b], 0, 8192, 8192, 128);
                (void)mustafar_paged_init(&x, P(0x100000), P(0x200000), P(0x300000), P(0x400000), P(0x500000), 2, ints[a],
                                          256, 64, ints[b], ints[c], 1, strides[a % NS], strides[b % NS], strides[c % NS]);
            }
    EXPECT(mustafar_paged_init(&p, P(0x100000), P(0x200000), P(0x300000), P(0x400000), P(0x500000), 3, 8, 128, 64, 100, 40,
                               MUSTAFAR_BF16, 8 * 64 * 128, 64 * 128, 128), MUSTAFAR_OK);
    for (int a = 0; a < NI; ++a) {
        const int n = ints[a];
        EXPECT(mustafar_paged_plan(&p, 0, P(0x10), P(0x400000), P(0x20), P(0x30), n, P(0x40), 0),
               n < 0 || n > MUSTAFAR_PAGED_MAX_STEP ? MUSTAFAR_EINVAL : MUSTAFAR_OK);
        EXPECT(mustafar_paged_write(&p, P(0x10), 1024, P(0x20), 1024, P(0x30), n, 0), n < 0 ? MUSTAFAR_EINVAL : MUSTAFAR_OK);
        /* the largest would be more workgroups than a launch has */
        EXPECT(mustafar_paged_gather(&p, 0, P(0x10), P(0x20), n, 0), n < 0 || n == INT_MAX ? MUSTAFAR_EINVAL : MUSTAFAR_OK);
        for (int b = 0; b < NI; ++b)
            for (int c = 0; c < NI; ++c) {
                (void)mustafar_paged_attn_workspace_bytes(&p, 32, n, ints[b], ints[c], 0);
                (void)mustafar_paged_attn_workspace_bytes(&p, n, ints[b], ints[c], INT_MAX, ints[b]);
                (void)mustafar_paged_attn(P(0x10), 4096, n, 32, &p, P(0x20), ints[b], ints[c], -1.f, P(0x30), 4096,
                                          ints[b], ints[c], ints[b], P(0x40), SIZE_MAX, 0);
                (void)mustafar_paged_attn(P(0x10), strides[a % NS], ints[b], ints[c], &p, P(0x20), 0, 0, 1.f, P(0x30),
                                          strides[b % NS], 1, 1, 0, P(0x40), 1 << 20, 0);
            }
    }
    if (mf_stub_launches < 100) ++failures;
    if (failures) return 1;
    printf("paged harness ok\n");
    return 0;
}
