/* Calls every entry point of the 8-bit paged cache and of rotary positions (csrc/paged8_api.hip) with valid,
 * invalid and extreme arguments under AddressSanitizer and UndefinedBehaviorSanitizer; the launchers are
 * stubs, device pointers are fake aligned addresses. Prints "paged8 harness ok" at the end. */
#include <limits.h>
#include <math.h>
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

static int init(mustafar_pages8_t* p, int B, int H, int d, int P_, int n, int most, int type, int code, int block, int64_t ps,
                int64_t hs, int64_t ts) {
    return mustafar_paged8_init(p, P(0x100000), P(0x200000), P(0x600001), P(0x700001), P(0x300000), P(0x400000), P(0x500000), B,
                                H, d, P_, n, most, type, code, block, ps, hs, ts);
}

int main(void) {
    static const int ints[] = {INT_MIN, -1, 0, 1, 8, 16, 64, 128, 256, 1024, 4096, 1 << 19, 1 << 20, INT_MAX};
    static const int64_t strides[] = {INT64_MIN, -16, 0, 16, 128, 8192, 1 << 20, (int64_t)1 << 31, (int64_t)1 << 41, INT64_MAX};
    static const double reals[] = {-INFINITY, -1, 0, 1e-308, 0.5, 1, 8, 10000, 1e308, INFINITY, NAN};
    enum { NI = sizeof ints / sizeof *ints, NS = sizeof strides / sizeof *strides, NR = sizeof reals / sizeof *reals };
    mustafar_pages8_t p, x;
    for (int a = 0; a < NI; ++a)
        for (int b = 0; b < NI; ++b)
            for (int c = 0; c < NI; ++c) {
                (void)init(&x, ints[a], ints[b], 128, ints[c], ints[a], ints[b], 0, 2, 16, 8192, 8192, 128);
                (void)init(&x, 2, ints[a], 256, 64, ints[b], ints[c], 1, 3, ints[a], strides[a % NS], strides[b % NS], strides[c % NS]);
                (void)init(&x, 2, 2, 64, 64, 4, 4, ints[a], ints[b], ints[c], 8192, 4096, 64);
            }
    EXPECT(init(&p, 3, 8, 128, 64, 100, 40, MUSTAFAR_BF16, MUSTAFAR_INT8, 32, 8 * 64 * 128, 64 * 128, 128), MUSTAFAR_OK);
    for (int a = 0; a < NI; ++a) {
        const int n = ints[a];
        /* the largest would be more workgroups than a launch has */
        EXPECT(mustafar_paged8_write(&p, P(0x10), 1024, P(0x20), 1024, P(0x30), n, 0), n < 0 || n == INT_MAX ? MUSTAFAR_EINVAL : MUSTAFAR_OK);
        EXPECT(mustafar_paged8_gather(&p, 0, P(0x10), P(0x20), n, 0), n < 0 || n == INT_MAX ? MUSTAFAR_EINVAL : MUSTAFAR_OK);
        for (int b = 0; b < NI; ++b)
            for (int c = 0; c < NI; ++c) {
                mustafar_rotation_t r = {(const double*)P(0x8), ints[b], ints[c] & 3, 1.f};
                double rates[MUSTAFAR_ROPE_MAX_D / 2];
                (void)mustafar_paged8_attn_workspace_bytes(&p, 32, n, ints[b], ints[c], 0);
                (void)mustafar_paged8_attn_workspace_bytes(&p, n, ints[b], ints[c], INT_MAX, ints[b]);
                (void)mustafar_paged8_attn(P(0x10), 4096, n, 32, &p, P(0x20), ints[b], ints[c], -1.f, P(0x30), 4096, ints[b], ints[c],
                                           ints[b], P(0x40), SIZE_MAX, 0);
                (void)mustafar_paged8_attn(P(0x10), strides[a % NS], ints[b], ints[c], &p, P(0x20), 0, 0, 1.f, P(0x30),
                                           strides[b % NS], 1, 1, 0, P(0x40), 1 << 20, 0);
                (void)mustafar_rope(&r, P(0x10), strides[a % NS], n, P(0x20), strides[b % NS], ints[c], ints[b], ints[c], n & 1,
                                    P(0x30), 0, 0, 1, P(0x40), strides[a % NS], P(0x50), strides[b % NS], 0);
                (void)mustafar_rope(&r, P(0x10), (int64_t)1 << 31, n, 0, 0, 0, 128, ints[c], 0, 0, &p.pages, P(0x60), 0, P(0x10),
                                    (int64_t)1 << 31, 0, 0, 0);
                (void)mustafar_rope_rates(rates, n, reals[b % NR], c % 6 - 1, reals[c % NR], reals[a % NR], reals[b % NR], reals[(a + c) % NR]);
            }
    }
    for (int rot = 2; rot <= MUSTAFAR_ROPE_MAX_D; rot += 2) {
        double rates[MUSTAFAR_ROPE_MAX_D / 2];
        EXPECT(mustafar_rope_rates(rates, rot, 10000, MUSTAFAR_ROPE_TURNS, 8, 8192, 1, 32), MUSTAFAR_OK);
        EXPECT(mustafar_rope_rates(rates, rot, 10000, MUSTAFAR_ROPE_BASE, 8, 0, 0, 0), rot == 2 ? MUSTAFAR_EINVAL : MUSTAFAR_OK);
    }
    if (mf_stub_launches < 100) ++failures;
    if (failures) return 1;
    printf("paged8 harness ok\n");
    return 0;
}
