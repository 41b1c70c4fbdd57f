// Drives the host side of the sequence operators (argument checks, overlap of
// strided regions, sizes) in a host-only build with AddressSanitizer and
// UndefinedBehaviorSanitizer: every call is host arithmetic or is rejected before
// any HIP call.  Test infrastructure: built and run by
// tests/test_sequence_sanitizers_cpu.py.
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "finc.h"

static int failures = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) {                                                      \
            fprintf(stderr, "%s:%d: expected %s\n", __FILE__, __LINE__, #cond); \
            ++failures;                                                     \
        }                                                                   \
    } while (0)

// Addresses that are never dereferenced.
static void *at(int i) { return (void *)(uintptr_t)(0x10000000ull * (i + 1)); }
static finc_raster raster(int i, long long sb, long long sd) { return {at(i), sb, sd}; }

static const int kBig[] = {-2147483647 - 1, -1, 0, 1, 2, 63, 64, 65, 4096, 1 << 29, 1 << 30,
                           2147483647};

static void sizes() {
    for (int B : kBig)
        for (int D : kBig)
            for (int L : kBig) {
                for (int N : {-1, 0, 1, 16, 64, 65, 2147483647}) {
                    const size_t s = finc_selective_scan_states_bytes(B, D, L, N);
                    EXPECT(s % 256 == 0);
                    for (int G : {-1, 0, 1, 2, 2147483647}) {
                        const size_t w = finc_selective_scan_workspace_bytes(B, D, L, N, G);
                        EXPECT(w % 256 == 0);
                    }
                }
                for (int K : {0, 1, 8, 9})
                    EXPECT(finc_causal_conv_workspace_bytes(B, D, L, K) % 256 == 0);
            }
    for (int M : kBig)
        for (int D : kBig) {
            EXPECT(finc_add_norm_workspace_bytes(M, D) % 256 == 0);
            finc_dropout_counters(M, D);
        }
}

// Every size and step, with one thing wrong: no step of the arithmetic overflows.
static void refusals() {
    const long long steps[] = {INT64_MIN, -1, 0, 1, 1ll << 40, 1ll << 61, INT64_MAX};
    for (int B : kBig)
        for (int D : kBig)
            for (int L : kBig)
                for (long long sb : steps)
                    for (long long sd : steps) {
                        finc_conv_args c;
                        memset(&c, 0, sizeof c);
                        c.type = 9;   // no such type
                        c.B = B;
                        c.D = D;
                        c.L = L;
                        c.K = 4;
                        c.x = c.y = raster(0, sb, sd);
                        EXPECT(finc_causal_conv_forward(&c, nullptr) == FINC_EINVAL);
                        c.type = FINC_BF16;
                        c.w = (const float *)((char *)at(2) + 1);   // not aligned
                        EXPECT(finc_causal_conv_forward(&c, nullptr) == FINC_EINVAL);
                        finc_scan_args s;
                        memset(&s, 0, sizeof s);
                        s.B = B;
                        s.D = D;
                        s.L = L;
                        s.N = 16;
                        s.G = 1;
                        s.x = s.dt = s.Bm = s.Cm = raster(0, sb, sd);
                        s.y = raster(1, sb, sd);
                        s.A = (const float *)((char *)at(2) + 1);
                        EXPECT(finc_selective_scan_forward(&s, nullptr) == FINC_EINVAL);
                        finc_scan_grads g;
                        memset(&g, 0, sizeof g);
                        g.dA = (float *)at(4);
                        g.workspace = (char *)at(5) + 8;
                        EXPECT(finc_selective_scan_backward(&s, &g, nullptr) == FINC_EINVAL);
                    }
    for (int M : kBig)
        for (int D : kBig)
            for (long long st : steps) {
                EXPECT(finc_dropout(FINC_F32, at(0), st, nullptr, 0, at(1), st, M, D, 1.5, 0, 0,
                                    nullptr) == FINC_EINVAL);
                finc_norm_args n;
                memset(&n, 0, sizeof n);
                n.M = M;
                n.D = D;
                n.x = at(0);
                n.y = at(1);
                n.sx = n.sy = n.sr = n.sres = st;
                n.w = (const float *)((char *)at(2) + 1);
                const int r = finc_add_norm_forward(&n, nullptr);
                EXPECT(r == FINC_EINVAL || r == FINC_EUNSUPPORTED);
            }
}

// Regions that share memory, by every route the check takes.
static void overlaps() {
    const int B = 3, D = 4, L = 8;
    for (int off = 0; off < 2 * D * L; ++off) {
        // x and y in rows of one buffer of 2 D L elements a batch row: refused unless y's
        // block lies beside x's
        finc_conv_args c;
        memset(&c, 0, sizeof c);
        c.type = FINC_F32;
        c.B = B;
        c.D = D;
        c.L = L;
        c.K = 2;
        c.x = raster(0, 2 * D * L, L);
        c.y = raster(0, 2 * D * L, L);
        c.y.p = (float *)c.y.p + off;
        c.w = (const float *)at(3);
        if (off != D * L)
            EXPECT(finc_causal_conv_forward(&c, nullptr) == FINC_EINVAL);
    }
}

int main() {
    sizes();
    refusals();
    overlaps();
    if (failures)
        fprintf(stderr, "%d checks failed\n", failures);
    else
        printf("sequence drive: all checks held\n");
    return failures ? 1 : 0;
}
