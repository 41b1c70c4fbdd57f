// Drives the host side of linear attention, projections and embeddings (argument checks,
// overlap of strided heads, sizes, plans, launches) in a host-only build with
// AddressSanitizer and UndefinedBehaviorSanitizer.  The HIP entry points below stand in
// for the runtime's: an accepted call launches nothing, its grids are checked.  Test
// infrastructure: built and run by tests/test_rows_sanitizers_cpu.py.
#include <hip/hip_runtime_api.h>
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "finc.h"

static int failures = 0;
static long long launches = 0;
#define EXPECT(cond)                                                        \
    do {                                                                    \
        if (!(cond)) {                                                      \
            fprintf(stderr, "%s:%d: expected %s\n", __FILE__, __LINE__, #cond); \
            ++failures;                                                     \
        }                                                                   \
    } while (0)

static struct {
    dim3 grid, block;
    size_t lds;
    hipStream_t stream;
} pushed;
extern "C" {
hipError_t __hipPushCallConfiguration(dim3 g, dim3 b, size_t lds, hipStream_t st) {
    pushed = {g, b, lds, st};
    return hipSuccess;
}
hipError_t __hipPopCallConfiguration(dim3 *g, dim3 *b, size_t *lds, hipStream_t *st) {
    *g = pushed.grid;
    *b = pushed.block;
    *lds = pushed.lds;
    *st = pushed.stream;
    return hipSuccess;
}
hipError_t hipLaunchKernel(const void *, dim3 g, dim3 b, void **, size_t, hipStream_t) {
    ++launches;
    // fewer than 2^32 threads in x and 2^16 workgroups in y, and no empty grid
    EXPECT((unsigned long long)g.x * b.x < 1ull << 32 && g.y < 1u << 16 && g.z == 1);
    EXPECT(g.x > 0 && g.y > 0 && b.x > 0 && b.x <= 1024);
    return hipSuccess;
}
hipError_t hipGetLastError(void) { return hipSuccess; }
}

// Addresses that are never dereferenced, and one that no element starts at.
static void *at(int i) { return (void *)((uintptr_t)(i + 1) << 52); }
static float *f32(int i) { return (float *)at(i); }
static float *odd() { return (float *)((char *)at(60) + 1); }

static const int kBig[] = {-2147483647 - 1, -1, 0, 1, 2, 64, 513, 4096, 1 << 24, 1 << 30,
                           2147483647};
static const long long kSteps[] = {INT64_MIN, -1, 0, 1, 1ll << 40, 1ll << 57, 1ll << 61, INT64_MAX};

static void sizes() {
    for (int B : kBig)
        for (int L : kBig)
            for (int H : {-1, 0, 1, 3, 2147483647})
                for (int D : {-1, 0, 1, 100, 128, 129}) {
                    EXPECT(finc_linear_attention_states_bytes(B, L, H, D, 128) % 256 == 0);
                    for (int G : {-1, 0, 1, 3, 2147483647})
                        EXPECT(finc_linear_attention_workspace_bytes(B, L, H, G, D, 128) % 256 == 0);
                }
    for (int M : kBig)
        for (int K : kBig)
            for (int N : kBig) {
                for (int type : {-1, 0, 1, 2, 3}) {
                    EXPECT(finc_linear_workspace_bytes(type, M, K, N) % 256 == 0);
                    for (int act : {-1, 0, 2, 4})
                        EXPECT(finc_linear_grad_workspace_bytes(type, act, M, K, N) % 256 == 0);
                }
                EXPECT(finc_embed_workspace_bytes(M, K, N) % 256 == 0);
            }
}

// Every size and step with one thing wrong: no step of the arithmetic overflows.
static void attention_refusals() {
    for (int B : kBig)
        for (int L : kBig)
            for (int H : {-1, 0, 1, 6, 1 << 24, 2147483647})
                for (long long sb : kSteps)
                    for (long long st : kSteps)
                        for (long long sh : kSteps) {
                            finc_attention_args a;
                            memset(&a, 0, sizeof a);
                            a.type = FINC_BF16;
                            a.B = B;
                            a.L = L;
                            a.H = H;
                            a.G = H == 6 ? 3 : 1;
                            a.DK = 128;
                            a.DV = 64;
                            a.q = a.k = a.v = a.g = {at(0), sb, st, sh};
                            a.y = {at(1), sb, st, sh};
                            a.states = f32(2);
                            a.decay = odd();
                            a.scale = 1.0;
                            EXPECT(finc_linear_attention_forward(&a, nullptr) == FINC_EINVAL);
                            finc_attention_grads g;
                            memset(&g, 0, sizeof g);
                            g.dy = a.q;
                            g.dq = {at(3), sb, st, sh};
                            g.dk = {at(4), sb, st, sh};
                            g.dv = {at(5), sb, st, sh};
                            g.dg = {at(6), sb, st, sh};
                            g.workspace = at(7);
                            EXPECT(finc_linear_attention_backward(&a, &g, nullptr) == FINC_EINVAL);
                            finc_attention_step_args s;
                            memset(&s, 0, sizeof s);
                            s.B = B;
                            s.S = L;
                            s.H = H;
                            s.G = 1;
                            s.DK = s.DV = 128;
                            s.q = s.k = s.v = s.g = a.q;
                            s.y = a.y;
                            s.state = f32(2);
                            s.slots = (int *)at(3);
                            s.decay = odd();
                            EXPECT(finc_linear_attention_step(&s, nullptr) == FINC_EINVAL);
                        }
}

static void row_refusals() {
    for (int M : kBig)
        for (int K : kBig)
            for (int N : kBig)
                for (long long st : kSteps) {
                    finc_linear_args a;
                    memset(&a, 0, sizeof a);
                    a.type = FINC_F16;
                    a.act = FINC_ACT_SILU;
                    a.M = M;
                    a.K = K;
                    a.N = N;
                    a.x = at(0);
                    a.w = at(1);
                    a.residual = at(2);
                    a.y = at(3);
                    a.pre = at(4);
                    a.sx = a.sw = a.sres = a.sy = a.spre = st;
                    a.bias = odd();
                    a.workspace = at(6);
                    EXPECT(finc_linear_forward(&a, nullptr) == FINC_EINVAL);
                    finc_linear_grad_args g;
                    memset(&g, 0, sizeof g);
                    g.type = FINC_BF16;
                    g.act = FINC_ACT_GELU;
                    g.M = M;
                    g.K = K;
                    g.N = N;
                    g.dy = at(0);
                    g.x = at(1);
                    g.w = at(2);
                    g.pre = at(3);
                    g.dx = at(4);
                    g.dw = at(5);
                    g.sdy = g.sx = g.sw = g.spre = g.sdx = g.sdw = st;
                    g.dbias = odd();
                    g.workspace = at(7);
                    EXPECT(finc_linear_backward(&g, nullptr) == FINC_EINVAL);
                    EXPECT(finc_embed_forward(FINC_BF16, FINC_F32, (char *)at(0) + 1, 1, at(1), st,
                                              at(2), st, M, K, N, 1.0, nullptr) == FINC_EINVAL ||
                           M == 0);
                    EXPECT(finc_embed_backward(FINC_F32, at(0), 0, at(1), st, odd(), M, K, N, 1.0,
                                               at(3), nullptr) == FINC_EINVAL ||
                           K == 0);
                }
}

// y in rows of one buffer beside v: refused where they share an element.
static void overlaps() {
    const int B = 2, L = 3, H = 2, D = 4, row = 2 * H * D;
    for (int off = 0; off < B * L * row + row; ++off) {
        finc_attention_args a;
        memset(&a, 0, sizeof a);
        a.B = B;
        a.L = L;
        a.H = H;
        a.G = 1;
        a.DK = D;
        a.DV = D;
        a.q = {at(0), L * D, D, D};
        a.k = {at(1), L * D, D, D};
        a.v = {at(2), (long long)L * row, row, D};
        a.y = {f32(2) + off, (long long)L * row, row, D};
        const int r = finc_linear_attention_forward(&a, nullptr);
        const bool beside = off % row == H * D || off >= (B * L - 1) * row + H * D;
        EXPECT(r == (beside ? FINC_OK : FINC_EINVAL));
        // and heads that lie in turns with another tensor's: as all that they span
        a.v.sh = a.y.sh = 2 * D;
        EXPECT(off >= (B * L - 1) * row + 3 * D || finc_linear_attention_forward(&a, nullptr) == FINC_EINVAL);
    }
}

// Sizes up to the documented limits, all the way to the launches.
static void attention_launches() {
    const int shapes[][5] = {{1, 0, 1, 1, 1}, {1, 1, 1, 1, 1}, {3, 512, 4, 2, 128}, {2, 513, 4, 1, 100},
                             {1, 2049, 2, 2, 64}, {(1 << 24) - 1, 1, 1, 1, 1}, {1, 1, (1 << 24) - 1, 1, 1},
                             {4, 1 << 30, 1, 1, 128}, {1, 2147483647, 1, 1, 128}, {64, 65536, 16, 4, 128},
                             {1 << 20, 513, 1, 1, 8}, {(1 << 24) - 1, 513, 1, 1, 1}};
    for (auto &s : shapes)
        for (int type : {FINC_F32, FINC_BF16, FINC_F16}) {
            const long long B = s[0], L = s[1], H = s[2], G = s[3], D = s[4];
            finc_attention_args a;
            memset(&a, 0, sizeof a);
            a.type = type;
            a.B = s[0];
            a.L = s[1];
            a.H = s[2];
            a.G = s[3];
            a.DK = a.DV = s[4];
            a.q = {at(0), L * G * D, G * D, D};
            a.k = {at(1), L * G * D, G * D, D};
            a.v = {at(2), L * H * D, H * D, D};
            a.g = {at(3), L * H, H, 1};
            a.y = {at(4), L * H * D, H * D, D};
            a.state = f32(5);
            a.state_out = f32(6);
            a.states = f32(7);
            a.decay = f32(8);
            a.lengths = (int *)at(9);
            EXPECT(finc_linear_attention_forward(&a, nullptr) == FINC_OK);
            for (int with = 0; with < 4; ++with) {   // dg and dstate, or not
                finc_attention_grads g;
                memset(&g, 0, sizeof g);
                g.dy = {at(10), L * H * D, H * D, D};
                g.dq = {at(11), L * G * D, G * D, D};
                g.dk = {at(12), L * G * D, G * D, D};
                g.dv = {at(13), L * H * D, H * D, D};
                if (with & 1)
                    g.dg = {at(14), L * H, H, 1};
                g.dstate_out = f32(15);
                g.dstate = with & 2 ? f32(16) : nullptr;
                g.workspace = at(17);
                EXPECT(finc_linear_attention_backward(&a, &g, nullptr) == FINC_OK);
            }
            finc_attention_step_args p;
            memset(&p, 0, sizeof p);
            p.type = type;
            p.B = p.S = s[0];
            p.H = s[2];
            p.G = s[3];
            p.DK = p.DV = s[4];
            p.q = {at(0), G * D, 0, D};
            p.k = {at(1), G * D, 0, D};
            p.v = {at(2), H * D, 0, D};
            p.y = {at(4), H * D, 0, D};
            p.state = f32(5);
            EXPECT(finc_linear_attention_step(&p, nullptr) == FINC_OK);
        }
}

static void row_launches() {
    const int sizes[] = {0, 1, 7, 8, 64, 129, 2048, 100003, (1 << 30) - 1};
    const long long most = 1ll << 40;
    for (long long M : sizes)
        for (long long K : sizes)
            for (long long N : sizes) {
                if (K == 0 || N == 0 || M * K >= most || M * N >= most || K * N >= most)
                    continue;
                for (int type : {FINC_F32, FINC_BF16})
                    for (int off : {0, 1})   // another address than a multiple of 16 bytes
                        for (int act : {FINC_ACT_NONE, FINC_ACT_GELU}) {
                            const int sz = type == FINC_F32 ? 4 : 2;
                            finc_linear_args a;
                            memset(&a, 0, sizeof a);
                            a.type = type;
                            a.act = act;
                            a.M = (int)M;
                            a.K = (int)K;
                            a.N = (int)N;
                            a.x = (char *)at(0) + off * sz;
                            a.w = at(1);
                            a.residual = a.y = at(2);
                            a.pre = at(3);
                            a.sx = a.sw = K;
                            a.sres = a.sy = a.spre = N;
                            a.bias = f32(4);
                            a.workspace = finc_linear_workspace_bytes(type, a.M, a.K, a.N) ? at(5) : nullptr;
                            EXPECT(finc_linear_forward(&a, nullptr) == FINC_OK);
                            finc_linear_grad_args g;
                            memset(&g, 0, sizeof g);
                            g.type = type;
                            g.act = act;
                            g.M = a.M;
                            g.K = a.K;
                            g.N = a.N;
                            g.dy = at(0);
                            g.x = (char *)at(1) + off * sz;
                            g.w = at(2);
                            g.pre = at(3);
                            g.sdy = g.spre = N;
                            g.sx = g.sw = g.sdx = g.sdw = K;
                            g.workspace = at(7);
                            for (int with = 0; with < 8; ++with) {
                                g.dx = with & 1 ? at(4) : nullptr;
                                g.dw = with & 2 ? at(5) : nullptr;
                                g.dbias = with & 4 ? f32(6) : nullptr;
                                EXPECT(finc_linear_backward(&g, nullptr) == FINC_OK);
                            }
                        }
            }
    for (long long M : sizes)
        for (long long V : sizes)
            for (long long D : sizes) {
                const long long vecs = (D + 7) / 8;
                if (D == 0 || M * vecs >= 1ll << 31 || V * vecs >= 1ll << 37)
                    continue;
                EXPECT(finc_embed_forward(FINC_BF16, FINC_F32, at(0), 1, at(1), D, at(2), D, (int)M,
                                          (int)V, (int)D, 1.0, nullptr) == FINC_OK);
                EXPECT(finc_embed_backward(FINC_BF16, at(0), 0, at(1), D, f32(2), (int)M, (int)V,
                                           (int)D, 1.0, at(3), nullptr) == FINC_OK);
            }
}

int main() {
    sizes();
    attention_refusals();
    row_refusals();
    EXPECT(launches == 0);
    overlaps();
    attention_launches();
    row_launches();
    EXPECT(launches > 0);
    if (failures)
        fprintf(stderr, "%d checks failed\n", failures);
    else
        printf("rows drive: all checks held\n");
    return failures ? 1 : 0;
}
