/* abi_host_block_driver.c -- the host side of the gated recurrence, layer norm and
 * dropout without a GPU, as abi_host_driver.c does it for the other entry points:
 * workspace queries over a grid of sizes (including extents whose products overflow) and
 * calls that must be rejected before any HIP call (fake, aligned device addresses that
 * are never dereferenced).  Built by tests/test_abi_asan_block.py with AddressSanitizer
 * and UndefinedBehaviorSanitizer on the host code; any report aborts the run.
 * TEST INFRASTRUCTURE. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>

#include "memoroid.h"

#define CHECK(cond)                                                              \
    do {                                                                         \
        if (!(cond)) {                                                           \
            fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #cond);   \
            return 1;                                                            \
        }                                                                        \
    } while (0)
/* refused, or nothing to do; a launch would have been a HIP error here */
#define REFUSED(call)                  \
    do {                               \
        const int st = (call);         \
        CHECK(st != MEMOROID_EHIP);    \
        ++refused;                     \
    } while (0)

static void* P(int n) { return (void*)((uintptr_t)0x10000 * (uintptr_t)(n + 1)); }

int main(void) {
    const int64_t ext[] = {-1, 0, 1, 7, 8, 31, 32, 33, 63, 64, 65, 512, 513, 2047, 8193, 16384, 16385, 65536, (int64_t)1 << 18,
                           ((int64_t)1 << 18) + 1, (int64_t)1 << 23, ((int64_t)1 << 30) - 1, (int64_t)1 << 30,
                           ((int64_t)1 << 31) - 1, (int64_t)1 << 31, (int64_t)1 << 40, INT64_MAX / 3, INT64_MAX};
    const double ps[] = {-0.1, 0.0, 1e-300, 0x1p-33, 0.1, 1.0 - 0x1p-53, 1.0, 1.5, INFINITY, NAN};
    const int n = (int)(sizeof ext / sizeof ext[0]), np = (int)(sizeof ps / sizeof ps[0]);
    size_t sink = 0;
    long refused = 0;
    for (int i = 0; i < n; ++i)
        for (int j = 0; j < n; ++j) {
            const int64_t T = ext[i], d = ext[j];
            sink += memoroid_layer_norm_bwd_workspace_bytes(T, d);
            for (int k = 0; k < n; ++k) {
                const int64_t B = ext[k];
                for (int op = MEMOROID_OP_GATED; op <= MEMOROID_OP_LAYER_NORM_BWD; ++op)
                    sink += memoroid_workspace_bytes((memoroid_op)op, B, T, d, 64, 64, 64);
                for (int dt = -1; dt < 4; ++dt) {
                    const size_t fwd = memoroid_scan_gated_workspace_bytes(B, T, d, dt);
                    const size_t bwd = memoroid_scan_gated_bwd_workspace_bytes(B, T, d, dt);
                    CHECK((fwd == 0) == (bwd == 0));
                    sink += fwd + bwd;
                    /* no workspace, or one byte too few */
                    REFUSED(memoroid_scan_gated(P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), B, T, d, dt, NULL, 0, NULL));
                    REFUSED(memoroid_scan_gated(P(0), P(1), P(2), P(3), NULL, P(5), NULL, NULL, B, T, d, dt, P(8),
                                                fwd ? fwd - 1 : 0, NULL));
                    REFUSED(memoroid_scan_gated_bwd(P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(8), P(9), P(10), B, T, d,
                                                    dt, NULL, 0, NULL));
                    REFUSED(memoroid_scan_gated_bwd(P(0), P(1), P(2), P(3), P(4), P(5), NULL, P(7), P(8), NULL, NULL, B, T, d,
                                                    dt, P(11), bwd ? bwd - 1 : 0, NULL));
                    REFUSED(memoroid_gated_step(NULL, P(1), P(2), NULL, P(4), P(5), T, d, dt, NULL));
                }
            }
            for (int dt = -1; dt < 4; ++dt)
                for (int k = 0; k < np; ++k) {
                    const size_t ws = memoroid_layer_norm_bwd_workspace_bytes(T, d);
                    REFUSED(memoroid_dropout(P(0), P(1), P(2), NULL, ps[k], ext[i], T, d, dt, NULL));
                    REFUSED(memoroid_dropout(P(0), NULL, P(2), P(0), ps[k], 3, T, d, dt, NULL));
                    REFUSED(memoroid_layer_norm(NULL, P(1), P(2), P(3), P(4), P(5), P(6), P(7), 1e-5f, ps[k], 3, T, d, dt, NULL));
                    REFUSED(memoroid_layer_norm(P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), (float)NAN, ps[k], 3, T, d, dt,
                                                NULL));
                    REFUSED(memoroid_layer_norm_bwd(P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(8), P(9), P(10), ps[k], 3, T,
                                                    d, dt, NULL, 0, NULL));
                    REFUSED(memoroid_layer_norm_bwd(P(0), NULL, NULL, P(3), P(4), P(5), NULL, P(7), NULL, P(9), NULL, ps[k],
                                                    ext[j], T, d, dt, P(11), ws ? ws - 1 : 0, NULL));
                }
        }
    /* overlapping, missing and misaligned operands */
    CHECK(memoroid_scan_gated(P(0), P(1), P(2), P(3), P(4), P(0), NULL, NULL, 2, 100, 30, MEMOROID_F32, P(8), 1 << 30, NULL) ==
          MEMOROID_EINVAL);
    CHECK(memoroid_scan_gated(P(0), P(1), P(2), P(3), P(4), P(5), P(4), NULL, 2, 100, 30, MEMOROID_F32, P(8), 1 << 30, NULL) ==
          MEMOROID_EINVAL);
    CHECK(memoroid_scan_gated_bwd(P(0), P(1), P(2), P(3), NULL, P(5), P(6), P(7), P(8), P(9), P(10), 2, 100, 30, MEMOROID_BF16,
                                  P(11), 1 << 30, NULL) == MEMOROID_EINVAL);
    CHECK(memoroid_gated_step(P(0), P(1), P(2), P(3), P(4), P(4), 2, 30, MEMOROID_F32, NULL) == MEMOROID_EINVAL);
    CHECK(memoroid_layer_norm_bwd(P(0), P(1), P(2), P(3), P(4), P(5), P(6), P(7), P(7), P(9), P(10), 0.1, 3, 10, 30,
                                  MEMOROID_F32, P(11), 1 << 30, NULL) == MEMOROID_EINVAL);
    CHECK(memoroid_dropout(P(0), P(1), (const int64_t*)P(2), P(2), 0.5, 0, 10, 30, MEMOROID_F32, NULL) == MEMOROID_EINVAL);
    printf("validation done (%zu, %ld)\n", sink, refused);
    return 0;
}
