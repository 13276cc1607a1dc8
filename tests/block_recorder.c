/* The launches of the block operators' calls (layer with an epilogue, routing,
 * experts, combination), recorded on the CPU as launch_recorder.c does: this
 * program's own definitions of the HIP calls that launch kernels take the
 * runtime's place, so that nothing reaches a device, and a launch of 2^32
 * threads or more in one dimension is refused.  Pointers are fake and never
 * dereferenced.
 *
 * Each line on stdin is a call; for each, one line on stdout: its status and
 * "gx,gy,gz,bx" of every launch that was accepted.  A call whose workspace is
 * given one byte too small must be refused first.
 *   epilogue T K N rank n_mod dt lr_dt bits act
 *   route    T n_experts top_k dt modality
 *   experts  T n_slots n_experts K N rank n_mod dt bits act gathered
 *   combine  T n_slots N top_k dt */
#include <stdint.h>
#include <stdio.h>
#include <string.h>

#include "masq.h"

typedef struct { uint32_t x, y, z; } dim3;
static struct { dim3 grid, block; size_t shared; void* stream; } pushed;
static char launches[1 << 16];
static int last_error = 0;

int __hipPushCallConfiguration(dim3 grid, dim3 block, size_t shared, void* stream) {
    pushed.grid = grid;
    pushed.block = block;
    pushed.shared = shared;
    pushed.stream = stream;
    return 0;
}
int __hipPopCallConfiguration(dim3* grid, dim3* block, size_t* shared, void** stream) {
    *grid = pushed.grid;
    *block = pushed.block;
    *shared = pushed.shared;
    *stream = pushed.stream;
    return 0;
}
int hipLaunchKernel(const void* f, dim3 g, dim3 b, void** args, size_t shared, void* stream) {
    (void)f; (void)args; (void)shared; (void)stream;
    if ((uint64_t)g.x * b.x >> 32 || (uint64_t)g.y * b.y >> 32 || (uint64_t)g.z * b.z >> 32 ||
        !g.x || !g.y || !g.z)
        return last_error = 9;                       /* hipErrorInvalidConfiguration */
    const size_t n = strlen(launches);
    snprintf(launches + n, sizeof launches - n, " %u,%u,%u,%u", g.x, g.y, g.z, b.x);
    return 0;
}
int hipGetLastError(void) {
    const int e = last_error;
    last_error = 0;
    return e;
}
int hipGetDevice(int* dev) {
    *dev = 0;
    return 0;
}
int hipDeviceGetAttribute(int* value, int attribute, int dev) {
    (void)attribute; (void)dev;
    *value = 256;                                    /* compute units */
    return 0;
}

int main(void) {
    char line[256], what[16];
    void* P = (void*)(uintptr_t)(1u << 20);
    const masq_dtype dts[2] = {MASQ_F32, MASQ_BF16};
    while (fgets(line, sizeof line, stdin)) {
        long long a[11] = {0};
        if (sscanf(line, "%15s %lld %lld %lld %lld %lld %lld %lld %lld %lld %lld %lld", what, a, a + 1, a + 2,
                   a + 3, a + 4, a + 5, a + 6, a + 7, a + 8, a + 9, a + 10) < 1)
            continue;
        long long st = -1;
        launches[0] = 0;
        for (int shy = 1; shy >= 0; --shy) {
            size_t ws = 0;
            if (!strcmp(what, "epilogue")) {
                ws = masq_linear_fused_workspace_bytes(a[0], a[1], a[2], (int32_t)a[3], (int32_t)a[4]);
                st = masq_linear_epilogue(P, dts[a[5] & 1], P, P, P, (int32_t)a[7], P, P, P, dts[a[6] & 1], a[0],
                                          a[1], a[2], (int32_t)a[3], (int32_t)a[4], P, (int32_t)a[8], P, P,
                                          dts[a[5] & 1], P, ws - (size_t)shy, NULL);
            } else if (!strcmp(what, "route")) {
                ws = masq_route_experts_workspace_bytes(a[0], (int32_t)a[1]);
                if (ws == 0) shy = 0;
                st = masq_route_experts(P, dts[a[3] & 1], a[4] ? P : NULL, a[0], (int32_t)a[1], (int32_t)a[2], 1,
                                        P, P, P, P, P, a[4] ? P : NULL, P, ws - (size_t)shy, NULL);
            } else if (!strcmp(what, "experts")) {
                ws = masq_expert_linear_workspace_bytes(a[0], a[1], a[3], (int32_t)a[5], (int32_t)a[6]);
                st = masq_expert_linear(P, dts[a[7] & 1], a[0], P, P, P, (int32_t)a[8], P, P, P, dts[a[7] & 1],
                                        a[10] ? P : NULL, P, a[1], (int32_t)a[2], a[3], a[4], (int32_t)a[5],
                                        (int32_t)a[6], P, (int32_t)a[9], P, dts[a[7] & 1], P, ws - (size_t)shy,
                                        NULL);
            } else if (!strcmp(what, "combine")) {
                shy = 0;
                st = masq_combine_experts(P, dts[a[4] & 1], P, P, a[0], a[1], a[2], (int32_t)a[3], P, P, NULL);
            }
            if (shy && st != MASQ_ERR_WORKSPACE) break;
        }
        printf("%lld%s\n", st, launches);
    }
    return 0;
}
