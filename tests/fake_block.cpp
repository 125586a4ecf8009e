// The host side of the residual feed-forward block's calls on a device that does not exist: this program defines the HIP runtime
// functions that they use, so that the choice of kernels and the sizes of launches can be tested without a GPU.  Launched kernels do
// nothing but leave their (mangled) name, workgroups (x, y) and threads of one in the log; a launch of 2^32 threads or more fails, as it does on a device.
//
//   fake_block COMMAND...
//     linear:0:100:64:48:0      dn_linear_forward, then dn_linear_backward: type, rows, n_in, n_out, bytes by which every tensor misses 256
//     block:2:100:64:48:0       dn_ffn_forward, then dn_ffn_backward: type, rows, d, f, the same; dropout and every bias, fp32 gradients
//     norm:1:100:64:7:0         dn_norm_forward, then dn_norm_backward: type, rows, d, rows of a gate, the same; layer norms with everything
// One line per call: its status and its launches (name/x/y/threads).
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <string>
#include <vector>

#include <unistd.h>

#include "dn.h"

namespace {

std::string launches;
struct Dim3 { uint32_t x, y, z; };
struct Call { Dim3 grid, block; size_t shared; void *stream; } call;
int last = 0;

std::map<const void *, std::string> &names()   // (the library registers its kernels before this file's objects exist)
{
    static std::map<const void *, std::string> m;
    return m;
}

}  // namespace

extern "C" {

void **__hipRegisterFatBinary(const void *) { static void *module; return &module; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *f, char *, const char *name, unsigned, void *, void *, void *, void *, int *) { names()[f] = name; }
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t shared, void *stream) { call = Call{grid, block, shared, stream}; return 0; }
int __hipPopCallConfiguration(Dim3 *grid, Dim3 *block, size_t *shared, void **stream)
{
    *grid = call.grid; *block = call.block; *shared = call.shared; *stream = call.stream;
    return 0;
}
int hipLaunchKernel(const void *f, Dim3 grid, Dim3 block, void **, size_t, void *)
{
    launches += " " + names()[f] + "/" + std::to_string(grid.x) + "/" + std::to_string(grid.y) + "/" + std::to_string(block.x);
    if ((uint64_t)grid.x * block.x >> 32 || grid.y > 65535) return last = 9;   // hipErrorInvalidConfiguration
    return 0;
}
int hipGetLastError() { const int e = last; last = 0; return e; }

}  // extern "C"

int main(int argc, char **argv)
{
    for (int i = 1; i < argc; ++i) {
        char kind[16];
        int type, rows, n, m, off;
        if (sscanf(argv[i], "%15[^:]:%d:%d:%d:%d:%d", kind, &type, &rows, &n, &m, &off) != 6) return 2;
        void *const p = (void *)(uintptr_t)(0x10000 + off), *const ws = (void *)(uintptr_t)0x10000;   // nothing reads them
        int status[2];
        std::string made[2];
        if (kind[0] == 'l') {
            const dn_linear_desc d = {type, DN_F32, DN_ACT_GELU, rows, n, m, 0, 0, 0, 0, 0.1f, 1.f, 1, 2};
            status[0] = dn_linear_forward(&d, p, p, p, p, p, p, ws, dn_linear_forward_workspace_bytes(&d), nullptr);
            made[0].swap(launches);
            status[1] = dn_linear_backward(&d, p, p, p, p, p, p, p, ws, dn_linear_backward_workspace_bytes(&d), nullptr);
            made[1].swap(launches);
        } else if (kind[0] == 'n') {
            const dn_norm_desc d = {type, DN_F32, rows, n, DN_NORM_LAYER, DN_NORM_LAYER, m, 1.f, 1e-5f};
            status[0] = dn_norm_forward(&d, p, p, p, p, p, p, p, p, p, nullptr);
            made[0].swap(launches);
            status[1] = dn_norm_backward(&d, p, p, p, p, p, p, p, p, p, p, p, p, p, p, p, ws, dn_norm_backward_workspace_bytes(&d), nullptr);
            made[1].swap(launches);
        } else {
            const dn_ffn_desc d = {type, DN_F32, DN_ACT_SILU, rows, n, m, 0, 0, 0, 0.1f, 1.f, 1, 2};
            status[0] = dn_ffn_forward(&d, p, p, p, p, p, p, p, p, p, p, ws, dn_ffn_forward_workspace_bytes(&d), nullptr);
            made[0].swap(launches);
            status[1] = dn_ffn_backward(&d, p, p, p, p, p, p, p, p, p, p, p, p, p, ws, dn_ffn_backward_workspace_bytes(&d), nullptr);
            made[1].swap(launches);
        }
        for (int k = 0; k < 2; ++k) printf("%d%s\n", status[k], made[k].c_str());
        fflush(stdout);
    }
    _exit(0);
}
