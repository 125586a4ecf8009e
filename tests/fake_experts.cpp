// The host side of the calls of a block of experts on the device that does not exist (fake_block.cpp).
//
//   fake_experts COMMAND...
//     experts:0:100:8:2:64:48:0   dn_experts_forward, then dn_experts_backward: type, rows, experts, k, d, f, bytes by which X, R, Y, dX and dY miss 256
//     route:1:100:64:8:1:1:0      dn_route_forward with its lists, then dn_route_backward: type, rows, experts, k, bias (0 or 1), groups (of which half stay), 0
//     clip:0:300:1000:1:0:0:0     dn_clip, twice (in place; the norm only): type, tensors, elements of each, 1 (rest 0)
// One line per call: its status and its launches (name/x/y/threads).
#define main block_main
#include "fake_block.cpp"
#undef main

int main(int argc, char **argv)
{
    for (int i = 1; i < argc; ++i) {
        char kind[16];
        int type, n[6];
        if (sscanf(argv[i], "%15[^:]:%d:%d:%d:%d:%d:%d:%d", kind, &type, n, n + 1, n + 2, n + 3, n + 4, n + 5) != 8) return 2;
        void *const ws = (void *)(uintptr_t)0x10000, *const w = ws;   // nothing reads them
        int32_t *const whole = (int32_t *)ws;
        float *const f32 = (float *)ws;
        int status[2];
        std::string made[2];
        if (kind[0] == 'e') {
            void *const p = (void *)(uintptr_t)(0x10000 + n[5]);
            const dn_experts_desc d = {type, DN_F32, DN_ACT_SILU, n[0], n[3], n[4], n[1], n[2], 0, 0, 0, 1.f};
            status[0] = dn_experts_forward(&d, p, w, w, w, f32, whole, whole, whole, p, p, w, ws, dn_experts_forward_workspace_bytes(&d), nullptr);
            made[0].swap(launches);
            status[1] = dn_experts_backward(&d, p, w, w, w, f32, whole, whole, whole, w, p, p, w, w, w, f32, ws, dn_experts_backward_workspace_bytes(&d), nullptr);
            made[1].swap(launches);
        } else if (kind[0] == 'r') {
            const int top = n[4] > 1 ? n[4] / 2 : 1;
            const dn_route_desc d = {type, DN_SCORE_SIGMOID, n[0], n[1], n[2], n[4], top, 1, 1, 1.f, 0};
            status[0] = dn_route_forward(&d, ws, n[3] ? f32 : nullptr, whole, f32, whole, whole, whole, ws, dn_route_workspace_bytes(n[0], n[1], n[2]), nullptr);
            made[0].swap(launches);
            status[1] = dn_route_backward(&d, ws, whole, f32, ws, nullptr);
            made[1].swap(launches);
        } else {
            std::vector<dn_span> s;
            for (int k = 0; k < n[0]; ++k) {
                char *at = (char *)ws + (size_t)k * n[1] * 4;
                s.push_back({at, at, n[1], type, type});
            }
            for (int k = 0; k < 2; ++k) {
                status[k] = dn_clip(s.data(), n[0], 1.f, (float *)(uintptr_t)0x1000, ws, dn_clip_workspace_bytes(s.data(), n[0]), nullptr);
                made[k].swap(launches);
                for (auto &v : s) v.out_dev = nullptr;
            }
        }
        for (int k = 0; k < 2; ++k) printf("%d%s\n", status[k], made[k].c_str());
        fflush(stdout);
    }
    _exit(0);
}
