// Host side of the calls for k experts per token under AddressSanitizer / UndefinedBehaviorSanitizer: argument checks with the kernel
// launchers replaced by stubs.  Built and run by tests/test_topk_abi.py: the run must end with "ok" and no sanitizer report.
#define main abi_driver_main
#include "abi_driver.cpp"
#undef main
#include <climits>
#include <cmath>

int smoe_launch_permute_topk(const smoe_layer*, const void*, const int32_t*, int, int, void*, int32_t*, int32_t*, int32_t*, hipStream_t) { return 0; }
int smoe_launch_combine_topk(const smoe_layer*, const void*, const int32_t*, const float*, const void*, int, int, void*, hipStream_t) { return 0; }
int smoe_launch_router_norm(const smoe_layer*, hipStream_t) { return 0; }
int smoe_launch_route_topk(const smoe_layer*, const smoe_topk_rule&, const float*, const void*, int, int32_t*, float*, int32_t*, float*, float*,
                           hipStream_t) { return 0; }
int smoe_launch_add_norm(const smoe_layer*, const void*, const void*, const float*, float, int, void*, void*, void*, void*, hipStream_t) { return 0; }
int smoe_launch_ffn_mx(const smoe_layer*, const void*, const void*, const int32_t*, int, const int32_t*, int, void*, hipStream_t) { return 0; }

int main() {
    void* p = (void*)0x10000;
    int32_t* i = (int32_t*)p;
    float* f = (float*)p;
    smoe_config c{12, 3, 64, 96, 128, SMOE_MXFP8, SMOE_GATE_FULL, 1};
    smoe_layer_t* h = nullptr;
    EXPECT(smoe_create(&c, &h), SMOE_OK);
    if (smoe_workspace_bytes(h) == 0 || smoe_slot_weight_bytes(h) == 0) return 2;
    smoe_topk_rule ok{2, SMOE_SCORE_SIGMOID, 4, 2, 2, 1, 1.f};
    EXPECT(smoe_route_topk(h, &ok, nullptr, p, 4, i, f, i, f, f, nullptr), SMOE_ESTATE);
    EXPECT(smoe_bind(h, f, p, p, f, p), SMOE_OK);
    for (int bad = 0; bad < 12; ++bad) {
        smoe_topk_rule r = ok;
        int32_t* v = &r.k;
        if (bad < 6) v[bad] = INT_MAX;
        else if (bad < 11) v[bad - 6] = INT_MIN;
        else r.scale = NAN;
        EXPECT(smoe_route_topk(h, &r, nullptr, p, 4, i, f, i, f, f, nullptr), SMOE_EINVAL);
    }
    EXPECT(smoe_route_topk(h, &ok, nullptr, p, INT_MAX, i, f, i, f, f, nullptr), SMOE_EINVAL);
    EXPECT(smoe_route_topk(h, &ok, nullptr, p, 65, i, f, i, f, f, nullptr), SMOE_EINVAL);
    EXPECT(smoe_permute_topk(h, p, i, INT_MAX, 16, p, i, i, i, nullptr), SMOE_EINVAL);
    EXPECT(smoe_permute_topk(h, p, i, 8, 16, p, i, i, i, nullptr), SMOE_OK);
    EXPECT(smoe_permute_topk(h, nullptr, i, 8, 16, nullptr, i, i, i, nullptr), SMOE_OK);
    EXPECT(smoe_combine_topk(h, p, i, f, nullptr, 64, 2, p, nullptr), SMOE_OK);
    EXPECT(smoe_combine_topk(h, p, i, f, nullptr, 64, 3, p, nullptr), SMOE_EINVAL);
    EXPECT(smoe_add_norm(h, p, nullptr, f, 0.f, 128, nullptr, p, nullptr, nullptr, nullptr), SMOE_OK);
    EXPECT(smoe_add_norm(h, p, nullptr, f, 0.f, INT_MIN, nullptr, p, nullptr, nullptr, nullptr), SMOE_EINVAL);
    EXPECT(smoe_expert_ffn_mx(h, p, p, i, 2, i, 64, p, nullptr), SMOE_ESTATE);
    EXPECT(smoe_expert_ffn_mx(h, p, p, nullptr, 2, i, 64, p, nullptr), SMOE_EINVAL);
    if (smoe_mx_scale_pitch(INT_MAX) || smoe_mx_scale_pitch(INT_MIN)) return 3;
    EXPECT(smoe_destroy(h), SMOE_OK);
    printf("ok\n");
    return 0;
}
