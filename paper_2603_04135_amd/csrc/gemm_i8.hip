// 8-bit integer GEMMs: C[n, V] = (int8 H) (int8 W)^T with exact int32 sums, a scale per token and one per vocabulary row.
#include "few_tokens.h"

namespace dppo {
namespace {

DeviceSetup g_setup;
typedef EpiOut<true, float> EpiOutF32;
typedef EpiOut<true, uint16_t> EpiOutBf16;

hipError_t allow_all() {
    hipError_t e = allow_logits<EpiOutF32>();
    if (e == hipSuccess) e = allow_logits<EpiOutBf16>();
    if (e == hipSuccess) e = allow_logits<EpiStats<true, false>>();
    if (e == hipSuccess) e = allow_logits<EpiStats<true, true>>();
    if (e == hipSuccess) e = allow_few<true, FewStats<true>>();
    if (e == hipSuccess) e = allow_few<true, FewOut<true, float>>();
    if (e == hipSuccess) e = allow_few<true, FewOut<true, uint16_t>>();
    return e;
}

}  // namespace

int mfma_i8_setup(int* compute_units) { return g_setup.run(&allow_all, compute_units); }

void launch_logits_i8(const LogitsOut& g, const OperandScales& s, bool out_bf16, int cus, hipStream_t st) {
    if (out_bf16) launch_logits_out<true, uint16_t>(g, s, cus, st);
    else launch_logits_out<true, float>(g, s, cus, st);
}

void launch_stats_i8(const LogitsOut& g, const OperandScales& s, const StatsTiles& t, int cus, hipStream_t st) {
    launch_stats_tiles<true>(g, s, t, cus, st);
}

}  // namespace dppo
