// What the translation units of the C entry points share: stage timing, chunk sizes and small helpers.
#pragma once
#include "dppo_internal.h"

namespace dppo {

// Records a pair of events around its lifetime on the caller's stream while stage timing is on (dppo_timing_enable).
struct StageTimer {
    int stage; hipStream_t st; hipEvent_t a = nullptr, b = nullptr;
    StageTimer(int stage_, hipStream_t st_);
    ~StageTimer();
};

constexpr int32_t CHUNK_ALIGN = 256;      // token-chunk granularity (= GEMM tile edge)
constexpr size_t REGION_ALIGN = 256;
constexpr int DEFAULT_CUS = 256;          // MI355X; used where no device is at hand (size queries)

static inline int32_t round_up32(int64_t x, int32_t a) { return (int32_t)((x + a - 1) / a * a); }
static inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// End of an LM-head call without loss tokens, which writes its status word and nothing else.
int finish_without_tokens(const char* what, int32_t* status, hipStream_t st);

// Whether the dH GEMM of a call of N loss tokens reads W as it lies instead of a transposed blocked copy.
bool reads_w_directly(int64_t N, int32_t D);
// Chunk size for N loss tokens whose forward and backward run chunk by chunk (es: bytes of an operand element).
int32_t target_chunk(int64_t N, int32_t D, int32_t V, size_t es, int cus);

}  // namespace dppo
