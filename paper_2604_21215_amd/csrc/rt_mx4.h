// Internal interface of the 4-bit read-out (rt_mx4.hip).
#pragma once
#include "rt_common.h"
#include "rt_paged_args.h"

namespace rt {

template <typename T>
hipError_t mx4_head_launch(const uint8_t *codes, const uint8_t *exps, const void *g, const void *z, long long z_stride, float *logits, int B,
                           int d, int vocab, float eps, int norm_free, hipStream_t st);
// host memory: rows x cols weights (fp32, or bf16 bits) -> codes [rows][cols / 2], exps [rows][cols / 32]; false: a value is not finite
bool mx4_pack_host(const void *W, bool bf16, long long rows, int cols, uint8_t *codes, uint8_t *exps);

}  // namespace rt
