// The cross entropy's tensor-core products (k_ce_tc.cu), on 16-bit operands or fp32 ones split into three bf16 parts.
#pragma once
#include "internal.h"

namespace zoact {
namespace ce {

// A row-major matrix [rows, cols] (rows ld apart) of dtype BF16 or FP16; parts 1, or 3 slabs part_stride elements apart.
struct Operand {
  const void* p;
  int dtype;
  int64_t rows, cols, ld;
  int parts;
  int64_t part_stride;
};

constexpr int V_TILE = 128;          // vocabulary entries of one pair of column statistics
enum { KEEP_NONE = 0, KEEP_LOG = 1, KEEP_Z = 2 };

// z^T = W H^T: per column n the maximum and the sum of exp(z - maximum) of each V_TILE entries (part, rows part_ld apart)
// and the target's logit (zt); keep: min(65535, round(4096 (maximum - z))) as 16-bit integers, or z in fp32, to G [H.rows, ldg].
int launch_logits(Ctx* ctx, const Operand& W, const Operand& H, float2* part, int64_t part_ld, float* zt, const void* targets,
                  int id64, int64_t T, int keep, void* G, int64_t ldg);
// out [G.rows, W.cols] of dtype = scale / max(count, 1) G W.
int launch_by_h(Ctx* ctx, const Operand& W, const Operand& G, const double* count, float scale, void* out, int dtype);
// out [G.cols, H.cols] of dtype = scale / max(count, 1) G^T H, added to out (fp32) with add.
int launch_by_w(Ctx* ctx, const Operand& G, const Operand& H, const double* count, float scale, void* out, int dtype, int add);

}  // namespace ce
}  // namespace zoact
