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

constexpr float LOG_STEPS = 2048.f;  // steps of a kept logit's fixed point
constexpr int V_TILE = 128;          // vocabulary entries of one pair of a row's statistics
enum { KEEP_NONE = 0, KEEP_LOG = 1, KEEP_Z = 2 };

// What the logits leave for the gradient and what it becomes, in blocks of 64 vocabulary entries: [parts][blocks][rows][64]
// of 16 bits (KEEP_Z: fp32, one part), zero from the vocabulary's end to its last block's.
struct Blocks {
  void* p;
  int dtype;
  int64_t rows, vocab;
  int parts;
  int64_t blocks() const { return (vocab + 63) / 64; }
};

// Logits z = H W^T: of each row the maximum and the sum of exp(z - maximum) over every V_TILE entries without the target (part,
// [tile][part_ld]; minus infinity and 0 where there is none) and the target's logit (zt; row r has targets[r % T]); keep:
// min(65535, round(LOG_STEPS (maximum - z))) as 16-bit integers, or z in fp32, to G (the target's entry there is not its logit).
int launch_logits(Ctx* ctx, const Operand& W, const Operand& H, float2* part, int64_t part_ld, float* zt, const void* targets,
                  int id64, int64_t T, int keep, const Blocks& G);
// The same for a few fp32 rows as they are (keep: KEEP_NONE or KEEP_Z); few_rows says when.
int launch_logits_few(Ctx* ctx, const float* W, int64_t vocab, const float* H, int64_t rows, int d, float2* part,
                      int64_t part_ld, float* zt, const void* targets, int id64, int64_t T, int keep, const Blocks& G);
bool few_rows(const Ctx* ctx, int64_t rows, int64_t vocab, int d);
// out [G.rows, W.cols] of dtype = alpha G W.
int launch_by_h(Ctx* ctx, const Operand& W, const Blocks& G, const float* alpha, void* out, int dtype);
// out [G.vocab, H.cols] of dtype = alpha G^T H, added to out (fp32) with add; rows without a target are not taken.
int launch_by_w(Ctx* ctx, const Blocks& G, const Operand& H, const void* targets, int id64, const float* alpha, void* out,
                int dtype, int add);

}  // namespace ce
}  // namespace zoact
