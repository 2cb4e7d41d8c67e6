// What the kernels of packed attention share: where a sequence's rows lie.
#pragma once
#include "vit_internal.h"

namespace vit {

struct SeqRange { int q_begin, q_len, k_begin, k_len; };

// The offsets live on the device and are the caller's: a sequence whose rows are not in order, not inside
// the buffers or more than the call allowed for is skipped, and the status word says so.
__device__ __forceinline__ bool seq_range(const vit_attention_problem& p, int seq, SeqRange& r, int* dev_status, bool report) {
  const int qb = p.q_offsets[seq], qe = p.q_offsets[seq + 1], kb = p.k_offsets[seq], ke = p.k_offsets[seq + 1];
  const bool ok = qb >= 0 && qe >= qb && qe <= p.q_rows && qe - qb <= p.max_q &&
                  kb >= 0 && ke >= kb && ke <= p.k_rows && ke - kb <= p.max_k;
  if (!ok) {
    if (report) atomicExch(dev_status, (int)VIT_ERR_OFFSETS);
    return false;
  }
  r = SeqRange{qb, qe - qb, kb, ke - kb};
  return true;
}

// The factor of dq and dk.  The one probability of a sequence with one key is 1 whatever its score, so that its
// gradient is zero; dout v and dout out are summed in different orders and leave a rounding of it.
__device__ __forceinline__ float gradient_scale(const vit_attention_problem& p, int k_len) { return k_len == 1 ? 0.f : p.scale; }

}  // namespace vit
