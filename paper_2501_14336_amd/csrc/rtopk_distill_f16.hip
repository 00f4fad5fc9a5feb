// Distillation in one launch, for RTOPK_F16 logits.
#include "rtopk_distill_step.inl"

namespace rtopk {
rtopk_status launch_distill_step_f16(const DistillParams& P, int64_t vecs, hipStream_t st) { return launch_step_of<RTOPK_F16>(P, vecs, st); }
}  // namespace rtopk
