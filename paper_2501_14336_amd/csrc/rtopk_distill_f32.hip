// Distillation in one launch, for RTOPK_F32 logits.
#include "rtopk_distill_step.inl"

namespace rtopk {
rtopk_status launch_distill_step_f32(const DistillParams& P, int64_t vecs, hipStream_t st) { return launch_step_of<RTOPK_F32>(P, vecs, st); }
}  // namespace rtopk
