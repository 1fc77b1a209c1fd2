// Slot attention, the backward pass's kernels for bf16: slot_attend.cuh.
#include "slot_attend.cuh"

namespace tgnn_slots {

template cudaError_t launch_type<true, __nv_bfloat16>(SlotArgs&, int*, cudaStream_t);

}  // namespace tgnn_slots
