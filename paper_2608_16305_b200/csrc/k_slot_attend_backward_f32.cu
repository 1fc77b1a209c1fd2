// Slot attention, the backward pass's kernels for fp32: slot_attend.cuh.
#include "slot_attend.cuh"

namespace tgnn_slots {

template cudaError_t launch_type<true, float>(SlotArgs&, int*, cudaStream_t);

}  // namespace tgnn_slots
