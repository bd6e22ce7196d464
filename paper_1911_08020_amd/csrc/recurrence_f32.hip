// The gated recurrence of fp32 operands, and what its calls share: see recurrence_kernel.h.
#include "recurrence_kernel.h"

namespace darb {

hipError_t launch_recurrence_f16(const RecurrenceCall &c, hipStream_t s);
hipError_t launch_recurrence_bf16(const RecurrenceCall &c, hipStream_t s);

int64_t recurrence_workspace_bytes(int dtype, bool back, bool rows, int64_t H, int64_t T, int64_t batch) {
    const int size = dtype == DARB_F32 ? 4 : 2;
    const int V = kVector, C = back ? kSteps<true> : kSteps<false>;
    const Cut k = cut_of(V, C, size, rows, T, rows ? H : batch, rows ? batch : H);
    if (k.slabs == 1) return 0;
    const int64_t series = H * batch;
    return padded(8 * series * k.slabs) + padded(4 * series) + padded(series * k.slabs);
}

hipError_t launch_recurrence(const RecurrenceCall &c, hipStream_t s) {
    if (c.dtype == DARB_F32) return launch_type<float>(c, s);
    return c.dtype == DARB_F16 ? launch_recurrence_f16(c, s) : launch_recurrence_bf16(c, s);
}

}  // namespace darb
