// The gated recurrence of bf16 operands: see recurrence_kernel.h.
#include "recurrence_kernel.h"

namespace darb {
hipError_t launch_recurrence_bf16(const RecurrenceCall &c, hipStream_t s) { return launch_type<bf16_t>(c, s); }
}  // namespace darb
