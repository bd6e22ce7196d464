// The gated recurrence of fp16 operands: see recurrence_kernel.h.
#include "recurrence_kernel.h"

namespace darb {
hipError_t launch_recurrence_f16(const RecurrenceCall &c, hipStream_t s) { return launch_type<half_t>(c, s); }
}  // namespace darb
