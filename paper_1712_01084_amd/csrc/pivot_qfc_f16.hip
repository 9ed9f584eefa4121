// Layers with 4-bit weights, fp16 inputs (see pivot_qfc_kernel.h).
#include "pivot_qfc_kernel.h"

namespace pivot {
int qfc_launch_f16(const QfcHost& h, const QfcForm& f, const QfcArgs& a, void* stream) { return qfc_dispatch<false>(h, f, a, stream); }
}  // namespace pivot
