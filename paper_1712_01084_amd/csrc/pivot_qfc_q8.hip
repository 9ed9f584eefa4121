// Layers with 4-bit weights, 8-bit inputs (see pivot_qfc_kernel.h).
#include "pivot_qfc_kernel.h"

namespace pivot {
int qfc_launch_q8(const QfcHost& h, const QfcForm& f, const QfcArgs& a, void* stream) { return qfc_dispatch<true>(h, f, a, stream); }
}  // namespace pivot
