// The forward state-space scan of bf16 sequences.
#include "scan_forward.h"

namespace dtst {
template int launch_scan_type<bf16_t>(const ScanArgs&, const ScanPointers&, hipStream_t);
}  // namespace dtst
