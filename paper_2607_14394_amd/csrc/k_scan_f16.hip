// The forward state-space scan of f16 sequences.
#include "scan_forward.h"

namespace dtst {
template int launch_scan_type<f16_t>(const ScanArgs&, const ScanPointers&, hipStream_t);
}  // namespace dtst
