// The forward state-space scan of f32 sequences.
#include "scan_forward.h"

namespace dtst {
template int launch_scan_type<float>(const ScanArgs&, const ScanPointers&, hipStream_t);
}  // namespace dtst
