// The selective scan's kernels with 4 states a lane.
#define SCAN_NS 4
#define SCAN_NAMESPACE scan_ns4
#include "ssm_scan_kernels.hpp"

void scan_launch_ns4(ScanPass pass, const ScanP& p, int lpc, int precision, int mode, unsigned blocks, hipStream_t s) {
  scan_ns4::launch(pass, p, lpc, precision, mode, blocks, s);
}
