// The selective scan's kernels with 8 states a lane.
#define SCAN_NS 8
#define SCAN_NAMESPACE scan_ns8
#include "ssm_scan_kernels.hpp"

void scan_launch_ns8(ScanPass pass, const ScanP& p, int lpc, int precision, int mode, unsigned blocks, hipStream_t s) {
  scan_ns8::launch(pass, p, lpc, precision, mode, blocks, s);
}
