// Where a bias's buckets begin (csrc/rkb_buckets.h), for tests on the host.
#include "rkb_buckets.h"

extern "C" void borders(int count, int max_distance, int *out) { rkb::set_borders(out, 128, count, max_distance); }
