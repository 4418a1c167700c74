// Which form of attention's forward takes a call (csrc/rkb_attn_cut.h), for tests on the host.
#include "rkb_attn_cut.h"

extern "C" int few_queries_win(int64_t queries, int64_t columns, int bias) { return rkb::few_queries_win(queries, columns, bias != 0); }
