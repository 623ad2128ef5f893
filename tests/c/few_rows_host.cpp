// How many rows a block of the fp32 gradient for few rows takes, on the host (tests/test_few_rows.py).
#include "../../paper_2102_10485_amd/csrc/few_rows.h"

extern "C" int dgrad_sixteens(long long each, long long blocks, int k) { return gan::dgrad_sixteens(each, blocks, k); }
