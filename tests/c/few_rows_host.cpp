// The rules for products of few rows, on the host (tests/test_few_rows.py).
#include "../../paper_2102_10485_amd/csrc/few_rows.h"

extern "C" int dgrad_sixteens(long long each, long long blocks, int k) { return gan::dgrad_sixteens(each, blocks, k); }
extern "C" int two_sets8(long long each, long long groups, long long cols, int k) { return gan::two_sets8(each, groups, cols, k); }
