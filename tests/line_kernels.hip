// A kernel of the attention of a draft tree that gives short pairs to one wave each, and one that does not.  Compiled to assembly by test_line_sums.py.
#include "decode_tree.h"
template __global__ void fairkv::fairkv_decode_tree_kernel<64, true, 1, 4, 2, 2>(fairkv::TreeArgs);
template __global__ void fairkv::fairkv_decode_tree_kernel<64, true, 8, 1, 4, 2>(fairkv::TreeArgs);
