// The kernels of the attention of a draft tree that are launched for heads of 128, bf16 rows or (-DROWS_OF_8_BITS=true) 8-bit ones.  Compiled to assembly by
// test_tree_assembly.py.
#include "decode_tree.h"
#define FAIRKV_BOTH(WC, WT, STAGES)                                                                                          \
    template __global__ void fairkv::fairkv_decode_tree_kernel<128, ROWS_OF_8_BITS, WC, WT, STAGES, 2>(fairkv::TreeArgs);               \
    template __global__ void fairkv::fairkv_decode_tree_kernel<128, ROWS_OF_8_BITS, WC, WT, STAGES, 3>(fairkv::TreeArgs);
FAIRKV_BOTH(1, 4, 2)
FAIRKV_BOTH(2, 4, 2)
FAIRKV_BOTH(4, 2, 3)
FAIRKV_BOTH(8, 1, 4)
