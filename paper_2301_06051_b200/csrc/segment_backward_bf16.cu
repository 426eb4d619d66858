// Segment attention, backward, rows of __nv_bfloat16.
#include "segment_backward.cuh"

template int dsvt_train::launch_backward<__nv_bfloat16>(dsvt_ctx*, const dsvt_train::SegArgs&);
