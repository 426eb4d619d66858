// Segment attention, forward, rows of __nv_bfloat16.
#include "segment_forward.cuh"

template int dsvt_train::launch_forward<__nv_bfloat16>(dsvt_ctx*, const dsvt_train::SegArgs&);
