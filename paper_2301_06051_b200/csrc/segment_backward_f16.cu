// Segment attention, backward, rows of __half.
#include "segment_backward.cuh"

template int dsvt_train::launch_backward<__half>(dsvt_ctx*, const dsvt_train::SegArgs&);
