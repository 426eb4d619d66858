// Segment attention, forward, rows of __half.
#include "segment_forward.cuh"

template int dsvt_train::launch_forward<__half>(dsvt_ctx*, const dsvt_train::SegArgs&);
