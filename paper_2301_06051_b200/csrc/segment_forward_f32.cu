// Segment attention, forward, rows of float.
#include "segment_forward.cuh"

template int dsvt_train::launch_forward<float>(dsvt_ctx*, const dsvt_train::SegArgs&);
