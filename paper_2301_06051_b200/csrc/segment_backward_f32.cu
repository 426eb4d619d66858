// Segment attention, backward, rows of float.
#include "segment_backward.cuh"

template int dsvt_train::launch_backward<float>(dsvt_ctx*, const dsvt_train::SegArgs&);
