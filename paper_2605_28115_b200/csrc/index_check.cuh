// The fault record that kernels with device-side index validation write.
#pragma once
#include <cstdint>
#include <cuda_runtime.h>

namespace civic {

// Fault record of the checked kernels: {code, plane, position, offending value}.  The first
// thread to find a fault claims word 0 (0 -> code) and fills in the rest; later faults leave the
// record alone, so it names ONE offending entry.  The record is sticky: only the caller clears it.
enum IndexFault { kIndexOk = 0, kIndexOutOfRange = 1, kIndexNotAscending = 2, kIndexBadPage = 3 };
__device__ __forceinline__ void report_bad_index(int32_t* record, int code, int plane, int pos, int value)
{
    if (atomicCAS(record, 0, code) == 0) {
        record[1] = plane;
        record[2] = pos;
        record[3] = value;
    }
}

}  // namespace civic
