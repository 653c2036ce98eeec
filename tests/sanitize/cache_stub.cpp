// Host-only stand-ins for the launchers of the operators on paged caches, for the
// sanitizer build (see kernels_stub.cpp).
#include "cache.h"

namespace mstar {
hipError_t launch_append4(const Append4Args&, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_unpack4(const Unpack4Args&, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_tables(const TablesArgs&, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_tiles4(const KArgs&, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_cascade4(const KArgs&, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_few4(const KArgs&, int, int, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_mixed4(const KArgs&, const KArgs&, bool, int, int, hipStream_t) { return hipErrorNotSupported; }
}  // namespace mstar
