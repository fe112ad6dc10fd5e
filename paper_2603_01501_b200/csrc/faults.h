// Who has been told of what: faults that kernels count on a device are told to everyone who asks, not to the first alone.
#pragma once

#include <map>
#include <utility>

namespace {

// Per host thread: how many faults of a device it had been told of when it last asked on a stream.
struct FaultLedger {
    std::map<std::pair<int, const void *>, unsigned> told;
    bool news(int device, const void *stream, unsigned count) {
        unsigned &seen = told[{device, stream}];
        const bool more = count != seen;
        seen = count;
        return more;
    }
};

}  // namespace
