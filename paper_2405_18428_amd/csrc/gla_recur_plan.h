// Gated recurrence of channels: what host and kernels count by, with nothing of the GPU's in it.
#pragma once

namespace gla {

// Looks of a wait at what another unit publishes: `most` of them, or, where there is nothing to fall back to, any number, which is not counted
constexpr int kRecurNoEnd = -1;
struct RecurLooks {
    int most, made;
    constexpr bool another() {
        if (most == kRecurNoEnd) return true;
        if (made >= most) return false;
        ++made;
        return true;
    }
};

}  // namespace gla
