// Who holds which slot of a static table of device words (host code only, no CUDA).
//
// A plan's kernels count in its slot, and a run is asynchronous: a plan may be destroyed while its runs are still queued.
// Its slot then stays out of use until something has waited for the device, and one whose runs were captured in a graph, which
// may be replayed at any time, is never handed on.  Slots that no run can touch any more go first, so that waiting is for a
// program that has destroyed as many plans as there are slots.
#pragma once
#include <cstdint>
#include <mutex>

namespace nk {

class SlotTable {
public:
    static constexpr int SLOTS = 1024;

    // A slot, or -1.  `wait`: returns once every run queued on the device has ended, or false.
    template <typename Wait>
    int take(Wait wait) {
        std::lock_guard<std::mutex> lock(mutex_);
        int slot = find_idle();
        if (slot < 0 && any(IN_FLIGHT) && wait()) {
            for (uint8_t& s : state_)
                if (s == IN_FLIGHT) s = IDLE;
            slot = find_idle();
        }
        if (slot >= 0) state_[slot] = TAKEN;
        return slot;
    }
    // in_flight: a run may not have ended; captured: a graph holds one
    void give(int slot, bool in_flight, bool captured) {
        if (slot < 0) return;
        std::lock_guard<std::mutex> lock(mutex_);
        state_[slot] = captured ? RETIRED : in_flight ? IN_FLIGHT : IDLE;
    }

private:
    enum : uint8_t { IDLE = 0, TAKEN, IN_FLIGHT, RETIRED };
    int find_idle() const {
        for (int i = 0; i < SLOTS; ++i)
            if (state_[i] == IDLE) return i;
        return -1;
    }
    bool any(uint8_t what) const {
        for (uint8_t s : state_)
            if (s == what) return true;
        return false;
    }
    std::mutex mutex_;
    uint8_t state_[SLOTS] = {};
};

}  // namespace nk
