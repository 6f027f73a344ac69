// Device memory that a handle's operators use one after the other and that grows with the calls: host code on any memory functions.
#pragma once

#include <stdint.h>

namespace moshpit {

// A captured graph holds the address of the block that was in use at the capture, so a block that was outgrown stays until
// release().  Each block is at least half as large again as the one before it where there is memory for that, so the
// outgrown ones together are at most twice the one in use, and are few.
class Workspace {
public:
    static constexpr int kMost = 96;     // (1.5^96 > 2^56)

    void *block() const { return count ? blocks[count - 1] : nullptr; }

    // Whether block() has `bytes` bytes now.  get(bytes): new memory, or nullptr.
    template <typename Get> bool reserve(int64_t bytes, Get get)
    {
        if (bytes <= size) return true;
        if (count == kMost) return false;
        int64_t want = bytes > size + size / 2 ? bytes : size + size / 2;
        void *p = get(want);
        if (!p && want > bytes) p = get(want = bytes);
        if (!p) return false;
        blocks[count++] = p;
        size = want;
        return true;
    }

    // put(block): its memory goes back.
    template <typename Put> void release(Put put)
    {
        while (count > 0) put(blocks[--count]);
        size = 0;
    }

private:
    void *blocks[kMost] = {};
    int count = 0;
    int64_t size = 0;                    // of the last one
};

}  // namespace moshpit
