// Which form of a pass of attention its units can be counted in; plain C++, so that it can be tested without a device.
#pragma once

namespace asx {

// Units of work (2^shift tokens of an entry and a head) are counted in 31 bits on the device.  entries: lanes or groups x row
// tiles; tokens: the most that a lane can have.
inline bool units_fit(long long entries, long long heads, long long tokens, int shift) {
    const long long each = (tokens + (1LL << shift) - 1) >> shift;
    return (double)entries * (double)heads * (double)each <= 2147483647.0;
}

// A run for each warp counts units of 32 tokens, a run for each CTA units of 128, of which the entry point has made sure
// that they fit.  Warps where the items are many, or behind shared beginnings, where they are short (the figures stand at
// the launch), as long as their units can be counted.
inline bool runs_by_warps(long long entries, long long heads, long long tokens, bool behind_shared) {
    return (behind_shared || entries * heads >= 512) && units_fit(entries, heads, tokens, 5);
}

}  // namespace asx
