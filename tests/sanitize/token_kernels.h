// What the geometry-only launcher of a decoding tenant's operators has been asked to do.
#pragma once
#include <map>
namespace gacer {
struct TokenLaunches {
    long all = 0, stray_positions = 0;            // all: launches; rotations of no feature that were given positions all the same
    int device = -1;                              // that was current at the last launch
    std::map<const void *, long> in_place_at;     // rotations in place, by their memory
};
extern TokenLaunches token_launches;
extern int current_device;                        // what hipGetDevice says and hipSetDevice sets in this program
}  // namespace gacer
