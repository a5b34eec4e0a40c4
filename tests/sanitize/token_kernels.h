// What the geometry-only launcher of a decoding tenant's operators has been asked to do.
#pragma once
#include <map>
namespace gacer {
struct TokenLaunches {
    long all = 0, stray_positions = 0;            // all: launches; rotations of no feature that were given positions all the same
    std::map<const void *, long> in_place_at;     // rotations in place, by their memory
};
extern TokenLaunches token_launches;
}  // namespace gacer
