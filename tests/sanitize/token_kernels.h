// What the geometry-only launcher of a decoding tenant's operators has been asked to do.
#pragma once
namespace gacer {
struct TokenLaunches { long all = 0, in_place = 0; const void *last_in_place = nullptr; };
extern TokenLaunches token_launches;
}  // namespace gacer
