// Positions asked for ahead of those that are worked on, kept inside a range (nothing of HIP in here: a test compiles it for the host).
#pragma once

namespace lccrf {
namespace enc {

// Whether l + more lies before `stop`; positions go up to 2^31 - 1024 and loads ahead of the last ones reach past 2^31, so the sum is not formed.
constexpr bool before(int l, int more, int stop) { return more < stop - l; }
// l + more, or the last position where that is past it.
constexpr int or_last(int l, int more, int stop) { return before(l, more, stop) ? l + more : stop - 1; }

}  // namespace enc
}  // namespace lccrf
