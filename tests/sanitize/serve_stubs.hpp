// Launches of the ragged-batch and query/key calls, noted while serve_record is set.
#pragma once

#include <utility>
#include <vector>

#include "sf_launch.hpp"

namespace sf {
struct ServeRecord {
    std::vector<GdnRaggedArgs> gdn, prep, walk;
    std::vector<ConvRaggedArgs> conv;
    std::vector<std::pair<bool, QkArgs>> qk;
};
extern ServeRecord *serve_record;
}  // namespace sf
