// How the heads of a token are shared out between waves (qk_norm.hip).
#pragma once

#include <cstdint>

namespace same {

// `cut` shares of `part` heads each; the last one may be smaller.
struct NormShares {
    int32_t part, cut;
};

// At most `split` shares, none of them empty: a wave reads its share's first head
// whatever else it finds there.
inline NormShares norm_shares(int32_t heads, int32_t split) {
    const int32_t part = (heads + split - 1) / split;
    return {part, (heads + part - 1) / part};
}

}  // namespace same
