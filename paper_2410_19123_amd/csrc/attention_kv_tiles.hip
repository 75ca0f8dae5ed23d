// The kernels of attention_kv_tiles.hpp for rows that follow one another.
#include "attention_kv_tiles.hpp"

namespace readme {

hipError_t launch_attention_tiles(readme_kv_type kt, const KvAttnArgs& a, bool shares, hipStream_t s) {
    return tiles_by_type<false>(kt, a, shares, s);
}

}  // namespace readme
