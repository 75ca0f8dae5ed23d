// The kernels of attention_kv_rows.hpp for rows of a draft tree.
#include "attention_kv_rows.hpp"

namespace readme {

hipError_t launch_attention_tree_rows(readme_kv_type kt, const KvAttnArgs& a, int waves, hipStream_t s) {
    return rows_by_type<true>(kt, a, waves, s);
}

}  // namespace readme
