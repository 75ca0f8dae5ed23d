// The kernels of attention_kv_rows.hpp for rows that follow one another.
#include "attention_kv_rows.hpp"

namespace readme {

hipError_t launch_attention_rows(readme_kv_type kt, const KvAttnArgs& a, int waves, hipStream_t s) {
    return rows_by_type<false>(kt, a, waves, s);
}

}  // namespace readme
