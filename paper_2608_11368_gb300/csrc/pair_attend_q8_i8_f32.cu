// pair_attend_paged_q8 for chunks with few rows: fp32 queries over codes that are whole numbers.
#include "pair_attend_q8_few.cuh"

namespace pairk {
namespace attend {

pair_status launch_few_i8_f32(Launch *l, int D, int64_t most_rows, int slots, cudaStream_t s) {
  return run_few<float, kI8>(l, D, most_rows, slots, s);
}

}  // namespace attend
}  // namespace pairk
