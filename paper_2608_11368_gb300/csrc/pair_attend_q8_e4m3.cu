// pair_attend_paged_q8 for chunks with few rows: bf16 queries over codes that are e4m3.
#include "pair_attend_q8_few.cuh"

namespace pairk {
namespace attend {

pair_status launch_few_e4m3(Launch *l, int D, int64_t most_rows, int slots, cudaStream_t s) {
  return run_few<__nv_bfloat16, kE4M3>(l, D, most_rows, slots, s);
}

}  // namespace attend
}  // namespace pairk
