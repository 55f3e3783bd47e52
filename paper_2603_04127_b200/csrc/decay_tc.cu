#include "decay.cuh"
namespace darkattn {
bool decay_tc_supported(const darkattn_decay_desc_t &) { return false; }
void decay_tc_split(darkattn_decay_plan_s *) {}
darkattn_status_t decay_tc_run(DecayArgs &, DecayPass *, int, cudaStream_t) { return DARKATTN_ERR_UNSUPPORTED; }
}
