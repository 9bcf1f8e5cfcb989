// Linear attention, forward and the walks of the state, bf16 tensors.
#include "gspn_linattn_fwd_impl.hpp"
#include "gspn_linattn_state_impl.hpp"

namespace gspn {
namespace la {
hipError_t linattn_fwd_bf16(const FwdArgs& a) { return linattn_fwd_t<bf16>(a); }
hipError_t linattn_state_bf16(const StateArgs& a, const StateArgs* b) { return linattn_state_t<bf16>(a, b); }
}  // namespace la
}  // namespace gspn
