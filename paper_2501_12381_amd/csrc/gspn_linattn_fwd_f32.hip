// Linear attention, forward and the walks of the state, f32 tensors.
#include "gspn_linattn_fwd_impl.hpp"
#include "gspn_linattn_state_impl.hpp"

namespace gspn {
namespace la {
hipError_t linattn_fwd_f32(const FwdArgs& a) { return linattn_fwd_t<float>(a); }
hipError_t linattn_state_f32(const StateArgs& a, const StateArgs* b) { return linattn_state_t<float>(a, b); }
}  // namespace la
}  // namespace gspn
