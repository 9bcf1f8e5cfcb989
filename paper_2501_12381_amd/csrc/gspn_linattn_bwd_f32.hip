// Linear attention, backward, f32 tensors.
#include "gspn_linattn_bwd_impl.hpp"

namespace gspn {
namespace la {
hipError_t linattn_bwd_f32(const BwdArgs& a) { return linattn_bwd_t<float>(a); }
}  // namespace la
}  // namespace gspn
