// Linear attention, backward, bf16 tensors.
#include "gspn_linattn_bwd_impl.hpp"

namespace gspn {
namespace la {
hipError_t linattn_bwd_bf16(const BwdArgs& a) { return linattn_bwd_t<bf16>(a); }
}  // namespace la
}  // namespace gspn
