// Group norm with an activation, channels last, bf16 tensors.
#include "gspn_groupnorm_impl.hpp"

namespace gspn {
namespace gn {
hipError_t fwd_bf16(const Args& a) { return fwd_t<bf16>(a); }
hipError_t bwd_bf16(const Args& a) { return bwd_t<bf16>(a); }
}  // namespace gn
}  // namespace gspn
