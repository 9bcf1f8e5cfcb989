// Group norm with an activation, channels last, f32 tensors.
#include "gspn_groupnorm_impl.hpp"

namespace gspn {
namespace gn {
hipError_t fwd_f32(const Args& a) { return fwd_t<float>(a); }
hipError_t bwd_f32(const Args& a) { return bwd_t<float>(a); }
}  // namespace gn
}  // namespace gspn
