// Attention items over the 4-bit cache.
#include "attn_items.h"

namespace pa {
namespace dev {

template int launch_items<4>(const AttnArgs&, int32_t, int32_t, int32_t, hipStream_t, hipEvent_t,
                              hipEvent_t);

}  // namespace dev
}  // namespace pa
