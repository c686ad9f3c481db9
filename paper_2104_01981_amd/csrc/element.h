// Sizes of the element types.
#pragma once

#include "ecrm.h"
#include "host_device.h"

namespace ecrm {

ECRM_HD uint32_t type_bytes(uint32_t type) { return type == ECRM_F32 ? 4u : 2u; }

}  // namespace ecrm
