#include "ffn_launch.h"

template struct ecrm::BlockLaunch<__bf16>;
