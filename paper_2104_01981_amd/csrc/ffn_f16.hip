#include "ffn_launch.h"

template struct ecrm::BlockLaunch<_Float16>;
