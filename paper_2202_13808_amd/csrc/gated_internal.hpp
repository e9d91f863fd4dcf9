// What the sources of the gated projection share (internal header).
#pragma once

#include "common.hpp"
#include "dropit_layers.h"
