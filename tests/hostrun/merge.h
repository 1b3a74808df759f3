// The device helpers are in common.h here.
#pragma once
#include "common.h"
