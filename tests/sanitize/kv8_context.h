// For stream_checks.cpp: its contexts keep their cache in 8 bits.
#pragma once
#include "hh.h"
#define HH_WF_DTYPE HH_KV_Q8
