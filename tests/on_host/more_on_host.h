// What the kernels of drafted tokens and of the rotation use beyond hip_on_host.h.
#pragma once
#include "hip_on_host.h"
#define __builtin_amdgcn_s_waitcnt(x) emu_wave("waitcnt")
inline void sincospif(float x, float *s, float *c) { *s = (float)sin(M_PI * (double)x); *c = (float)cos(M_PI * (double)x); }
