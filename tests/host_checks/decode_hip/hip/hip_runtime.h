// The stand-in of tests/host_checks/serve_hip, with the vector types that salt_decode.cpp names.
#pragma once
#include "../../serve_hip/hip/hip_runtime.h"

struct float2 { float x, y; };
struct double2 { double x, y; };
