// Layout and codes of caches in 8 bits: shared by the kernels that store, load and attend.
#pragma once
#include "psd_internal.h"
#include "device_types.h"

// The codes of a tile lie in the order in which a lane of a 32x32 product takes them, 16 bytes at a time (psd.h): keys 16 channels of one position, values 16
// positions of one channel, those that the scores of the lane's half are of (8 b + 4 h + j).

// the largest code
__host__ __device__ constexpr float kv8_most(int format) { return format == PSD_KV8_INT8 ? 127.f : 448.f; }

// length of a unit: what lies outside the cache is cut
__device__ __forceinline__ int kv8_keys(const Kv8 &c, int u) { return c.lens ? min(max(c.lens[u], 0), c.len) : c.len; }
