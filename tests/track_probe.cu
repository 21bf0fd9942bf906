// Brings a plan's tracked tables into the state that a call leaves whose
// waits gave up: parts counted that never met, and the word that says so.
#include <vector>

#include "salt_attn.cuh"

extern "C" int track_after_timeout(salt_attn *a)
{
    const std::vector<uint32_t> counts(salt::TRACK_SLOTS * 8, 1u);
    const int32_t failed = 1;
    if (cudaDeviceSynchronize() != cudaSuccess) return 1;
    if (cudaMemcpy(a->track.arrived, counts.data(), counts.size() * 4, cudaMemcpyHostToDevice) != cudaSuccess) return 2;
#ifndef COUNTS_ONLY
    if (cudaMemcpy(a->track.table + salt::TH_FAILED, &failed, 4, cudaMemcpyHostToDevice) != cudaSuccess) return 3;
#else
    (void)failed;
#endif
    return cudaDeviceSynchronize() != cudaSuccess;
}
// Parts of units that meet in the plan's batch.
extern "C" int track_split(const salt_attn *a) { return a->track.split; }
