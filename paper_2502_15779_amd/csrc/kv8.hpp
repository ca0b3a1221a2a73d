// Paged 8-bit cache: what the append kernel and the attention kernels share.
#pragma once

#include "kv8_plan.hpp"
#include "rcp_internal.hpp"

namespace rcp {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v16f __attribute__((ext_vector_type(16)));

struct Kv8Table {
    const int* starts;   // null: one new token a sequence
    const int* lengths;
    const int* table;    // [sequences][width]
    int sequences, width, shift, n_pages, capacity;  // pages of 1 << shift tokens; capacity = width << shift
};

// Finds the unit `target` of a numbering in which sequence after sequence has count(b) units: (sequence, unit within it), or
// sequence -1 beyond the last one.  All lanes of a wavefront call it with the same target.
struct Kv8Unit {
    int b, within;
};

// sum over this lane and those below it
__device__ __forceinline__ int kv8_scan(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // from the lane before, two, four and eight before in a row of sixteen
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // a row's sum to the next one
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // the first half's to the second
    return v;
}

template <class F>
__device__ __forceinline__ Kv8Unit kv8_find(int sequences, int target, int lane, F count)
{
    int before = 0;
    for (int base = 0; base < sequences; base += 64) {
        const int b = base + lane;
        const int n = b < sequences ? count(b) : 0;
        const int sum = kv8_scan(n);
        const unsigned long long past = __builtin_amdgcn_ballot_w64(before + sum > target);
        if (past != 0) {
            const int at = __builtin_ctzll(past);
            const int prefix = __builtin_amdgcn_readlane(sum, at) - __builtin_amdgcn_readlane(n, at);
            return {base + at, target - before - prefix};
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return {-1, 0};
}

// sum of count(b) over the sequences, the same in every lane
template <class F>
__device__ __forceinline__ int kv8_total(int sequences, int lane, F count)
{
    int total = 0;
    for (int base = 0; base < sequences; base += 64) total += wave_sum(base + lane < sequences ? count(base + lane) : 0);
    return total;
}

}  // namespace rcp
