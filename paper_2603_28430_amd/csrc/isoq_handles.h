// The handles of the C ABI and what its translation units share (isoq_api.cpp:
// stage 1, append, logits, sketch; isoq_attn_api.cpp: attention and the pages
// of a cache).
#pragma once

#include <hip/hip_runtime_api.h>

#include <atomic>
#include <vector>

#include "isoq_attn_tables.h"
#include "isoq_internal.h"
#include "isoquant.h"

struct isoq_params {
    int variant, d, bits, n_sets;
    int device;
    float *dparams;                 // device, [n_sets][slots_per_set][params_per_slot], then the LUT
    size_t lut_offset;              // floats from dparams to the magnitude LUT (0: none)
    size_t mfma_offset;             // floats from dparams to the matrix-core parameters (0: none)
    int lut_cells;
    float lut_inv_h;
    std::vector<float> exported;    // unit parameters as used (Table 1 layout)
    float levels[16], thresholds[15];
    isoq::LevelDigits lv;             // levels as digits (the first set)
    size_t lv_offset;               // floats from dparams to the further sets
    int n_pass;                     // sets in all
    bool wide;                      // the logits need all sets and digit products
    bool attn_by_tables;              // AttnTables hold the levels (else attention decodes by the fp32 ones)
    // made by the first attention (0.05 to 0.09 ms, which handles that never attend do not pay)
    mutable std::atomic<const isoq::AttnTables *> attn_tables{nullptr};

    ~isoq_params() { delete attn_tables.load(); }
};

struct isoq_sketch {
    int variant, d, n_sets, m;
    int device;
    uint16_t *dfrag;                // device, [n_sets][m/16][d/32][64][8] fp16 of S' = S T^{-1}
    float *dS;                      // device, [m][d] fp32 of S (query side)
    std::vector<float> S;           // host copy of S as used
};

namespace isoq {

// Status `st` for a HIP call that returned e, its text kept for
// isoq_last_hip_error on this thread.
isoq_status hip_fail(hipError_t e, const char *where, isoq_status st = ISOQ_E_HIP);
// Whether the current device is the handle's.
isoq_status check_device(const isoq_params *p);
// Launch with `lds` bytes of dynamic LDS and pick up launch errors.
isoq_status launch_lds(const void *fn, dim3 grid, int threads, void **args, size_t lds, void *stream);
size_t record_bytes(int variant, int d, int bits);
// Widths of the decoding calls' tuned kernels.
bool decode_d(int d);
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p % a) == 0; }

}  // namespace isoq
