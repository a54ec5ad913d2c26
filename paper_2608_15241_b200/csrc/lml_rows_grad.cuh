// Adapter gradients with x as bf16 rows or as a checkpoint: what the host side of the library calls.
#pragma once
#include "lml_rows.cuh"

namespace lml {

struct RowsGradCall {
    const SlotSnapshot *snap, *snap_T;
    const __nv_bfloat16* low[2];   // the packed A of the table and of the transposed one, [slots][64][d_in, d_out]
    int slots[2];
    TmapCache* cache;
    uint32_t *status, *status_T;
    Rows x;
    const void* dy;
    const int32_t *seg_offsets, *ids, *ids_T;
    float *dA, *dB;
    void* workspace;
    uint32_t* arrived;   // of the table: a counter per CTA and pass, zero between calls
    int T, G, d_in, d_out, num_sms;
    bool accumulate;
};
size_t rows_grad_ws_bytes(int T, int G, int num_sms);
cudaError_t rows_grad_init();   // sets the dynamic shared memory attributes
cudaError_t launch_rows_grad(const RowsGradCall& a, cudaStream_t stream, int* launches);

}  // namespace lml
