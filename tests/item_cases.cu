// Work items of the MoE layer made from tables that the caller fills in, with the checking
// build's bounds checks (test_gpu_item_checks.py).
#include <cuda.h>

#include "moe_experts.cuh"

using namespace crc;

struct Tables {
    int M, N, K, slots;
    int slot0, count, tile_e, tile_row, tile_rows;      // of tile 0 and of its expert's slot
    int ok, e, row0, rows;                               // the item
};

template <bool W8, int NT>
__global__ void item_kernel(uint8_t* shared, Tables* t, uint32_t* err) {
    MoeShared<W8, NT> s(shared);
    for (int e = 0; e < 128; ++e) s.slot[e] = t->slot0;
    s.count[0] = t->count;
    s.tile_e[0] = (uint16_t)t->tile_e;
    s.tile_row[0] = (uint16_t)t->tile_row;
    s.tile_rows[0] = (uint16_t)t->tile_rows;
    MoeArgs a = {};
    a.M = t->M, a.N = t->N, a.K = t->K, a.slots = t->slots;
    a.ft = a.dt = 1;
    a.err = err;
    MoeItems n = {};
    n.split_h = n.down = 1, n.end = 2, n.parts = 1;
    const MoeItem it = moe_item<W8, NT>(a, s, n, 0);
    t->ok = it.ok, t->e = it.e, t->row0 = it.row0, t->rows = it.rows;
}

extern "C" int item_bytes() { return MoeCfg<true, 64>::SMEM; }
extern "C" int item_run(int wide, uint8_t* shared, Tables* t, uint32_t* err) {
    if (wide) item_kernel<true, 64><<<1, 1>>>(shared, t, err);
    else item_kernel<false, 16><<<1, 1>>>(shared, t, err);
    return (int)cudaDeviceSynchronize();
}
