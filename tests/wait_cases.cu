// Kernels that make bounded waits run out for some threads of a group and not for
// others, with the library's own helpers (test_gpu_wait_groups.py).
#include "row_team.cuh"

using namespace crc;

// Thread i's wait gives up at row give_up[i]; left[i]: the row at which it left.
__global__ void row_team_kernel(int warps, int rows, const int* give_up, int* left) {
    __shared__ float red[2][32];
    __shared__ uint32_t lost[2][32];
    const RowTeam team(warps);
    if (team.thread == 0) lost[0][team.id] = lost[1][team.id] = 0u;
    __syncthreads();
    int row = 0;
    for (int flip = 0; row < rows; ++row, flip ^= 1) {
        bool ok = row_tell(row != give_up[threadIdx.x], &lost[flip][team.id]);
        (void)row_reduce<false>(1.f, red[flip], team);
        ok = row_all(ok, &lost[flip][team.id], team);
        if (!ok) break;
    }
    left[threadIdx.x] = row;
}

extern "C" int row_team_run(int threads, int warps, int rows, const int* give_up, int* left) {
    row_team_kernel<<<1, threads>>>(warps, rows, give_up, left);
    return (int)cudaDeviceSynchronize();
}
