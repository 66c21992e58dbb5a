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

// Lanes 0 .. few - 1 of a warp wait 1 ms at most, the others 2 s, for an arrival that
// comes after 300 ms.  got[lane]: mbar_wait_warp's outcome, or mbar_wait's.
__global__ void warp_wait_kernel(int few, int together, int* got) {
    __shared__ uint64_t bar;
    if (threadIdx.x == 0) {
        mbar_init(&bar, 1);
        fence_mbar_init();
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        const uint64_t limit = (int)threadIdx.x < few ? 1000000ull : kWaitLimitNs;
        got[threadIdx.x] = together ? mbar_wait_warp(&bar, 0u, limit) : mbar_wait(&bar, 0u, limit);
    } else if (threadIdx.x == 32) {
        const uint64_t t0 = globaltimer_ns();
        for (int i = 0; i < 100000000 && globaltimer_ns() - t0 < 300000000ull; ++i) __nanosleep(1000);
        mbar_arrive(&bar);
    }
}

extern "C" int warp_wait_run(int few, int together, int* got) {
    warp_wait_kernel<<<1, 64>>>(few, together, got);
    return (int)cudaDeviceSynchronize();
}
