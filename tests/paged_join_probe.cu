// The joining of sc_paged_decode_attn's partial sums (paged_attn.cuh) with made-up sums: clusters of blocks go along a line of units as the decode
// kernels do, block `late` waits for `delay_ns` before it joins its segment `late_segment`.  Every wait here ends: the delay and the limits are
// clocked, a block that left is not waited for.
#include "paged_attn.cuh"

namespace {

using namespace sc;
using namespace sc::pg;

constexpr int kD = 64, kNh = 3;

// What block `rank` of a party has for a unit: four columns' weighted sums, and a head's maximum and sum of weights.
__device__ __forceinline__ float value(int unit, int party, int rank, int hd, int column) {
    return (float)((unit * 7 + party * 13 + rank * 29 + hd * 3 + column) % 97) / 16.f;
}

__global__ void __launch_bounds__(kThreads) probe(Line line, const Division how, int late, int late_segment, long long delay_ns, unsigned long long limit_ns,
                                                  float* out, int32_t* tickets, float* part, int32_t* status, unsigned long long* left) {
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int sh_last;
    __shared__ __align__(8) unsigned long long sh_bar[2];
    const int lane = threadIdx.x & 31;
    Party me;
    me.set_up(sh_bar);
    if (me.plan(line, how, lane)) {
        Joiner joiner = {sh_bar, smem, &sh_last, tickets, part, status, kHeads, 0u, true, limit_ns};
        int segment = 0;
        for (Place p = me.begin(line, lane);; ++segment) {
            const int nt = line.tiles(p.entry), take = (int)min((unsigned)(nt - p.tile), me.left);
            if ((int)blockIdx.x == late && segment == late_segment) {
                const unsigned long long t0 = umma::global_ns();
                while (umma::global_ns() - t0 < (unsigned long long)delay_ns) {}
            }
            __syncthreads();
            const auto sum = [&](int e4) {
                const int hd = e4 / (kD / 4), c = e4 % (kD / 4) * 4;
                return make_float4(value(p.entry, me.party, me.crank, hd, c), value(p.entry, me.party, me.crank, hd, c + 1),
                                   value(p.entry, me.party, me.crank, hd, c + 2), value(p.entry, me.party, me.crank, hd, c + 3));
            };
            const auto ml = [&](int hd) { return make_float2((float)((p.entry + me.party * 3 + me.crank * 2 + hd) % 5 - 2), 1.f + me.crank); };
            joiner.join(me, p, nt, take, kNh, kD, out + (int64_t)p.entry * kNh * kD, sum, ml);
            me.left -= take;
            if (me.left == 0) break;
            next_unit(line, p, nt);
            joiner.next(me);
        }
        joiner.leave(me);
    } else {
        me.step();
    }
    __syncthreads();
    if (threadIdx.x == 0) left[blockIdx.x] = umma::global_ns();
}

}  // namespace

extern "C" int run_probe(const int32_t* lens, int units, int parties, int cluster, int late, int late_segment, long long delay_ns, unsigned long long limit_ns,
                         float* out, int32_t* tickets, float* part, int32_t* status, unsigned long long* left, void* stream) {
    Line line;
    line.lens = lens; line.entries = units; line.per_entry = 1; line.cap = 1 << 20; line.parties = parties; line.spare = 0;
    const Division how = {cluster, 0u, 0xffffffffu, 0};
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(parties * cluster);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = 2 * recv_bytes(kD, kHeads);
    cfg.stream = (cudaStream_t)stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return (int)cudaLaunchKernelEx(&cfg, probe, line, how, late, late_segment, delay_ns, limit_ns, out, tickets, part, status, left);
}
