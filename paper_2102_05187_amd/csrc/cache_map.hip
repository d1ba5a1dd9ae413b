// Block tables and slots from the lengths of requests.
#include "cache.hpp"

namespace comet {

namespace {

// What the steps tell each other about a request: its length and blocks before the call adds to them, what it adds, the running number of its
// first new block, and, where it has ended, how many blocks come back and where among all that do.
struct Plan {
    int32_t length, held, fresh, gone;
    int64_t first, back;
};
struct Head { int64_t before, count; };      // spare blocks before the call, and with the ended requests' among them

constexpr int kPlan = 1024;

__device__ __forceinline__ int64_t within(int64_t x, int64_t hi) { return x < 0 ? 0 : x > hi ? hi : x; }

// One workgroup: running sums over the requests, of the blocks that come back, of the blocks and tokens asked for, and of what is granted.  What
// was asked for grows with b, so that the requests that get new blocks are the first of those that want some: the running number of a
// block among all that are asked for is that among those granted.
__device__ void plan(const MapArgs &a, Plan *p, Head *head) {
    __shared__ int64_t buf[kPlan / kWave];
    const int t = threadIdx.x;
    int64_t back = 0, blocks = 0, tokens = 0, rows = 0, taken = 0, all;
    const int64_t before = within(*a.count, a.S);
    if (a.ended)
        for (int64_t b0 = 0; b0 < a.B; b0 += kPlan) {
            const int64_t b = b0 + t;
            const int64_t n = b < a.B && a.ended[b] ? within(a.held[b], a.M) : 0;
            const int64_t upto = block_scan<kPlan>(n, buf, all);
            if (b < a.B) p[b].gone = (int32_t)n, p[b].back = back + upto - n;
            back += all;
        }
    const int64_t count = within(before + back, a.S);
    for (int64_t b0 = 0; b0 < a.B; b0 += kPlan) {
        const int64_t b = b0 + t;
        const bool on = b < a.B, stays = on && !(a.ended && a.ended[b]);
        const int64_t held = stays ? within(a.held[b], a.M) : 0;
        const int64_t length = stays ? within(a.length[b], held * a.block) : 0;
        const int64_t asked = on && a.add[b] > 0 ? a.add[b] : 0;
        const bool fits = length + asked <= a.M * a.block;
        const int64_t need = fits ? (length + asked + a.block - 1) / a.block - held : 0;
        const int64_t want = need > 0 ? need : 0;
        const int64_t block_no = blocks + block_scan<kPlan>(want, buf, all);
        blocks += all;
        const int64_t token_no = tokens + block_scan<kPlan>(fits ? asked : 0, buf, all);
        tokens += all;
        const bool granted = fits && token_no <= a.N && (want == 0 || block_no <= count);
        const int64_t add = granted ? asked : 0, fresh = granted ? want : 0;
        const int64_t row = rows + block_scan<kPlan>(add, buf, all);
        rows += all;
        block_scan<kPlan>(fresh, buf, all);
        taken += all;
        if (on) {
            Plan &x = p[b];
            x.length = (int32_t)length, x.held = (int32_t)held, x.fresh = (int32_t)fresh, x.first = block_no - want;
            a.length[b] = (int32_t)(length + add);
            a.held[b] = (int32_t)(held + fresh);
            a.pos[b + 1] = (int32_t)row;
        }
    }
    if (t == 0) {
        a.pos[0] = 0;
        head->before = before, head->count = count;
        *a.count = (int32_t)(count - taken);
    }
}

// The blocks of ended requests b, b + step, ..: behind the spare ones, as far as there is room.
__device__ __forceinline__ void give_back(const MapArgs &a, const Plan *p, const Head *head, int64_t b, int64_t step) {
    for (; b < a.B; b += step) {
        if (!a.ended[b]) continue;
        const int64_t n = p[b].gone, to = head->before + p[b].back;
        for (int64_t j = threadIdx.x; j < n && to + j < a.S; j += blockDim.x) a.spare[to + j] = a.table[b * a.ldt + j];
    }
}

// Token i: its request by halving, its block from the table or, where that is new, from the spare ones.  A new block's first place is
// always among the call's tokens: that one enters it into the table.
__device__ __forceinline__ void token(const MapArgs &a, const Plan *p, const Head *head, int64_t i) {
    int64_t lo = 0, hi = a.B;                                    // pos[lo] <= i < pos[hi]
    if (a.B == 0 || i >= a.pos[a.B]) {
        a.slot[i] = -1, a.place[i] = -1;
        return;
    }
    while (hi - lo > 1) {
        const int64_t mid = (lo + hi) >> 1;
        if (a.pos[mid] <= i) lo = mid;
        else hi = mid;
    }
    const Plan x = p[lo];
    const int64_t place = x.length + (i - a.pos[lo]), j = place / a.block, in = place - j * a.block;
    int32_t *entry = a.table + lo * a.ldt + j;
    int32_t id;
    if (j >= x.held) {
        id = a.spare[head->count - 1 - (x.first + j - x.held)];
        if (in == 0) *entry = id;
    } else {
        id = *entry;
    }
    a.slot[i] = (int64_t)id * a.block + in;
    a.place[i] = (int32_t)place;
}

__global__ void __launch_bounds__(kPlan) k_map_all(MapArgs a, Plan *p, Head *head) {
    plan(a, p, head);
    __syncthreads();
    if (a.ended) {
        give_back(a, p, head, 0, 1);
        __syncthreads();
    }
    for (int64_t i = threadIdx.x; i < a.N; i += kPlan) token(a, p, head, i);
}
__global__ void __launch_bounds__(kPlan) k_map_plan(MapArgs a, Plan *p, Head *head) { plan(a, p, head); }
__global__ void __launch_bounds__(256) k_map_back(MapArgs a, const Plan *p, const Head *head) { give_back(a, p, head, blockIdx.x, gridDim.x); }
__global__ void __launch_bounds__(256) k_map_tokens(MapArgs a, const Plan *p, const Head *head) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.N; i += (int64_t)gridDim.x * 256) token(a, p, head, i);
}

}  // namespace

int64_t cache_map_work(int64_t B, int64_t, int64_t) { return (int64_t)sizeof(Head) + B * (int64_t)sizeof(Plan); }

hipError_t cache_map(const MapArgs &a, void *work, hipStream_t st) {
    Head *head = (Head *)work;
    Plan *p = (Plan *)(head + 1);
    if (a.N <= 4 * kPlan && (!a.ended || a.B * a.M <= 65536)) {
        hipLaunchKernelGGL(k_map_all, dim3(1), dim3(kPlan), 0, st, a, p, head);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(k_map_plan, dim3(1), dim3(kPlan), 0, st, a, p, head);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && a.ended) {
        hipLaunchKernelGGL(k_map_back, dim3((unsigned)(a.B < 4096 ? a.B : 4096)), dim3(256), 0, st, a, p, head);
        e = hipGetLastError();
    }
    if (e == hipSuccess && a.N > 0) {
        const int64_t groups = (a.N + 255) / 256;
        hipLaunchKernelGGL(k_map_tokens, dim3((unsigned)(groups < 65536 ? groups : 65536)), dim3(256), 0, st, a, p, head);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace comet
