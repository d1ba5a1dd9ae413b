// Block tables and slots from the lengths of requests.
#include "cache.hpp"

namespace comet {

namespace {

// What the steps tell each other about a request: its length and blocks before the call adds to them, what it adds, and the running number of its
// first new block.
struct Plan {
    int32_t length, held, fresh, add;
    int64_t first;
};
struct Head { int64_t count, left; };         // spare blocks with the ended requests' among them, and those that are left

constexpr int kPlan = 1024, kPos = 4096;      // requests whose places among the tokens a workgroup keeps in LDS

__device__ __forceinline__ int64_t within(int64_t x, int64_t hi) { return x < 0 ? 0 : x > hi ? hi : x; }

// Two running sums over the workgroup at once, in 32 bits (data-parallel moves) or 64: x and y become the sums up to and with each thread's, all_x and
// all_y those of all.  buf is used in turn, so that one barrier is enough.
__device__ __forceinline__ int32_t wave_upto(int32_t x) { return lanes_scan(x); }
__device__ __forceinline__ int64_t wave_upto(int64_t x) { return wave_scan(x); }
template <class I, int T> struct Sums {
    I (*buf)[2][T / kWave];
    int turn = 0;
    __device__ __forceinline__ void operator()(I &x, I &y, I &all_x, I &all_y) {
        const int wave = threadIdx.x / kWave;
        x = wave_upto(x), y = wave_upto(y);
        if ((threadIdx.x & (kWave - 1)) == kWave - 1) buf[turn][0][wave] = x, buf[turn][1][wave] = y;
        __syncthreads();
        I px = 0, py = 0;
        all_x = all_y = 0;
#pragma unroll
        for (int w = 0; w < T / kWave; ++w) {
            const I bx = buf[turn][0][w], by = buf[turn][1][w];
            if (w < wave) px += bx, py += by;
            all_x += bx, all_y += by;
        }
        x += px, y += py;
        turn ^= 1;
    }
};

// One workgroup: running sums over the requests, of the blocks that come back, of the blocks and tokens asked for, and of what is granted.  What
// was asked for grows with b, so that the requests that get new blocks are the first of those that want some: the running number of a
// block among all that are asked for is that among those granted.  Bound by its waits (the arrays from memory, three sums one after the other): 512 requests 4.4 us,
// 11 with sums by 64-bit shuffles.
template <class I, int T> __device__ __forceinline__ void plan(const MapArgs &a, Plan *p, Head *head, int32_t *at) {
    __shared__ I buf[2][2][T / kWave];
    Sums<I, T> sums{buf};
    const int t = threadIdx.x;
    I back = 0, blocks = 0, tokens = 0, rows = 0, taken = 0, all, more;
    const int64_t before = within(*a.count, a.S);
    if (a.ended)
        for (int64_t b0 = 0; b0 < a.B; b0 += T) {
            const int64_t b = b0 + t;
            I n = b < a.B && a.ended[b] ? (I)within(a.held[b], a.M) : 0, none = 0;
            sums(n, none, all, more);
            back += all;
        }
    const int64_t count = within(before + back, a.S);
    for (int64_t b0 = 0; b0 < a.B; b0 += T) {
        const int64_t b = b0 + t;
        const bool on = b < a.B, stays = on && !(a.ended && a.ended[b]);
        const int64_t held = stays ? within(a.held[b], a.M) : 0;
        const int64_t length = stays ? within(a.length[b], held * a.block) : 0;
        const int64_t asked = on && a.add[b] > 0 ? a.add[b] : 0;
        const bool fits = length + asked <= a.M * a.block;
        const int64_t need = fits ? (int64_t)((uint32_t)(length + asked + a.block - 1) / (uint32_t)a.block) - held : 0;
        const I want = need > 0 ? (I)need : 0;
        I block_no = want, token_no = fits ? (I)asked : 0;
        sums(block_no, token_no, all, more);
        block_no += blocks, token_no += tokens;
        blocks += all, tokens += more;
        const bool granted = fits && token_no <= a.N && (want == 0 || block_no <= count);
        const I add = granted ? (I)asked : 0, fresh = granted ? want : 0;
        I row = add, new_no = fresh;
        sums(row, new_no, all, more);
        row += rows;
        rows += all, taken += more;
        if (on) {
            Plan &x = p[b];
            x.length = (int32_t)length, x.held = (int32_t)held, x.fresh = (int32_t)fresh, x.add = (int32_t)add, x.first = block_no - want;
            a.pos[b + 1] = (int32_t)row;
            if (at) at[b + 1] = (int32_t)row;
        }
    }
    if (t == 0) {
        a.pos[0] = 0;
        if (at) at[0] = 0;
        head->count = count, head->left = count - taken;
    }
}

// The blocks of ended requests: behind the spare ones, as far as there is room.  Every one of `groups` workgroups runs through all requests for where their
// blocks go, and moves those of some.
template <class I, int T> __device__ __forceinline__ void give_back(const MapArgs &a, int group, int groups) {
    __shared__ I buf[2][2][T / kWave];
    __shared__ I number[T], where[T];
    Sums<I, T> sums{buf};
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave;
    const int64_t before = within(*a.count, a.S);
    I back = 0, all, more;
    for (int64_t b0 = 0; b0 < a.B; b0 += T) {
        const int64_t b = b0 + threadIdx.x;
        const I n = b < a.B && a.ended[b] ? (I)within(a.held[b], a.M) : 0;
        I upto = n, none = 0;
        sums(upto, none, all, more);
        number[threadIdx.x] = n, where[threadIdx.x] = back + upto - n;
        back += all;
        __syncthreads();
        for (int i = group * (T / kWave) + wave; i < T; i += groups * (T / kWave)) {
            const int64_t to = before + where[i];
            for (I j = lane; j < number[i] && to + j < a.S; j += kWave) a.spare[to + j] = a.table[(b0 + i) * a.ldt + j];
        }
        __syncthreads();
    }
}

// The requests' new lengths and blocks, once nobody reads the old ones any more.
__device__ __forceinline__ void bring_up_to_date(const MapArgs &a, const Plan *p, const Head *head, int64_t t, int64_t threads) {
    for (int64_t b = t; b < a.B; b += threads) a.length[b] = p[b].length + p[b].add, a.held[b] = p[b].held + p[b].fresh;
    if (t == 0) *a.count = (int32_t)head->left;
}

// Token i: its request by halving (pos is in LDS where there is room), its block from the table or, where that is new, from the spare ones.  A new
// block's first place is always among the call's tokens: that one enters it into the table.
__device__ __forceinline__ void token(const MapArgs &a, const Plan *p, const Head *head, const int32_t *pos, int64_t i) {
    const int B = (int)a.B;
    if (i >= pos[B]) {
        a.slot[i] = -1, a.place[i] = -1;
        return;
    }
    int lo = 0, hi = B;                                          // pos[lo] <= i < pos[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (pos[mid] <= i) lo = mid;
        else hi = mid;
    }
    const Plan x = p[lo];
    const uint32_t block = (uint32_t)a.block, place = (uint32_t)(x.length + ((int32_t)i - pos[lo])), j = place / block, in = place - j * block;
    int32_t *entry = a.table + lo * a.ldt + j;
    int32_t id;
    if ((int32_t)j >= x.held) {
        id = a.spare[head->count - 1 - (x.first + (int32_t)j - x.held)];
        if (in == 0) *entry = id;
    } else {
        id = *entry;
    }
    a.slot[i] = (int64_t)id * block + in;
    a.place[i] = (int32_t)place;
}

// The whole of it in one workgroup, with what the steps tell each other in LDS.
constexpr int kSmall = 512;                   // requests
template <int T> __global__ void __launch_bounds__(T) k_map_all(MapArgs a) {
    __shared__ Plan p[kSmall];
    __shared__ Head head;
    __shared__ int32_t pos[kSmall + 1];
    plan<int32_t, T>(a, p, &head, pos);
    if (a.ended) give_back<int32_t, T>(a, 0, 1);
    __syncthreads();
    bring_up_to_date(a, p, &head, threadIdx.x, T);
    for (int64_t i = threadIdx.x; i < a.N; i += T) token(a, p, &head, pos, i);
}
// The first workgroup plans; where requests have ended the others give their blocks back.
template <class I> __global__ void __launch_bounds__(kPlan) k_map_plan(MapArgs a, Plan *p, Head *head) {
    if (blockIdx.x == 0) plan<I, kPlan>(a, p, head, nullptr);
    else give_back<I, kPlan>(a, (int)blockIdx.x - 1, (int)gridDim.x - 1);
}
__global__ void __launch_bounds__(256) k_map_tokens(MapArgs a, const Plan *p, const Head *head) {
    bring_up_to_date(a, p, head, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256);
    __shared__ int32_t pos[kPos + 1];
    const bool near = a.B <= kPos;
    if (near) {
        for (int i = threadIdx.x; i <= a.B; i += 256) pos[i] = a.pos[i];
        __syncthreads();
    }
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < a.N; i += (int64_t)gridDim.x * 256) token(a, p, head, near ? pos : a.pos, i);
}

// One workgroup is enough for a few tokens: another launch and the memory between them take longer than its steps (8 requests: 2.9 us).
bool in_one(int64_t B, int64_t M, int64_t N) { return B <= kSmall && N <= 4 * kPlan && B * M <= 65536; }

}  // namespace

int64_t cache_map_work(int64_t B, int64_t M, int64_t N) { return in_one(B, M, N) ? 0 : (int64_t)sizeof(Head) + B * (int64_t)sizeof(Plan); }

hipError_t cache_map(const MapArgs &a, void *work, hipStream_t st) {
    if (in_one(a.B, a.M, a.N)) {
        if (a.N <= 256 && a.B <= 256) hipLaunchKernelGGL(k_map_all<256>, dim3(1), dim3(256), 0, st, a);
        else hipLaunchKernelGGL(k_map_all<kPlan>, dim3(1), dim3(kPlan), 0, st, a);
        return hipGetLastError();
    }
    Head *head = (Head *)work;
    Plan *p = (Plan *)(head + 1);
    // no sum is over all places of all requests
    const int64_t backs = !a.ended ? 0 : a.B < 16 * 64 ? (a.B + 15) / 16 : 64;
    if (a.B * a.M < (int64_t(1) << 31) / a.block) hipLaunchKernelGGL(k_map_plan<int32_t>, dim3((unsigned)(1 + backs)), dim3(kPlan), 0, st, a, p, head);
    else hipLaunchKernelGGL(k_map_plan<int64_t>, dim3((unsigned)(1 + backs)), dim3(kPlan), 0, st, a, p, head);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t groups = (a.N + 1023) / 1024;
    hipLaunchKernelGGL(k_map_tokens, dim3((unsigned)(groups < 1 ? 1 : groups < 65536 ? groups : 65536)), dim3(256), 0, st, a, p, head);
    return hipGetLastError();
}

}  // namespace comet
