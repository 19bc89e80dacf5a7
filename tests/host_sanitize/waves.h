// Runs kernels written for waves of 64 lanes on the CPU, a block at a time: every lane has a stack of its own and runs until
// it needs the others (a vote, an exchange, a barrier).  What is between two of these runs lane by lane, in a random order,
// and so do the waves between two barriers of the block: a result that depends on an order that no barrier gives comes out
// different.  Shared memory is static; memory accesses are what the compiler's sanitizers see.  x86-64 only (the switch of
// stacks).
#pragma once

#include <sys/mman.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <random>
#include <vector>

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static
#define __align__(n) __attribute__((aligned(n)))

struct Dim {
    uint32_t x;
};
inline Dim threadIdx, blockIdx, blockDim, gridDim;

namespace waves {

enum Need { kRuns, kVote, kExchange, kWaveBarrier, kBlockBarrier, kEnded };
struct Lane {
    void *stack = nullptr, *at = nullptr;
    Need need = kEnded;
    uint32_t value = 0;
};
struct State {
    std::vector<Lane> lanes;
    std::function<void()> kernel;
    void *scheduler = nullptr;
    uint32_t current = 0;
    uint64_t votes[16];
    uint32_t values[16][64];
};
inline State state;
constexpr size_t kStack = 256 << 10;

// Pushes what a function has to keep, leaves the stack in *from and goes on with `to`.
extern "C" void waves_switch(void **from, void *to);
asm(R"(
.text
.globl waves_switch
waves_switch:
    pushq %rbp
    pushq %rbx
    pushq %r12
    pushq %r13
    pushq %r14
    pushq %r15
    movq %rsp, (%rdi)
    movq %rsi, %rsp
    popq %r15
    popq %r14
    popq %r13
    popq %r12
    popq %rbx
    popq %rbp
    ret
)");

inline void fail(const char *what)
{
    std::printf("failed: %s (block %u, thread %u)\n", what, blockIdx.x, state.current);
    std::fflush(stdout);
    std::abort();
}
inline void wait(Need need, uint32_t value = 0)
{
    Lane &l = state.lanes[state.current];
    l.need = need;
    l.value = value;
    waves_switch(&l.at, state.scheduler);
}
inline void begin()
{
    state.kernel();
    wait(kEnded);
    fail("a lane that has ended runs");
}
inline void resume(uint32_t t)
{
    Lane &l = state.lanes[t];
    l.need = kRuns;
    state.current = t;
    threadIdx.x = t;
    waves_switch(&state.scheduler, l.at);
}

// A block of `threads` threads; rng (may be null) orders waves and lanes.
inline void run_block(uint32_t block, uint32_t threads, std::mt19937_64 *rng)
{
    blockIdx.x = block;
    if (state.lanes.size() < threads) state.lanes.resize(threads);
    for (uint32_t t = 0; t < threads; t++) {
        Lane &l = state.lanes[t];
        if (!l.stack) {
            l.stack = mmap(nullptr, kStack, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
            if (l.stack == MAP_FAILED) fail("no memory for a stack");
        }
        void **top = reinterpret_cast<void **>(static_cast<char *>(l.stack) + kStack) - 2;
        *top = reinterpret_cast<void *>(&begin);         // (the stack is aligned as behind a call)
        l.at = top - 6;
        l.need = kRuns;
    }
    const uint32_t count = threads / 64;
    std::vector<uint32_t> order(count), lanes(64);
    for (uint32_t w = 0; w < count; w++) order[w] = w;
    for (uint32_t l = 0; l < 64; l++) lanes[l] = l;
    for (;;) {
        if (rng) std::shuffle(order.begin(), order.end(), *rng);
        uint32_t at_barrier = 0, ended = 0;
        for (const uint32_t w : order) {
            // until all lanes of the wave have ended or are at the block's barrier
            for (;;) {
                if (rng) std::shuffle(lanes.begin(), lanes.end(), *rng);
                for (const uint32_t l : lanes)
                    if (state.lanes[w * 64 + l].need == kRuns) resume(w * 64 + l);
                uint32_t n[kEnded + 1] = {};
                for (uint32_t l = 0; l < 64; l++) n[state.lanes[w * 64 + l].need]++;
                if (n[kWaveBarrier]) {                   // (of the lanes of a branch; the others wait behind it)
                    for (uint32_t l = 0; l < 64; l++)
                        if (state.lanes[w * 64 + l].need == kWaveBarrier) state.lanes[w * 64 + l].need = kRuns;
                    continue;
                }
                if (n[kVote] + n[kExchange] == 0) {
                    if (n[kBlockBarrier] && n[kEnded]) fail("a barrier that not all lanes of a wave reach");
                    break;
                }
                if (n[kBlockBarrier] || (n[kVote] && n[kExchange])) fail("lanes that wait for different things");
                uint64_t vote = 0;
                for (uint32_t l = 0; l < 64; l++) {
                    Lane &x = state.lanes[w * 64 + l];
                    state.values[w][l] = x.value;
                    if (x.need == kEnded) continue;
                    if (x.value) vote |= uint64_t(1) << l;
                    x.need = kRuns;
                }
                state.votes[w] = vote;
            }
            (state.lanes[w * 64].need == kEnded ? ended : at_barrier)++;
        }
        if (ended == count) return;
        if (at_barrier && ended) fail("a barrier that not all waves reach");
        for (uint32_t t = 0; t < threads; t++) state.lanes[t].need = kRuns;
    }
}
template <class Kernel>
void launch(uint32_t blocks, uint32_t threads, std::mt19937_64 *rng, Kernel kernel)
{
    gridDim.x = blocks;
    blockDim.x = threads;
    state.kernel = kernel;
    std::vector<uint32_t> order(blocks);
    for (uint32_t b = 0; b < blocks; b++) order[b] = b;
    if (rng) std::shuffle(order.begin(), order.end(), *rng);
    for (const uint32_t b : order) run_block(b, threads, rng);
}

inline uint32_t exchange(uint32_t v, uint32_t from)
{
    const uint32_t t = state.current;
    wait(kExchange, v);
    return from < 64 ? state.values[t / 64][from] : v;
}
}  // namespace waves

inline uint64_t __ballot(int v)
{
    const uint32_t t = waves::state.current;
    waves::wait(waves::kVote, v != 0);
    return waves::state.votes[t / 64];
}
inline uint32_t __shfl_xor(uint32_t v, int mask, int) { return waves::exchange(v, (waves::state.current & 63) ^ uint32_t(mask)); }
inline uint32_t __shfl_up(uint32_t v, unsigned by, int)
{
    const uint32_t lane = waves::state.current & 63;
    return waves::exchange(v, lane >= by ? lane - by : lane);
}
inline int32_t __builtin_amdgcn_readlane(int32_t v, int lane)
{
    if (lane < 0 || lane > 63) waves::fail("a lane that there is not");
    return int32_t(waves::exchange(uint32_t(v), uint32_t(lane)));
}
template <class T>
T __builtin_amdgcn_readfirstlane(T v)
{
    const T first = T(waves::exchange(uint32_t(v), 0));
    if (first != v) waves::fail("lanes that disagree about what is uniform");
    return first;
}
inline uint32_t __builtin_amdgcn_mbcnt_lo(uint32_t mask, uint32_t add)
{
    const uint32_t lane = waves::state.current & 63;
    return add + uint32_t(__builtin_popcount(lane < 32 ? mask & ((1u << lane) - 1) : mask));
}
inline uint32_t __builtin_amdgcn_mbcnt_hi(uint32_t mask, uint32_t add)
{
    const uint32_t lane = waves::state.current & 63;
    return add + (lane < 32 ? 0u : uint32_t(__builtin_popcount(mask & ((1u << (lane - 32)) - 1))));
}
inline int __popcll(uint64_t v) { return __builtin_popcountll(v); }
inline void __builtin_amdgcn_wave_barrier() { waves::wait(waves::kWaveBarrier); }
inline void __syncthreads() { waves::wait(waves::kBlockBarrier); }
inline uint32_t atomicAdd(uint32_t *p, uint32_t v)
{
    const uint32_t before = *p;
    *p += v;
    return before;
}
