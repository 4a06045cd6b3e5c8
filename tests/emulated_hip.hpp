// Runs a kernel's device code on the CPU, one workgroup at a time: every thread is a context of its own, switched at barriers and at exchanges between the lanes
// of a wavefront, so that both mean what they mean on the device.  For integer code without matrix instructions (schedules and tables); included before the sources, whose
// qualifiers and builtins it takes over.  A barrier or an exchange that not all threads reach ends the run with an error.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <ucontext.h>

#include <cstdio>
#include <cstdlib>
#include <functional>
#include <vector>

namespace emulated {

struct Index { unsigned x = 0, y = 0, z = 0; };
inline Index thread_idx, block_idx, block_dim, grid_dim;

struct Meeting {                        // of `size` threads, generation after generation; two sets of values, so that a fast thread does not overwrite what a slow one reads
    unsigned size = 0, here = 0, turn = 0;
    std::vector<uint64_t> value[2];
};
struct Workgroup {
    unsigned threads = 0, running = 0, done = 0;
    uint64_t arrivals = 0;              // at meetings
    std::vector<ucontext_t> at;
    std::vector<char> finished;
    std::vector<std::vector<char>> stacks;
    std::vector<Meeting> waves;
    Meeting all;
    ucontext_t home;
    std::function<void()> body;
};
inline Workgroup group;

inline void step_aside() { swapcontext(&group.at[group.running], &group.home); }

// waits until every thread of the meeting has come; returns which of the two sets holds this generation's values
inline unsigned meet(Meeting &m, unsigned place, uint64_t v)
{
    const unsigned mine = m.turn, set = mine & 1;
    ++group.arrivals;
    if (!m.value[set].empty()) m.value[set][place] = v;
    if (++m.here == m.size) { m.here = 0; ++m.turn; }
    while (m.turn == mine) step_aside();
    return set;
}

inline void barrier() { meet(group.all, 0, 0); }
inline unsigned lane() { return group.running & 63; }
inline Meeting &wave() { return group.waves[group.running >> 6]; }

template <typename V> uint64_t bits(V v) { uint64_t r = 0; static_assert(sizeof(V) <= 8, ""); __builtin_memcpy(&r, &v, sizeof(V)); return r; }
template <typename V> V from_bits(uint64_t r) { V v; __builtin_memcpy(&v, &r, sizeof(V)); return v; }

template <typename V> V exchange(V v, int from)
{
    Meeting &w = wave();
    const unsigned set = meet(w, lane(), bits(v));
    return from_bits<V>(w.value[set][(unsigned)from & 63]);
}
template <typename V> V shfl(V v, int from, int) { return exchange(v, from); }
template <typename V> V shfl_up(V v, int by, int) { return exchange(v, (int)lane() < by ? (int)lane() : (int)lane() - by); }
template <typename V> V shfl_xor(V v, int with, int) { return exchange(v, (int)lane() ^ with); }
template <typename V> V readlane(V v, int from) { return exchange(v, from); }
inline uint64_t ballot(bool on)
{
    Meeting &w = wave();
    const unsigned set = meet(w, lane(), on);
    uint64_t r = 0;
    for (unsigned i = 0; i < w.size; ++i) r |= (uint64_t)(w.value[set][i] & 1) << i;
    return r;
}

inline void entry()
{
    group.body();
    group.finished[group.running] = 1;
    ++group.done;
    for (;;) step_aside();
}

// one workgroup of `threads` (a multiple of 64)
inline void run_block(unsigned threads, unsigned block, unsigned grid, std::function<void()> body, unsigned block_y = 0)
{
    block_dim.x = threads; block_idx.x = block; block_idx.y = block_y; grid_dim.x = grid;
    Workgroup &g = group;
    g.threads = threads;
    g.done = 0;
    g.body = std::move(body);
    g.at.resize(threads);
    g.finished.assign(threads, 0);
    if (g.stacks.size() < threads) g.stacks.resize(threads, std::vector<char>(64 << 10));
    g.all = Meeting{threads};
    g.waves.assign(threads / 64, Meeting{64});
    for (Meeting &w : g.waves) { w.value[0].resize(64); w.value[1].resize(64); }
    for (unsigned t = 0; t < threads; ++t) {
        getcontext(&g.at[t]);
        g.at[t].uc_stack.ss_sp = g.stacks[t].data();
        g.at[t].uc_stack.ss_size = g.stacks[t].size();
        g.at[t].uc_link = nullptr;
        makecontext(&g.at[t], entry, 0);
    }
    int idle = 0;                       // rounds in which nobody came any further: the last to arrive frees those before it for the next round
    while (g.done < threads) {
        const uint64_t before = g.arrivals + g.done;
        for (unsigned t = 0; t < threads; ++t) {
            if (g.finished[t]) continue;
            g.running = t;
            thread_idx.x = t;
            swapcontext(&g.home, &g.at[t]);
        }
        if (g.arrivals + g.done == before && g.done < threads && ++idle == 3) {
            std::fprintf(stderr, "emulated: %u of %u threads wait for a barrier or an exchange that the others never reach\n", threads - g.done, threads);
            std::exit(3);
        }
        if (g.arrivals + g.done != before) idle = 0;
    }
}

}  // namespace emulated

#undef __device__
#undef __global__
#undef __shared__
#undef __forceinline__
#undef __launch_bounds__
#define __device__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define threadIdx emulated::thread_idx
#define blockIdx emulated::block_idx
#define blockDim emulated::block_dim
#define gridDim emulated::grid_dim
#define __syncthreads emulated::barrier
#define __shfl emulated::shfl
#define __shfl_up emulated::shfl_up
#define __shfl_xor emulated::shfl_xor
#define __ballot emulated::ballot
#define __any(x) (emulated::ballot(x) != 0)
#define __builtin_amdgcn_readlane emulated::readlane
#define __builtin_amdgcn_readfirstlane(x) emulated::readlane(x, 0)
#define atomicAdd(p, v) emulated_add(p, v)
#define atomicMin(p, v) emulated_min(p, v)
#define __uint_as_float emulated::from_bits<float>
#define __float_as_uint(f) ((uint32_t)emulated::bits((float)(f)))
#define __hip_atomic_load(p, order, scope) (*(p))
template <typename T, typename V> T emulated_add(T *p, V v) { const T was = *p; *p = (T)(was + v); return was; }
template <typename T, typename V> T emulated_min(T *p, V v) { const T was = *p; if ((T)v < was) *p = (T)v; return was; }
