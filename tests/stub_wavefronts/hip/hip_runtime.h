// A workgroup on the host, for kernels that keep to one: every thread is a context of its own, and the order in which wavefronts run
// is the caller's.  What csrc/sample.hip uses of HIP, no more.
//
// A wavefront runs until all of its threads are at a barrier (or at their end), those of the other wavefronts meanwhile wait; then comes
// the next one in the chosen order.  Two accesses between two barriers therefore come in either order under some choice,
// and one that needs a barrier more gives a wrong result, every time.
#pragma once
#include <ucontext.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <memory>
#include <vector>

#define __global__
#define __device__
#define __host__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __align__(n) __attribute__((aligned(n)))

typedef int hipError_t;
typedef void* hipStream_t;
enum { hipSuccess = 0 };
inline hipError_t hipGetLastError() { return hipSuccess; }

struct dim3 {
    unsigned x;
    explicit dim3(unsigned x) : x(x) {}
};
struct alignas(8) float2 { float x, y; };
struct alignas(16) float4 { float x, y, z, w; };
struct alignas(8) uint2 { uint32_t x, y; };
struct alignas(16) uint4 { uint32_t x, y, z, w; };
inline float4 make_float4(float x, float y, float z, float w) { return float4{x, y, z, w}; }
inline float2 make_float2(float x, float y) { return float2{x, y}; }
using std::max;
using std::min;
inline long long max(long long a, int b) { return a > b ? a : b; }

namespace wavefronts {

constexpr int kLanes = 64;
struct Index { unsigned x; };

struct Thread {
    ucontext_t context;
    std::unique_ptr<char[]> stack;
    Index index;
    enum { kReady, kExchange, kBarrier, kEnd } state;
    int line;                   // of the barrier it is at
    uint64_t given;             // to the lanes of its wavefront
};
struct Group {
    std::vector<Thread> threads;
    ucontext_t scheduler;
    Thread* now = nullptr;
    std::function<void()> body;
    uint64_t seen[kLanes];      // what the lanes of the running wavefront gave last
};
inline Group group;
inline Index block;
// 0: the first wavefront first, and in a wavefront the last lane; 1: the other way round; others: wavefronts shuffled anew behind every
// barrier, by this seed
inline unsigned order = 0;
inline std::vector<int> lines;                          // of the barriers that were passed, once for each time
inline uint64_t random_state = 1;

struct Error { char text[160]; };
// (of the scheduler: the threads are left where they are)
[[noreturn]] inline void fail(const char* what, int a, int b) {
    Error e;
    snprintf(e.text, sizeof e.text, "workgroup %u: %s (%d, %d)", block.x, what, a, b);
    throw e;
}
inline void wait(int state, int line, uint64_t given) {
    Thread* t = group.now;
    t->state = (decltype(t->state))state;
    t->line = line;
    t->given = given;
    swapcontext(&t->context, &group.scheduler);
}
// what the lanes of the wavefront give, by lane
inline const uint64_t* exchange(uint64_t x) {
    wait(Thread::kExchange, 0, x);
    return group.seen;
}
inline int lane() { return group.now->index.x % kLanes; }

inline void begin(unsigned lo, unsigned hi) {
    Thread* t = reinterpret_cast<Thread*>((uintptr_t)lo | (uintptr_t)hi << 32);
    group.body();
    t->state = Thread::kEnd;
}
// Runs the wavefront until each of its threads is at a barrier or at its end.
inline void run_wavefront(int w) {
    Thread* t = &group.threads[w * kLanes];
    uint64_t mine[kLanes];
    for (;;) {
        for (int j = 0; j < kLanes; ++j) {
            const int i = order == 1 ? j : kLanes - 1 - j;
            if (t[i].state != Thread::kReady) continue;
            group.now = &t[i];
            swapcontext(&group.scheduler, &t[i].context);
        }
        int exchanging = 0;
        for (int i = 0; i < kLanes; ++i) exchanging += t[i].state == Thread::kExchange;
        if (!exchanging) return;
        if (exchanging != kLanes) fail("lanes apart at an exchange", w, exchanging);
        for (int i = 0; i < kLanes; ++i) mine[i] = t[i].given;
        memcpy(group.seen, mine, sizeof mine);
        for (int i = 0; i < kLanes; ++i) t[i].state = Thread::kReady;
    }
}
inline void run_workgroup(int threads, std::function<void()> body) {
    group.body = body;
    group.threads.resize(threads);
    for (int i = 0; i < threads; ++i) {
        Thread& t = group.threads[i];
        constexpr size_t kStack = 64 << 10;
        if (!t.stack) t.stack.reset(new char[kStack]);
        t.index.x = i;
        t.state = Thread::kReady;
        getcontext(&t.context);
        t.context.uc_stack.ss_sp = t.stack.get();
        t.context.uc_stack.ss_size = kStack;
        t.context.uc_link = &group.scheduler;
        const uintptr_t p = reinterpret_cast<uintptr_t>(&t);
        makecontext(&t.context, (void (*)())begin, 2, (unsigned)p, (unsigned)(p >> 32));
    }
    const int waves = threads / kLanes;
    std::vector<int> turn(waves);
    for (;;) {
        for (int w = 0; w < waves; ++w) turn[w] = order == 1 ? waves - 1 - w : w;
        if (order > 1)
            for (int w = waves - 1; w > 0; --w) {
                random_state = random_state * 6364136223846793005ull + 1442695040888963407ull;
                std::swap(turn[w], turn[(random_state >> 33) % (w + 1)]);
            }
        for (int w : turn) run_wavefront(w);
        int line = 0, waiting = 0;
        for (Thread& t : group.threads)
            if (t.state == Thread::kBarrier) {
                if (waiting++ && t.line != line) fail("threads at different barriers", line, t.line);
                line = t.line;
                t.state = Thread::kReady;
            }
        if (!waiting) return;
        lines.push_back(line);
    }
}
inline void launch(dim3 grid, int threads, std::function<void()> body) {
    random_state = order;
    for (unsigned b = 0; b < grid.x; ++b) {
        block.x = b;
        run_workgroup(threads, body);
    }
}

}  // namespace wavefronts

#define threadIdx (wavefronts::group.now->index)
#define blockIdx (wavefronts::block)
#define __syncthreads() wavefronts::wait(wavefronts::Thread::kBarrier, __LINE__, 0)

template <class T, class U>
T atomicAdd(T* p, U x) {
    const T old = *p;
    *p += (T)x;
    return old;
}

template <class To, class From>
To as(From x) {
    static_assert(sizeof(To) == sizeof(From), "");
    To y;
    memcpy(&y, &x, sizeof y);
    return y;
}
inline uint32_t __float_as_uint(float x) { return as<uint32_t>(x); }
inline float __uint_as_float(uint32_t x) { return as<float>(x); }
inline long long __double_as_longlong(double x) { return as<long long>(x); }
inline double __longlong_as_double(long long x) { return as<double>(x); }
inline int __popcll(unsigned long long x) { return __builtin_popcountll(x); }
inline int __ffsll(long long x) { return __builtin_ffsll(x); }
inline float __log2f(float x) { return std::log2(x); }

inline int __shfl_xor(int x, int s) { return (int)wavefronts::exchange((uint32_t)x)[wavefronts::lane() ^ s]; }
inline int __shfl_up(int x, int s) {
    const int at = wavefronts::lane() - s;
    return (int)wavefronts::exchange((uint32_t)x)[at < 0 ? wavefronts::lane() : at];
}
inline unsigned long long __ballot(int x) {
    const uint64_t* all = wavefronts::exchange(x != 0);
    unsigned long long m = 0;
    for (int i = 0; i < wavefronts::kLanes; ++i) m |= (unsigned long long)all[i] << i;
    return m;
}
inline int __builtin_amdgcn_readfirstlane(int x) { return (int)wavefronts::exchange((uint32_t)x)[0]; }
inline double __builtin_amdgcn_rcp(double x) { return (double)(float)(1.0 / x); }
// (masks of rows and banks are for other kernels than those that run here)
inline int __builtin_amdgcn_update_dpp(int, int x, int control, int, int, bool) {
    const int l = wavefronts::lane();
    const uint64_t* all = wavefronts::exchange((uint32_t)x);
    if (control < 0x100) return (int)all[(l & ~3) | ((control >> 2 * (l & 3)) & 3)];
    if (control == 0x141) return (int)all[l ^ 7];
    if (control == 0x128) return (int)all[l ^ 8];
    abort();                    // an exchange that is not known here
}
struct Pair {
    uint32_t v[2];
    uint32_t operator[](int i) const { return v[i]; }
};
// rows of 16 (halves of 32) that are odd in the first and even in the second change places; both operands are the same here
inline Pair __builtin_amdgcn_permlane16_swap(uint32_t x, uint32_t, bool, bool) {
    const int l = wavefronts::lane();
    const uint64_t* all = wavefronts::exchange(x);
    return Pair{{(uint32_t)all[l & ~16], (uint32_t)all[l | 16]}};
}
inline Pair __builtin_amdgcn_permlane32_swap(uint32_t x, uint32_t, bool, bool) {
    const int l = wavefronts::lane();
    const uint64_t* all = wavefronts::exchange(x);
    return Pair{{(uint32_t)all[l & ~32], (uint32_t)all[l | 32]}};
}
