// Stands in for csrc/common.h and csrc/merge.h where the tests compile a kernel
// source for the host: the workgroups of a launch run one after the other, in an
// order that the test chooses, their threads as fibers that meet at every barrier.
// Any order of workgroups is one that a device may take, so that a result that
// depends on it shows a race between them.
#pragma once

#include <stdint.h>
#include <ucontext.h>

#include <algorithm>
#include <memory>
#include <numeric>
#include <random>
#include <vector>

#include "wushkv.h"

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __shared__ static
#define __launch_bounds__(...)
#define __HIP_MEMORY_SCOPE_AGENT 0
#define __hip_atomic_load(p, order, scope) (*(p))

struct dim3 {
    unsigned x, y, z;
    dim3(unsigned x_ = 1, unsigned y_ = 1, unsigned z_ = 1) : x(x_), y(y_), z(z_) {}
};
struct alignas(16) int4 {
    int x, y, z, w;
};
static inline int4 make_int4(int x, int y, int z, int w) { return int4{x, y, z, w}; }
typedef void *hipStream_t;
enum { hipSuccess = 0 };
static inline int hipGetLastError() { return hipSuccess; }

static dim3 blockIdx, threadIdx, gridDim, blockDim;

namespace host {

constexpr size_t kStack = 32768;
static int order = 0;  // of the workgroups: 0 ascending, 1 descending, else shuffled by this seed
static ucontext_t scheduler, *current;
static void (*body)(void *);
static void *body_args;
static bool done;

static void enter()
{
    body(body_args);
    done = true;
    swapcontext(current, &scheduler);
}

static void barrier() { swapcontext(current, &scheduler); }

// One workgroup: every thread up to its next barrier, in turn, until all have ended.
static void run_workgroup(unsigned threads)
{
    static std::vector<ucontext_t> fibers(1024);
    static std::unique_ptr<char[]> stacks(new char[1024 * kStack]);
    std::vector<unsigned> alive(threads);
    std::iota(alive.begin(), alive.end(), 0u);
    for (unsigned t = 0; t < threads; ++t) {
        getcontext(&fibers[t]);
        fibers[t].uc_stack.ss_sp = stacks.get() + t * kStack;
        fibers[t].uc_stack.ss_size = kStack;
        fibers[t].uc_link = nullptr;
        makecontext(&fibers[t], enter, 0);
    }
    while (!alive.empty()) {
        std::vector<unsigned> next;
        for (unsigned t : alive) {
            threadIdx = dim3(t, 0, 0);
            current = &fibers[t];
            done = false;
            swapcontext(&scheduler, current);
            if (!done) next.push_back(t);
        }
        alive.swap(next);
    }
}

}  // namespace host

static inline void __syncthreads() { host::barrier(); }

template <class T, class U>
static inline T atomicAdd(T *p, U v)
{
    const T old = *p;
    *p = old + v;
    return old;
}
template <class T, class U>
static inline T atomicSub(T *p, U v)
{
    return atomicAdd(p, -v);
}
template <class T, class U>
static inline T atomicMin(T *p, U v)
{
    const T old = *p;
    *p = std::min<T>(old, v);
    return old;
}

namespace wushkv {

using std::max;
using std::min;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
constexpr int kPage = WUSHKV_PAGE_TOKENS;

// (called by every thread of a workgroup)
static inline int32_t wave_scan(int32_t x)
{
    static int32_t of[1024];
    const unsigned t = threadIdx.x;
    of[t] = x;
    __syncthreads();
    int32_t sum = 0;
    for (unsigned i = t & ~63u; i <= t; ++i) sum += of[i];
    __syncthreads();
    return sum;
}

template <class Args>
static void launch(const char *, void (*kernel)(Args), dim3 grid, dim3 block, hipStream_t, const Args &args)
{
    struct Call {
        void (*kernel)(Args);
        const Args *args;
    } call{kernel, &args};
    gridDim = grid;
    blockDim = block;
    host::body = [](void *p) { static_cast<Call *>(p)->kernel(*static_cast<Call *>(p)->args); };
    host::body_args = &call;
    std::vector<unsigned> groups(grid.x);
    std::iota(groups.begin(), groups.end(), 0u);
    if (host::order == 1) std::reverse(groups.begin(), groups.end());
    if (host::order > 1) std::shuffle(groups.begin(), groups.end(), std::mt19937(host::order));
    for (unsigned g : groups) {
        blockIdx = dim3(g, 0, 0);
        host::run_workgroup(block.x);
    }
}

}  // namespace wushkv

// what the page operators take from csrc/api.hip
int wushkv_validate_cache(const wushkv_cache *c) { return c != nullptr ? WUSHKV_OK : WUSHKV_EINVAL; }
extern "C" size_t wushkv_page_bytes(int32_t head_dim, int32_t bits)
{
    return (size_t)WUSHKV_PAGE_TOKENS * (2 * head_dim * (bits == 3 ? 4 : bits) / 8 + 8);
}
extern "C" void host_order(int order) { host::order = order; }
