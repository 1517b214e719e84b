// A kernel's own source on the host: every lane of a workgroup is a fiber, lanes of a wave meet where they exchange values, all of them at barriers, and workgroups
// run one after the other.  So memory that a kernel reads and writes meets the sanitizers of the host before it meets a GPU.  Matrix products give their last operand
// back: what is computed is not looked at.
#pragma once

#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <map>
#include <vector>

#define __device__
#define __host__
#define __global__
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __shared__ static
#define __align__(n) __attribute__((aligned(n)))

struct dim3 {
    uint32_t x, y, z;
    dim3(uint32_t a = 1, uint32_t b = 1, uint32_t c = 1) : x(a), y(b), z(c) {}
};
typedef void* hipStream_t;
typedef int hipError_t;
constexpr int hipSuccess = 0;
inline int hipGetLastError() { return 0; }
inline const char* hipGetErrorString(int) { return ""; }

namespace lanes {

// Keeps the own stack pointer at `keep` and goes on where `to` was kept.
extern "C" void lanes_switch(void** keep, void* to);
asm(R"(
.text
.weak lanes_switch
lanes_switch:
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

constexpr size_t kStack = 256 * 1024;
struct Lane {
    void* at = nullptr;
    char* stack = nullptr;
    dim3 tid;
    bool done = true;
};
struct Wave {
    uint64_t slot[2][64] = {};
    int arrived = 0, alive = 0;
    uint64_t turn = 0;
};
inline std::vector<Lane> all;
inline std::vector<Wave> waves;
inline Lane* cur = nullptr;
inline void* scheduler = nullptr;
inline dim3 block_index, block_dim, grid_dim;
inline int at_barrier = 0, alive = 0;
inline uint64_t barrier_turn = 0;
inline std::function<void()> body;

inline int index() { return (int)(cur - all.data()); }
inline void yield() { lanes_switch(&cur->at, scheduler); }
inline void begin() {
    body();
    cur->done = true;
    --alive;
    --waves[index() / 64].alive;
    for (;;) yield();
}
inline void run_block(int threads, std::function<void()> f) {
    if ((int)all.size() < threads) all.resize(threads);
    waves.assign((threads + 63) / 64, Wave{});
    body = f;
    at_barrier = 0;
    alive = threads;
    block_dim = dim3((uint32_t)threads);
    for (int i = 0; i < threads; ++i) {
        Lane& l = all[i];
        if (!l.stack) l.stack = static_cast<char*>(std::aligned_alloc(16, kStack));
        l.done = false;
        l.tid = dim3((uint32_t)i, 0, 0);
        ++waves[i / 64].alive;
        // what lanes_switch takes off the stack: six registers and where to go; then the stack is as behind a call
        void** top = reinterpret_cast<void**>(l.stack + kStack) - 1;
        *--top = reinterpret_cast<void*>(&begin);
        for (int r = 0; r < 6; ++r) *--top = nullptr;
        l.at = top;
    }
    while (alive > 0)
        for (int i = 0; i < threads; ++i) {
            cur = &all[i];
            if (!cur->done) lanes_switch(&scheduler, cur->at);
        }
}
// The values of all lanes of the wave that have not ended: they all take part.
inline const uint64_t* exchange(uint64_t v) {
    const int i = index();
    Wave& w = waves[i / 64];
    const uint64_t turn = w.turn;
    uint64_t* const s = w.slot[turn & 1];
    s[i % 64] = v;
    ++w.arrived;
    while (w.turn == turn) {
        if (w.arrived >= w.alive) {
            w.arrived = 0;
            ++w.turn;
        } else {
            yield();
        }
    }
    return s;
}
inline void barrier() {
    const uint64_t turn = barrier_turn;
    ++at_barrier;
    while (barrier_turn == turn) {
        if (at_barrier >= alive) {
            at_barrier = 0;
            ++barrier_turn;
        } else {
            yield();
        }
    }
}
template <typename T>
uint64_t bits(T v) {
    uint64_t b = 0;
    std::memcpy(&b, &v, sizeof v);
    return b;
}
template <typename T>
T value(uint64_t b) {
    T v;
    std::memcpy(&v, &b, sizeof v);
    return v;
}

// Kernels that a launch by their address runs.
inline std::map<const void*, std::function<void(void**)>> kernels;
template <typename A>
void runs(void (*kernel)(A)) {
    kernels[reinterpret_cast<const void*>(kernel)] = [kernel](void** list) { kernel(*static_cast<A*>(list[0])); };
}
template <typename A, typename B>
void runs(void (*kernel)(A, B)) {
    kernels[reinterpret_cast<const void*>(kernel)] = [kernel](void** list) { kernel(*static_cast<A*>(list[0]), *static_cast<B*>(list[1])); };
}

}  // namespace lanes

inline int hipLaunchKernel(const void* kernel, dim3 grid, dim3 block, void** list, size_t, hipStream_t) {
    const auto found = lanes::kernels.find(kernel);
    if (found == lanes::kernels.end()) std::abort();
    lanes::grid_dim = grid;
    for (uint32_t y = 0; y < grid.y; ++y)
        for (uint32_t x = 0; x < grid.x; ++x) {
            lanes::block_index = dim3(x, y);
            lanes::run_block((int)block.x, [&] { found->second(list); });
        }
    return 0;
}

#define threadIdx (lanes::cur->tid)
#define blockIdx (lanes::block_index)
#define blockDim (lanes::block_dim)
#define gridDim (lanes::grid_dim)

inline int __lane_id() { return lanes::index() % 64; }
inline void __syncthreads() { lanes::barrier(); }
template <typename T>
T __shfl(T v, int lane, int = 64) { return lanes::value<T>(lanes::exchange(lanes::bits(v))[lane & 63]); }
template <typename T>
T __shfl_xor(T v, int m, int = 64) {
    const int i = __lane_id();
    return lanes::value<T>(lanes::exchange(lanes::bits(v))[(i ^ m) & 63]);
}
template <typename T>
T __shfl_up(T v, int m, int = 64) {
    const int i = __lane_id();
    return lanes::value<T>(lanes::exchange(lanes::bits(v))[i >= m ? i - m : i]);
}
inline uint64_t __ballot(bool b) {
    const int first = lanes::index() / 64 * 64;
    const uint64_t* const s = lanes::exchange(b);
    uint64_t r = 0;
    for (int i = 0; i < 64 && first + i < (int)lanes::block_dim.x; ++i) r |= (uint64_t)(s[i] & 1) << i;
    return r;
}
inline bool __any(bool b) { return __ballot(b) != 0; }
inline int __builtin_amdgcn_readfirstlane(int v) { return lanes::value<int>(lanes::exchange(lanes::bits(v))[0]); }
inline int __builtin_amdgcn_readlane(int v, int lane) { return lanes::value<int>(lanes::exchange(lanes::bits(v))[lane]); }
typedef uint32_t swapped_pair __attribute__((ext_vector_type(2)));
// The odd sets of n lanes of a exchanged with the even ones of b.
inline swapped_pair swap_rows(uint32_t a, uint32_t b, int n) {
    const int i = __lane_id();
    const uint64_t* const s = lanes::exchange((uint64_t)a | (uint64_t)b << 32);
    return (i & n) ? swapped_pair{(uint32_t)(s[i ^ n] >> 32), b} : swapped_pair{a, (uint32_t)s[i ^ n]};
}
#define __builtin_amdgcn_permlane32_swap(a, b, ...) swap_rows(a, b, 32)
#define __builtin_amdgcn_permlane16_swap(a, b, ...) swap_rows(a, b, 16)
inline int __builtin_amdgcn_update_dpp(int, int, int, int, int, bool) { std::abort(); }  // no kernel that runs here takes one
inline float __builtin_amdgcn_exp2f(float x) { return exp2f(x); }
inline float __builtin_amdgcn_logf(float x) { return log2f(x); }
inline float __builtin_amdgcn_rcpf(float x) { return 1.0f / x; }
inline float __builtin_amdgcn_fmed3f(float a, float b, float c) { return fmaxf(fminf(a, b), fminf(fmaxf(a, b), c)); }
inline uint32_t __builtin_amdgcn_perm(uint32_t hi, uint32_t lo, uint32_t select) {
    const uint64_t x = (uint64_t)hi << 32 | lo;
    uint32_t r = 0;
    for (int i = 0; i < 4; ++i) r |= (uint32_t)(x >> (8 * (select >> (8 * i) & 7)) & 255) << (8 * i);
    return r;
}
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, ...) (c)
#define __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, ...) (c)
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, ...) (c)
inline uint32_t __float_as_uint(float f) { return lanes::value<uint32_t>(lanes::bits(f)); }
inline int __float_as_int(float f) { return lanes::value<int>(lanes::bits(f)); }
inline int __popcll(uint64_t x) { return __builtin_popcountll(x); }
inline float __uint_as_float(uint32_t u) { return lanes::value<float>(u); }
inline float __int_as_float(int u) { return lanes::value<float>((uint32_t)u); }
inline uint32_t __umulhi(uint32_t a, uint32_t b) { return (uint32_t)((uint64_t)a * b >> 32); }
inline int __double2loint(double d) { return (int)lanes::bits(d); }
inline int __double2hiint(double d) { return (int)(lanes::bits(d) >> 32); }
inline double __hiloint2double(int hi, int lo) { return lanes::value<double>((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo); }
inline float __fmul_rn(float a, float b) { return a * b; }
inline float __fdiv_rn(float a, float b) { return a / b; }
template <typename T>
T min(T a, T b) { return b < a ? b : a; }
template <typename T>
T max(T a, T b) { return a < b ? b : a; }
