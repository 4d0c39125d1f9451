// The token cache's kernels as host code: a lane is a thread, and what lanes do together (shuffles, barriers) is a rendezvous
// of theirs.  The wavefronts of a workgroup run one behind the other between two barriers, in an order that the caller
// chooses, so that what one does before the others have read is seen every time and not by chance.  "cache.inc" is the device
// sources' own text, put together by the test that builds this; its calls take host memory.
#include <algorithm>
#include <atomic>
#include <barrier>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <memory>
#include <thread>
#include <vector>

#define __device__
#define __global__
#define __shared__ static
#define __launch_bounds__(...)

struct dim3 {
    uint32_t x, y;
    dim3(uint32_t a, uint32_t b = 1) : x(a), y(b) {}
};
typedef int hipError_t;
typedef void *hipStream_t;
constexpr hipError_t hipSuccess = 0;
constexpr int hipDeviceAttributeMultiprocessorCount = 1;
inline hipError_t hipGetLastError() { return hipSuccess; }
inline hipError_t hipGetDevice(int *device) { return *device = 0, hipSuccess; }
inline hipError_t hipDeviceGetAttribute(int *value, int, int) { return *value = 256, hipSuccess; }

namespace {

thread_local struct { uint32_t x; } threadIdx;
thread_local dim3 blockIdx(0, 0);
dim3 gridDim(0, 0);
std::vector<uint64_t> launches;                  // lanes along x, workgroups along x and y of every launch
bool only_noted;                                 // launches are noted, nothing runs

constexpr uint32_t kMostWaves = 16;
uint32_t waves, first_wave;
std::unique_ptr<std::barrier<>> wave_meets[kMostWaves];
uint64_t said[kMostWaves * 64];                  // what every lane brings to a shuffle
std::atomic<uint32_t> turn;                      // the wavefront that runs: their place in the order, counted on from segment to segment
std::atomic<int> any;
thread_local uint32_t segment;

uint32_t wave_of() { return threadIdx.x / 64; }
uint32_t place() { return (wave_of() + waves - first_wave) % waves; }
void wave_meet() { wave_meets[wave_of()]->arrive_and_wait(); }

void wait_for_turn() {
    const uint32_t mine = segment * waves + place();
    for (uint32_t now = turn; now != mine; now = turn) turn.wait(now);
}

void end_turn() {
    wave_meet();
    if (threadIdx.x % 64 == 0) {
        ++turn;
        turn.notify_all();
    }
    ++segment;
}

void __syncthreads() {
    end_turn();
    wait_for_turn();
}

int __syncthreads_or(int x) {
    if (x) any = 1;
    __syncthreads();
    const int r = any;
    __syncthreads();
    any = 0;
    __syncthreads();
    return r;
}

void __threadfence_block() {}

int shuffle(int v, uint32_t from) {
    said[threadIdx.x] = static_cast<uint32_t>(v);
    wave_meet();
    const int r = static_cast<int>(said[wave_of() * 64 + (from & 63u)]);
    wave_meet();
    return r;
}

int __shfl_xor(int v, int o) { return shuffle(v, (threadIdx.x & 63u) ^ static_cast<uint32_t>(o)); }
int __shfl_up(int v, int d) { return shuffle(v, (threadIdx.x & 63u) >= static_cast<uint32_t>(d) ? (threadIdx.x & 63u) - d : threadIdx.x & 63u); }

int atomicMin(int32_t *p, int32_t v) {
    int32_t was = __atomic_load_n(p, __ATOMIC_RELAXED);
    while (v < was && !__atomic_compare_exchange_n(p, &was, v, true, __ATOMIC_RELAXED, __ATOMIC_RELAXED)) {}
    return was;
}

template <typename T> T min(T a, T b) { return b < a ? b : a; }
template <typename T> T max(T a, T b) { return a < b ? b : a; }
float __uint_as_float(uint32_t u) { return __builtin_bit_cast(float, u); }
uint32_t __float_as_uint(float f) { return __builtin_bit_cast(uint32_t, f); }

// D's bytes by the selectors' bytes: 0-3 of b, 4-7 of a, 12 zero
uint32_t perm(uint32_t a, uint32_t b, uint32_t select) {
    const uint64_t both = uint64_t{a} << 32 | b;
    uint32_t r = 0;
    for (int i = 0; i < 4; ++i) {
        const uint32_t s = select >> (8 * i) & 0xffu;
        r |= (s == 12 ? 0u : static_cast<uint32_t>(both >> (8 * s)) & 0xffu) << (8 * i);
    }
    return r;
}

#define __builtin_amdgcn_perm perm
#define __builtin_amdgcn_wave_barrier wave_meet

template <typename F>
void host_launch(dim3 grid, dim3 block, F kernel) {
    launches.insert(launches.end(), {uint64_t{grid.x} * block.x, grid.x, grid.y});
    if (only_noted) return;
    gridDim = grid;
    waves = block.x / 64;
    for (uint32_t i = 0; i < waves; ++i) wave_meets[i] = std::make_unique<std::barrier<>>(64);
    for (uint32_t y = 0; y < grid.y; ++y)
        for (uint32_t x = 0; x < grid.x; ++x) {
            turn = 0;
            std::vector<std::thread> lanes;
            for (uint32_t l = 0; l < block.x; ++l)
                lanes.emplace_back([&, l] {
                    threadIdx.x = l;
                    blockIdx = dim3(x, y);
                    segment = 0;
                    wait_for_turn();
                    kernel();
                    end_turn();
                });
            for (std::thread &lane : lanes) lane.join();
        }
}

// Attention's matrix instructions have no host form: its launches are only noted.
template <int W, typename T, typename... A> void k_attend_few(const A &...) {}
template <int W, typename T, typename... A> void k_attend_many(const A &...) {}
template <int W, typename T, typename... A> void k_attend_join(const A &...) {}
template <int W, typename T, typename... A> void k_attend_join_rows(const A &...) {}

}  // namespace

#define hipLaunchKernelGGL(kernel, grid, block, lds, stream, ...) host_launch(grid, block, [&] { kernel(__VA_ARGS__); })

#include "cache.inc"

void entro_detail_note_hip_error(const char *, int) {}

// The wavefront that runs first from here on.
extern "C" void host_first_wave(uint32_t wave) { first_wave = wave; }

// From here on launches are only noted.
extern "C" void host_only_note(int yes) { only_noted = yes != 0; }

// Lanes along x, workgroups along x and y of the launches since the last time, `most` numbers at most; returns how many.
extern "C" int host_launches(uint64_t *out, int most) {
    const int n = std::min(most, static_cast<int>(launches.size()));
    std::copy_n(launches.begin(), n, out);
    launches.clear();
    return n;
}
