// The model operators' C entries over stand-ins for CUDA and for their kernels: what reaches a
// launch, and who waits for whom, without a GPU.  The planner's stand-ins serve here too, but
// cudaEventSynchronize can be made to wait, as it does for an upload slot that is still in use.
#include <atomic>
#include <chrono>
#include <thread>

#include <cuda.h>
#include <cuda_runtime.h>

#define cudaEventSynchronize planner_event_synchronize
#include "planner_fake.cpp"
#undef cudaEventSynchronize

#include "kvs_ops.h"

namespace {
std::atomic<int> g_hold{0}, g_held{0}, g_ops{0};
}  // namespace

extern "C" {
// While held, an event is not reached (for ten seconds at most).
void fake_hold(int on) { g_hold = on; }
int fake_held() { return g_held; }
int fake_ops() { return g_ops; }

cudaError_t cudaEventSynchronize(cudaEvent_t) {
    ++g_held;
    for (int k = 0; g_hold && k < 10000; ++k) std::this_thread::sleep_for(std::chrono::milliseconds(1));
    --g_held;
    return cudaSuccess;
}
}

namespace kvs {
void set_divisors(StepView&) {}
AttendPlan attend_plan(const StepView&, int) { return AttendPlan{0, 1, 1, 0}; }
int launch_append(const AppendJob&, bool, cudaStream_t) { return ++g_ops, 1; }
int launch_attend(const AttendJob&, bool, cudaStream_t) { return ++g_ops, 1; }
int launch_weigh(const WeighJob&, bool, int, cudaStream_t) { return ++g_ops, 1; }
int launch_evict(const EvictJob&, cudaStream_t) { return ++g_ops, 1; }
}  // namespace kvs
