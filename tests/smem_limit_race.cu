// Host program: two threads use one kernel for the first time with different amounts of shared memory, in the order in which
// a table of what has been set and the runtime's attribute come apart.  set_attribute stands in for the runtime's call and,
// like it, keeps the value of the last one.  Prints the attribute, and what a third call that needs the larger one is told.
#include <cuda_runtime.h>

template <typename K>
cudaError_t set_attribute(K kernel, cudaFuncAttribute, int value);
#define cudaFuncSetAttribute set_attribute
#include "../paper_2401_09135_b200/csrc/alsgd_ops.cuh"
#undef cudaFuncSetAttribute

#include <chrono>
#include <condition_variable>
#include <cstdio>
#include <mutex>
#include <thread>

namespace {
std::mutex m;
std::condition_variable cv;
int attribute = 0, entered = 0;
bool second_done = false;
constexpr int kMore = 140 * 1024, kLess = 110 * 1024;
void kernel() {}
}  // namespace

template <typename K>
cudaError_t set_attribute(K, cudaFuncAttribute, int value) {
    std::unique_lock<std::mutex> lock(m);
    attribute = value;
    if (++entered == 1) {
        cv.notify_all();
        cv.wait_for(lock, std::chrono::milliseconds(500), [] { return second_done; });     // the first call returns last
    }
    return cudaSuccess;
}

int main() {
    static alsgd_ops::SmemLimit limit;
    std::thread first([] { limit.raise(kernel, 0, kMore); });
    std::thread second([] {
        {
            std::unique_lock<std::mutex> lock(m);
            cv.wait(lock, [] { return entered > 0; });
        }
        limit.raise(kernel, 0, kLess);
        std::lock_guard<std::mutex> lock(m);
        second_done = true;
        cv.notify_all();
    });
    first.join();
    second.join();
    const bool ok = limit.raise(kernel, 0, kMore);
    std::printf("%d %d %d\n", ok, attribute, kMore);
    const bool too_much = limit.raise(kernel, 0, 256 * 1024);
    std::printf("%d\n", too_much);
    return 0;
}
