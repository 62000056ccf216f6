// Host helpers of the training operators.
#include "a2sgd_train.cuh"

#include <map>
#include <mutex>
#include <thread>
#include <tuple>
#include <utility>

namespace a2sgd_train {

int sm_count(int device)
{
    static std::mutex lock;
    static std::map<int, int> known_counts;
    std::lock_guard<std::mutex> hold(lock);
    auto it = known_counts.find(device);
    if (it != known_counts.end()) return it->second;
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
        (void)cudaGetLastError();
        return 0;
    }
    try {
        known_counts[device] = n;
    } catch (...) { // no memory for the note: ask again next time
    }
    return n;
}

int resident_ctas(const void *fn, unsigned threads, size_t smem, int device)
{
    static std::mutex lock;
    static std::map<std::tuple<const void *, int, unsigned, size_t>, int> known_counts;
    std::lock_guard<std::mutex> hold(lock);
    const auto key = std::make_tuple(fn, device, threads, smem);
    auto it = known_counts.find(key);
    if (it != known_counts.end()) return it->second;
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, fn, (int)threads, smem) != cudaSuccess) {
        (void)cudaGetLastError();
        return 1;
    }
    n = n > 0 ? n : 1;
    try {
        known_counts[key] = n;
    } catch (...) { // as above
    }
    return n;
}

cudaError_t allow_smem(const void *fn, size_t bytes)
{
    static std::mutex lock;
    static std::map<std::pair<const void *, int>, size_t> allowed;
    int device = 0;
    const cudaError_t err = cudaGetDevice(&device);
    if (err != cudaSuccess) return err;
    std::lock_guard<std::mutex> hold(lock);
    const auto key = std::make_pair(fn, device);
    const auto it = allowed.find(key);
    if (it != allowed.end() && it->second >= bytes) return cudaSuccess;
    const cudaError_t set = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (set != cudaSuccess) return set;
    try {
        allowed[key] = bytes;
    } catch (...) { // no memory for the note: set again next time
    }
    return cudaSuccess;
}

bool count_moved(int device, cudaStream_t stream, unsigned int count, const void *counter)
{
    static std::mutex lock;
    static std::map<std::tuple<const void *, int, cudaStream_t, std::thread::id>, unsigned int> seen;
    if (count == 0) return false;
    const std::thread::id thread = stream == cudaStreamPerThread ? std::this_thread::get_id() : std::thread::id();
    std::lock_guard<std::mutex> hold(lock);
    const auto key = std::make_tuple(counter, device, stream, thread);
    const auto it = seen.find(key);
    if (it != seen.end() && it->second == count) return false;
    try {
        seen[key] = count;
    } catch (...) { // no memory for the note: told again next time
    }
    return true;
}

} // namespace a2sgd_train
