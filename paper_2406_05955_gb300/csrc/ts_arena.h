// ts_arena.h -- a handle's device scratch: one allocation with a guard zone behind every block of it.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>

#include <vector>

#include "ts_ffn.h"

namespace tsffn {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

// A handle's device scratch: blocks carved out of one allocation. Every block
// is followed by a guard zone of kGuardBytes filled with kGuardByte when the
// arena is allocated; check_arena reads the zones back, so a kernel that
// writes past the end of a scratch block is caught by the tests instead of
// silently corrupting the next block.
constexpr size_t kGuardBytes = kAlign;
constexpr unsigned char kGuardByte = 0xA5;

struct Arena {
    size_t bytes = 0;
    char* base = nullptr;
    std::vector<size_t> guards;  // offsets of the guard zones
    size_t take(size_t n) {
        const size_t off = bytes;
        bytes += align_up(n);
        guards.push_back(bytes);
        bytes += kGuardBytes;
        return off;
    }
    template <typename P>
    P* at(size_t off) const { return reinterpret_cast<P*>(base + off); }
};

inline ts_status alloc_arena(Arena* ar) {
    if (cudaMalloc(&ar->base, ar->bytes) != cudaSuccess) {
        cudaGetLastError();
        ar->base = nullptr;
        return TS_ERR_OOM;
    }
    bool ok = cudaMemset(ar->base, 0, ar->bytes) == cudaSuccess;
    for (size_t g : ar->guards) ok = ok && cudaMemset(ar->base + g, kGuardByte, kGuardBytes) == cudaSuccess;
    if (!ok) {
        cudaFree(ar->base);
        ar->base = nullptr;
        return TS_ERR_CUDA;
    }
    return TS_OK;
}

// Handles are also destroyed while some stream is being captured (a garbage collector picks its time): what is freed
// under this, which no captured work depends on, does not end that capture.
class WhileCapturing {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    bool relaxed = cudaThreadExchangeStreamCaptureMode(&mode) == cudaSuccess;

public:
    WhileCapturing() = default;
    WhileCapturing(const WhileCapturing&) = delete;
    ~WhileCapturing() {
        if (relaxed) cudaThreadExchangeStreamCaptureMode(&mode);
    }
};
inline void free_arena(Arena* ar) {
    if (!ar->base) return;
    const WhileCapturing may_free;
    cudaFree(ar->base);
    ar->base = nullptr;
}

// Synchronise `stream` and compare every guard zone with its fill.
inline ts_status check_arena(const Arena& ar, cudaStream_t stream) {
    if (!ar.base) return TS_ERR_INVALID_ARG;
    if (cudaStreamSynchronize(stream) != cudaSuccess) return TS_ERR_CUDA;
    std::vector<unsigned char> buf(kGuardBytes);
    for (size_t g : ar.guards) {
        if (cudaMemcpy(buf.data(), ar.base + g, kGuardBytes, cudaMemcpyDeviceToHost) != cudaSuccess)
            return TS_ERR_CUDA;
        for (unsigned char b : buf)
            if (b != kGuardByte) return TS_ERR_SCRATCH;
    }
    return TS_OK;
}

}  // namespace tsffn
