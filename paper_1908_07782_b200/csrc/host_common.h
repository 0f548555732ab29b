// What the translation units of libcombo_b200.so share on the host side.  Defined in combo_b200.cu.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/combo_b200.h"

namespace combo_host {

#pragma GCC visibility push(hidden)
// Records a failed CUDA call for combo_last_cuda_error() and returns COMBO_ERR_CUDA.
combo_status fail(cudaError_t e, const char* what);
// The current device's SM count and largest shared memory of a block; COMBO_ERR_UNSUPPORTED unless it is 10.x.
combo_status device(int* sms, int* smem_optin);
// What combo_last_step_path() answers on this thread.
enum StepPath { kPathNone = 0, kPathMultiplyAdd = 1, kPathTensor = 2, kPathTensorPairs = 3, kPathTensorThreads = 4, kPathResident = 5, kPathStreamed = 6 };
void set_step_path(StepPath path);
// Status word of the grouped products' kernels (see combo_device_status): reads it, and clears it if it is set.
cudaError_t grouped_linear_status(int* code);
// The same of the cross entropy's kernels.
cudaError_t cross_entropy_status(int* code);
// cuTensorMapEncodeTiled without interleaving, out-of-bounds elements read as zero; false (and a text for
// combo_last_cuda_error()) if it is missing or refuses.
bool encode_tiled(CUtensorMap* map, CUtensorMapDataType type, int rank, void* base, const cuuint64_t* dims, const cuuint64_t* strides,
                  const cuuint32_t* box, const cuuint32_t* elem_strides, CUtensorMapSwizzle swizzle);
#pragma GCC visibility pop

inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// Whether [a, a + na) and [b, b + nb) share a byte.
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return na && nb && x < y + nb && y < x + na;
}

// Rows of `width` bytes, `pitch` apart, and whether two such arrays share a byte.  Views of one wider array (equal pitches) lie
// beside each other where their columns do; other arrays are taken to share what their extents share.
struct Rows {
    const void* p;
    int64_t n;
    size_t width, pitch;
    size_t extent() const { return n < 1 ? 0 : (size_t)(n - 1) * pitch + width; }
};
inline bool overlap(const Rows& a, const Rows& b) {
    if (!overlap(a.p, a.extent(), b.p, b.extent())) return false;
    const size_t pitch = a.n > 1 ? a.pitch : b.pitch;
    if (b.n > 1 && b.pitch != pitch) return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    const size_t off = y >= x ? (y - x) % pitch : (pitch - (x - y) % pitch) % pitch;      // of b's columns behind the start of a's
    return off < a.width || off + b.width > pitch;
}

// Lets `kern` use up to `bytes` of dynamic shared memory, once per kernel and device: `done` is the kernel's own word
// of device bits (asking the driver costs as much as a launch).
template <typename K> inline cudaError_t allow_smem(K kern, int bytes, uint64_t* done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (__atomic_load_n(done, __ATOMIC_RELAXED) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) __atomic_fetch_or(done, bit, __ATOMIC_RELAXED);
    return e;
}

// Launches `kern` so that it may become resident while the stream's preceding kernel drains; the kernel
// itself waits for that one (pdl_wait) before it touches anything that one writes.
template <typename... P, typename... A>
inline cudaError_t launch_after(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, static_cast<P>(args)...);
}

}  // namespace combo_host
