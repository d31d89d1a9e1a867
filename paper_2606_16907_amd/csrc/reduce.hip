// reduce.hip -- sums over the rows of a table of 32-bit partial sums: the last
// step of the gradients that add over a batch's rows (weights of a norm, biases).
#include <utility>

#include "layer_device.h"

namespace tg {
namespace {

// Row 1 of blocks, where there is one, does the second table.
template <typename T>
__global__ __launch_bounds__(256) void column_sums(const float *__restrict__ partial, int rows, int64_t cols, int64_t first, T *out, T *out2) {
    if (blockIdx.y) partial += rows * cols, out = out2;
    column_sums_block(partial, rows, cols, first + (int64_t)blockIdx.x * 32, out);
}

constexpr int64_t kMostColumns = 1 << 25;  // of a launch: a grid holds fewer than 2^32 threads, 8 a column and table

template <typename T>
void launch(const float *partial, int rows, int64_t cols, void *out, void *out2, hipStream_t s) {
    for (int64_t first = 0; first < cols; first += kMostColumns) {
        const int64_t n = cols - first < kMostColumns ? cols - first : kMostColumns;
        hipLaunchKernelGGL(column_sums<T>, dim3((unsigned)ceil_div(n, 32), out2 ? 2 : 1), dim3(256), 0, s, partial, rows, cols, first, (T *)out, (T *)out2);
    }
}

}  // namespace

hipError_t launch_column_sums_of_two(const float *partial, int rows, int64_t cols, void *out, void *out2, int type, hipStream_t s) {
    if (!out) partial += rows * cols, std::swap(out, out2);
    if (!out) return hipSuccess;
    if (type == TG_F32)
        launch<float>(partial, rows, cols, out, out2, s);
    else if (type == TG_BF16)
        launch<bf16>(partial, rows, cols, out, out2, s);
    else
        launch<f16>(partial, rows, cols, out, out2, s);
    return hipGetLastError();
}

hipError_t launch_column_sums(const float *partial, int rows, int64_t cols, void *out, int type, hipStream_t s) {
    return launch_column_sums_of_two(partial, rows, cols, out, nullptr, type, s);
}

}  // namespace tg
