// reduce.hip -- sums over the rows of a table of 32-bit partial sums: the last
// step of the gradients that add over a batch's rows (weights of a norm, biases).
#include <utility>

#include "layer_device.h"

namespace tg {
namespace {

// Adding up in place of float atomics keeps the order, and so the result, the
// same every time.  A block has 32 columns by 8 strands; strand g adds rows
// g, g + 8, ..., then the strands are added in order.
// Row 1 of blocks, where there is one, does the second table.
template <typename T>
__global__ __launch_bounds__(256) void column_sums(const float *__restrict__ partial, int rows, int64_t cols, int64_t first, T *out, T *out2) {
    if (blockIdx.y) partial += rows * cols, out = out2;
    __shared__ float strand[8][33];
    const int lane = threadIdx.x % 32, g = threadIdx.x / 32;
    const int64_t col = first + (int64_t)blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (col < cols) {
#pragma unroll 8
        for (int r = g; r < rows; r += 8) sum += partial[r * cols + col];
    }
    strand[g][lane] = sum;
    __syncthreads();
    if (g == 0 && col < cols) {
#pragma unroll
        for (int h = 1; h < 8; ++h) sum += strand[h][lane];
        out[col] = (T)sum;
    }
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
