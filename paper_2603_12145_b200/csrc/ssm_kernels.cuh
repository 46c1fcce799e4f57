// ssm_kernels.cuh -- argument blocks and launchers of the kernels behind ssm.h.
#pragma once

#include "ssm_common.cuh"

namespace ssm_k {

// ---- kernels of one call that follow one another
//
// Every kernel begins with allow_next() and wait_for_previous(); those behind the first are launched by
// launch_after(): their blocks are placed while the kernel before them still runs and wait there for its results,
// which hides the launch.  Every block waits, so that kernels end in the order of the stream.

__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... Params, typename... Args>
bool launch_after(cudaStream_t stream, dim3 grid, unsigned threads, size_t smem, void (*kernel)(Params...), Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess;
}

// Sizes of a scan and how its work is cut.
struct ScanShape {
    int64_t batch;
    int time;
    int channels, states, groups;
    int group_channels;        // channels / groups
    int quads;                 // recurrent states of a channel in groups of four, as `saved` holds them
    int chunks;                // ceil(time / kScanChunk)
    int segments;              // pieces of the time axis worked on side by side
    int segment_steps;         // multiple of kScanChunk
    int slots;                 // blocks along the rows (backward): each takes several and keeps its sums
};

// Steps between saved states: the backward kernel keeps a chunk's intermediate states on the SM.
// With 16 states and a 16-bit type the saved states are as much memory as two of the sequences.
constexpr int kScanChunk = 16;

// Channels (and threads) of a block of the backward kernel.  Beyond 16 states shared memory limits the blocks: with 32, two
// of three warps fit on an SM and only one of four (3 x 777 x 330 x 24 states: 69 against 100 us).
__host__ __device__ constexpr int scan_back_channels(int states) { return states > 16 && states <= 32 ? 96 : 128; }

// Segments whose ends the joining kernels load together.
constexpr int kAhead = 8;

struct ScanParams {
    const float *a, *d, *dt_bias;
    const float *state;
    float *state_out;
    float *saved;
    float *carry;              // [batch][segments][quads][channels][4]: a segment's end, then its start
    float *span;               // [batch][segments][channels]: sum of delta, negative where a reset cuts the segment
    const float *dstate_out;
    float *dstate;
    float *da_part;            // [slots][quads][channels][4]
    float *dd_part;            // [slots][2][channels]: dd, ddt_bias
    float *dbc_part;           // [group tiles][batch][time][groups][2][16 * state blocks]
    float *da, *dd, *ddt_bias;
};

template <typename T>
struct ScanSeqs {
    Seq<const T> x, dt, z, b, c, dy;
    Seq<const uint8_t> reset;
    Seq<T> y, dx, ddt, dz, db, dc;
};

// Each returns the number of kernels launched, or -1 on a launch error.
template <typename T>
int launch_scan_forward(const ScanShape &s, const ScanParams &p, const ScanSeqs<T> &q, cudaStream_t stream);
template <typename T>
int launch_scan_backward(const ScanShape &s, const ScanParams &p, const ScanSeqs<T> &q, cudaStream_t stream);

struct StepParams {
    const float *a, *d, *dt_bias, *state;
    float *state_out;
    const uint8_t *done;
    int64_t x_stride, dt_stride, z_stride, b_stride, c_stride, y_stride, done_stride;
    int64_t n;
    int channels, states, group_channels;
    int sms;
};
template <typename T>
int launch_scan_step(const StepParams &p, const T *x, const T *dt, const T *z, const T *b, const T *c, T *y,
                     cudaStream_t stream);

struct ConvShape {
    int64_t batch;
    int time, channels, width;
    int run;                   // steps per unit of work
    int runs;                  // ceil(time / run)
    int slots;                 // blocks along the units (backward)
    int sms;
};
struct ConvParams {
    const float *w, *bias;
    float *dw, *dbias;
    float *part;               // [slots][width + 1][channels]
};
template <typename T>
struct ConvSeqs {
    Seq<const T> x, dy;
    Seq<const uint8_t> reset;
    Seq<T> y, dx;
    const T *history;
    T *history_out;
};
template <typename T>
int launch_conv_forward(const ConvShape &s, const ConvParams &p, const ConvSeqs<T> &q, cudaStream_t stream);
template <typename T>
int launch_conv_backward(const ConvShape &s, const ConvParams &p, const ConvSeqs<T> &q, cudaStream_t stream);
template <typename T>
int launch_conv_step(const ConvShape &s, const ConvParams &p, const T *x, int64_t x_stride, const uint8_t *done,
                     int64_t done_stride, const T *history, T *history_out, T *y, int64_t y_stride,
                     cudaStream_t stream);

}  // namespace ssm_k
