// ssm_api.cu -- the C ABI of ssm.h: checks, workspaces, launches.
#include <new>

#include "on_device.cuh"
#include "ssm_kernels.cuh"

using namespace ssm_k;

struct ssm {
    int channels = 0, states = 0, groups = 0, width = 0, type = 0;
    int device = 0, sms = 0;
    cudaStream_t stream = nullptr;
    int64_t launches = 0;
};

namespace {

constexpr int64_t kMaxBlocks = 0x7FFFFFFF;

size_t align16(size_t v) { return (v + 15) & ~static_cast<size_t>(15); }

int element_bytes(const ssm *p) { return p->type == SSM_F32 ? 4 : 2; }

bool aligned(const void *ptr, size_t bytes) { return reinterpret_cast<uintptr_t>(ptr) % bytes == 0; }

int quads_of(int states)
{
    int n = 4;
    while (n < states) n *= 2;
    return n / 4;
}

// Lanes per channel of the kernels that keep a channel's states in registers (16 per lane at most).
int lanes_of(int states) { return states <= 16 ? 1 : states <= 32 ? 2 : 4; }

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool sizes_ok(int64_t batch, int64_t time)
{
    return batch >= 1 && time >= 1 && batch <= kMaxBlocks && time <= kMaxBlocks / 2;
}

// The cut of the time axis.  One segment costs one pass over its steps, several cost two, so the cut pays
// where the rows alone occupy less than half of the `resident` blocks that the device holds.  The
// segments then fill one or a few whole rounds of resident blocks, whichever is the shortest.
void cut_time(ScanShape &s, int64_t blocks_per_segment, int64_t resident)
{
    s.segments = 1;
    s.segment_steps = s.chunks * kScanChunk;
    if (resident / blocks_per_segment < 2 || s.chunks < 2) return;
    int64_t best = -1;
    int best_per = s.chunks;
    for (int rounds = 1; rounds <= 4; ++rounds) {
        const int64_t most = rounds * resident / blocks_per_segment;
        const int64_t per = div_up(s.chunks, most < s.chunks ? most : s.chunks);
        const int64_t taken = div_up(div_up(s.chunks, per) * blocks_per_segment, resident);
        const int64_t cost = taken * (4 * per + 1);      // a block's start and end: about a quarter of a chunk
        if (best < 0 || cost < best) {
            best = cost;
            best_per = static_cast<int>(per);
        }
    }
    s.segments = static_cast<int>(div_up(s.chunks, best_per));
    s.segment_steps = best_per * kScanChunk;
}

ScanShape scan_shape(const ssm *p, int64_t batch, int64_t time, bool backward)
{
    ScanShape s = {};
    s.batch = batch;
    s.time = static_cast<int>(time);
    s.channels = p->channels;
    s.states = p->states;
    s.groups = p->groups;
    s.group_channels = p->channels / p->groups;
    s.quads = quads_of(p->states);
    s.chunks = static_cast<int>(div_up(time, kScanChunk));
    const int64_t per_block = backward ? scan_back_channels(p->states) : 128 / lanes_of(p->states);
    const int64_t tiles = div_up(s.group_channels, per_block) * s.groups;
    // resident blocks per SM: by registers, beyond 32 states backward by shared memory
    const int lanes = lanes_of(p->states);
    const int per_sm = backward ? (lanes <= 2 ? 2 : 1) : (lanes == 1 ? 4 : 3);
    cut_time(s, batch * tiles, static_cast<int64_t>(p->sms) * per_sm);
    s.slots = 1;
    if (backward) {
        // about four rounds of resident blocks, each with the same number of rows
        const int64_t units = batch * s.segments;
        int64_t slots = div_up(static_cast<int64_t>(p->sms) * 8, tiles);
        if (slots > units) slots = units;
        s.slots = static_cast<int>(div_up(units, div_up(units, slots)));
    }
    return s;
}

struct ScanScratch {
    size_t carry, span, da_part, dd_part, dbc_part, total;
};

ScanScratch scan_scratch(const ScanShape &s, bool backward)
{
    ScanScratch w = {};
    size_t at = 0;
    const size_t rows = static_cast<size_t>(s.batch) * s.segments;
    w.carry = at;
    if (s.segments > 1) at += rows * s.quads * s.channels * 16;
    w.span = at;
    if (s.segments > 1) at = align16(at + rows * s.channels * 4);
    if (backward) {
        w.da_part = at;
        at += static_cast<size_t>(s.slots) * s.quads * s.channels * 16;
        w.dd_part = at;
        at = align16(at + static_cast<size_t>(s.slots) * 2 * s.channels * 4);
        w.dbc_part = at;
        const size_t tiles = div_up(s.group_channels, scan_back_channels(s.states));
        const size_t padded = s.states <= 16 ? 16 : s.states <= 32 ? 32 : 64;
        at += tiles * static_cast<size_t>(s.batch) * s.time * s.groups * 2 * padded * 4;
    }
    w.total = at;
    return w;
}

int check_seq(const ssm_seq &q, size_t bytes)
{
    if (q.ptr == nullptr) return SSM_ENULL;
    if (q.stride_b < 0 || q.stride_t < 0) return SSM_EINVAL;
    return aligned(q.ptr, bytes) ? SSM_OK : SSM_EALIGN;
}

// Do rows of `row` elements, of which `many` are `step` apart and these in turn `few` times `jump`, stay clear of
// one another?  They do where a jump passes all the steps; else the i-th jump has to land between two steps.
bool rows_apart(int64_t row, int64_t many, int64_t step, int64_t few, int64_t jump)
{
    if ((many > 1 && step < row) || (few > 1 && jump < row)) return false;
    if (many == 1 || few == 1) return true;
    using wide = __int128;
    if (jump >= static_cast<wide>(many - 1) * step + row || step >= static_cast<wide>(few - 1) * jump + row) return true;
    for (int64_t i = 1; i < few; ++i) {
        const wide at = static_cast<wide>(i) * jump, below = at / step;
        if (below < many && at - below * step < row) return false;
        if (below + 1 < many && (below + 1) * step - at < row) return false;
    }
    return true;
}

// Outputs must not share elements.
int check_out(const ssm_seq &q, size_t bytes, int64_t row, int64_t batch, int64_t time)
{
    const int rc = check_seq(q, bytes);
    if (rc != SSM_OK) return rc;
    const bool apart = batch < time ? rows_apart(row, time, q.stride_t, batch, q.stride_b)
                                    : rows_apart(row, batch, q.stride_b, time, q.stride_t);
    return apart ? SSM_OK : SSM_EINVAL;
}

int check_scan(const ssm *p, const ssm_scan_args *a, bool backward)
{
    if (p == nullptr || a == nullptr) return SSM_ENULL;
    if (!sizes_ok(a->batch, a->time)) return SSM_EINVAL;
    const size_t e = element_bytes(p);
    const int64_t wide = p->channels, narrow = static_cast<int64_t>(p->groups) * p->states;
    int rc;
    for (const ssm_seq *q : {&a->x, &a->dt, &a->b, &a->c})
        if ((rc = check_seq(*q, e)) != SSM_OK) return rc;
    if (a->z.ptr != nullptr && (rc = check_seq(a->z, e)) != SSM_OK) return rc;
    if (a->reset.ptr != nullptr && (rc = check_seq(a->reset, 1)) != SSM_OK) return rc;
    if (a->a == nullptr) return SSM_ENULL;
    const float *vectors[] = {a->a, a->d, a->dt_bias, a->da, a->dd, a->ddt_bias};
    for (const float *v : vectors)
        if (!aligned(v, 4)) return SSM_EALIGN;
    const void *wide_ptrs[] = {a->state, a->state_out, a->saved, a->dstate_out, a->dstate, a->workspace};
    for (const void *v : wide_ptrs)
        if (!aligned(v, 16)) return SSM_EALIGN;
    if (!backward) {
        if (a->state != nullptr && a->state == a->state_out) return SSM_EINVAL;
        return check_out(a->y, e, wide, a->batch, a->time);
    }
    if ((rc = check_seq(a->dy, e)) != SSM_OK) return rc;
    if (a->saved == nullptr || a->da == nullptr) return SSM_ENULL;
    if ((a->z.ptr == nullptr) != (a->dz.ptr == nullptr)) return SSM_ENULL;
    for (const ssm_seq *q : {&a->dx, &a->ddt})
        if ((rc = check_out(*q, e, wide, a->batch, a->time)) != SSM_OK) return rc;
    if (a->dz.ptr != nullptr && (rc = check_out(a->dz, e, wide, a->batch, a->time)) != SSM_OK) return rc;
    for (const ssm_seq *q : {&a->db, &a->dc})
        if ((rc = check_out(*q, e, narrow, a->batch, a->time)) != SSM_OK) return rc;
    return SSM_OK;
}

template <typename T>
int run_scan(ssm *p, const ssm_scan_args *a, bool backward)
{
    const ScanShape s = scan_shape(p, a->batch, a->time, backward);
    const int64_t per_block = backward ? scan_back_channels(p->states) : 128 / lanes_of(p->states);
    const int64_t tiles = div_up(s.group_channels, per_block) * s.groups;
    // the grids below have one dimension
    if (s.batch * s.segments * div_up(s.group_channels, 128 / lanes_of(p->states)) * s.groups > kMaxBlocks ||
        s.slots * tiles > kMaxBlocks || s.batch * s.quads * s.channels / 256 >= kMaxBlocks ||
        (backward && s.batch * s.time * s.groups * 2 * 64 / 256 >= kMaxBlocks))
        return SSM_EINVAL;
    const ScanScratch w = scan_scratch(s, backward);
    if (w.total > 0 && a->workspace == nullptr) return SSM_ENULL;
    if (w.total > a->workspace_bytes) return SSM_ENOMEM;
    uint8_t *base = static_cast<uint8_t *>(a->workspace);
    ScanParams k = {};
    k.a = a->a;
    k.d = a->d;
    k.dt_bias = a->dt_bias;
    k.state = a->state;
    k.state_out = a->state_out;
    k.saved = a->saved;
    k.dstate_out = a->dstate_out;
    k.dstate = a->dstate;
    k.da = a->da;
    k.dd = a->dd;
    k.ddt_bias = a->ddt_bias;
    if (w.total > 0) {
        k.carry = reinterpret_cast<float *>(base + w.carry);
        k.span = reinterpret_cast<float *>(base + w.span);
        k.da_part = reinterpret_cast<float *>(base + w.da_part);
        k.dd_part = reinterpret_cast<float *>(base + w.dd_part);
        k.dbc_part = reinterpret_cast<float *>(base + w.dbc_part);
    }
    ScanSeqs<T> q = {};
    q.x = seq_of<const T>(a->x);
    q.dt = seq_of<const T>(a->dt);
    q.z = seq_of<const T>(a->z);
    q.b = seq_of<const T>(a->b);
    q.c = seq_of<const T>(a->c);
    q.reset = seq_of<const uint8_t>(a->reset);
    int launched;
    if (backward) {
        q.dy = seq_of<const T>(a->dy);
        q.dx = seq_of<T>(a->dx);
        q.ddt = seq_of<T>(a->ddt);
        q.dz = seq_of<T>(a->dz);
        q.db = seq_of<T>(a->db);
        q.dc = seq_of<T>(a->dc);
        launched = launch_scan_backward<T>(s, k, q, p->stream);
    } else {
        q.y = seq_of<T>(a->y);
        launched = launch_scan_forward<T>(s, k, q, p->stream);
    }
    if (launched < 0) {
        cudaGetLastError();
        return SSM_ECUDA;
    }
    p->launches += launched;
    return SSM_OK;
}

int scan(ssm *p, const ssm_scan_args *a, bool backward)
{
    const int rc = check_scan(p, a, backward);
    if (rc != SSM_OK) return rc;
    const OnDevice on(p->device);
    if (!on.ok()) return SSM_ECUDA;
    if (p->type == SSM_F32) return run_scan<float>(p, a, backward);
    return p->type == SSM_BF16 ? run_scan<__nv_bfloat16>(p, a, backward) : run_scan<__half>(p, a, backward);
}

// Units of work of the convolution: runs of steps, a warp for every 128 channels of each.  A run
// re-reads width - 1 steps and starts with nothing in flight, so it is as long as the device
// stays full, 128 steps at most.
ConvShape conv_shape(const ssm *p, int64_t batch, int64_t time)
{
    ConvShape s = {};
    s.batch = batch;
    s.time = static_cast<int>(time);
    s.channels = p->channels;
    s.width = p->width;
    s.sms = p->sms;
    const int64_t warps = div_up(p->channels, 128);          // of a run, where vectors can be used
    const int64_t resident = static_cast<int64_t>(p->sms) * 16;
    s.run = 128;
    while (s.run > 8 && batch * div_up(time, s.run) * warps < 2 * resident) s.run /= 2;
    s.runs = static_cast<int>(div_up(time, s.run));
    const int64_t units = batch * s.runs;
    int64_t slots = div_up(resident, warps);
    if (slots > units) slots = units;
    s.slots = static_cast<int>(div_up(units, div_up(units, slots)));
    return s;
}

int check_conv(const ssm *p, const ssm_conv_args *a, bool backward)
{
    if (p == nullptr || a == nullptr) return SSM_ENULL;
    if (!sizes_ok(a->batch, a->time)) return SSM_EINVAL;
    const size_t e = element_bytes(p);
    int rc = check_seq(a->x, e);
    if (rc != SSM_OK) return rc;
    if (a->reset.ptr != nullptr && (rc = check_seq(a->reset, 1)) != SSM_OK) return rc;
    if (a->w == nullptr) return SSM_ENULL;
    const float *vectors[] = {a->w, a->bias, a->dw, a->dbias};
    for (const float *v : vectors)
        if (!aligned(v, 4)) return SSM_EALIGN;
    if (!aligned(a->history, e) || !aligned(a->history_out, e)) return SSM_EALIGN;
    if (!backward) {
        if (a->history != nullptr && a->history == a->history_out) return SSM_EINVAL;
        return check_out(a->y, e, p->channels, a->batch, a->time);
    }
    if ((rc = check_seq(a->dy, e)) != SSM_OK) return rc;
    if ((rc = check_out(a->dx, e, p->channels, a->batch, a->time)) != SSM_OK) return rc;
    return a->dw == nullptr ? SSM_ENULL : SSM_OK;
}

size_t conv_scratch(const ConvShape &s)
{
    return static_cast<size_t>(s.slots) * (s.width + 1) * s.channels * sizeof(float);
}

template <typename T>
int run_conv(ssm *p, const ssm_conv_args *a, bool backward)
{
    const ConvShape s = conv_shape(p, a->batch, a->time);
    if (s.batch * s.runs > kMaxBlocks * 128 / (s.channels + 31)) return SSM_EINVAL;   // threads, rows of whole warps
    ConvParams k = {a->w, a->bias, a->dw, a->dbias, static_cast<float *>(a->workspace)};
    ConvSeqs<T> q = {};
    q.x = seq_of<const T>(a->x);
    q.reset = seq_of<const uint8_t>(a->reset);
    q.history = static_cast<const T *>(a->history);
    int launched;
    if (backward) {
        if (a->workspace == nullptr) return SSM_ENULL;
        if (!aligned(a->workspace, 16)) return SSM_EALIGN;
        if (a->workspace_bytes < conv_scratch(s)) return SSM_ENOMEM;
        q.dy = seq_of<const T>(a->dy);
        q.dx = seq_of<T>(a->dx);
        launched = launch_conv_backward<T>(s, k, q, p->stream);
    } else {
        q.y = seq_of<T>(a->y);
        q.history_out = static_cast<T *>(a->history_out);
        launched = launch_conv_forward<T>(s, k, q, p->stream);
    }
    if (launched < 0) {
        cudaGetLastError();
        return SSM_ECUDA;
    }
    p->launches += launched;
    return SSM_OK;
}

int conv(ssm *p, const ssm_conv_args *a, bool backward)
{
    const int rc = check_conv(p, a, backward);
    if (rc != SSM_OK) return rc;
    const OnDevice on(p->device);
    if (!on.ok()) return SSM_ECUDA;
    if (p->type == SSM_F32) return run_conv<float>(p, a, backward);
    return p->type == SSM_BF16 ? run_conv<__nv_bfloat16>(p, a, backward) : run_conv<__half>(p, a, backward);
}

}  // namespace

extern "C" {

int ssm_create(ssm **out, int channels, int states, int groups, int width, int type)
{
    if (out == nullptr) return SSM_ENULL;
    *out = nullptr;
    if (channels < 1 || channels > SSM_MAX_CHANNELS || states < 1 || states > SSM_MAX_STATES) return SSM_EINVAL;
    if (groups < 1 || groups > channels || channels % groups != 0) return SSM_EINVAL;
    if (width < 2 || width > SSM_MAX_WIDTH || type < SSM_F32 || type > SSM_F16) return SSM_EINVAL;
    int device = 0, sms = 0;
    if (cudaGetDevice(&device) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
        cudaGetLastError();
        return SSM_ECUDA;
    }
    ssm *p = new (std::nothrow) ssm;
    if (p == nullptr) return SSM_ENOMEM;
    p->channels = channels;
    p->states = states;
    p->groups = groups;
    p->width = width;
    p->type = type;
    p->device = device;
    p->sms = sms;
    *out = p;
    return SSM_OK;
}

int ssm_destroy(ssm *p)
{
    if (p == nullptr) return SSM_ENULL;
    delete p;
    return SSM_OK;
}

int ssm_set_stream(ssm *p, void *cuda_stream)
{
    if (p == nullptr) return SSM_ENULL;
    p->stream = static_cast<cudaStream_t>(cuda_stream);
    return SSM_OK;
}

size_t ssm_conv_workspace_bytes(const ssm *p, int64_t batch, int64_t time)
{
    if (p == nullptr || !sizes_ok(batch, time)) return 0;
    return conv_scratch(conv_shape(p, batch, time));
}

int ssm_conv_forward(ssm *p, const ssm_conv_args *a) { return conv(p, a, false); }

int ssm_conv_backward(ssm *p, const ssm_conv_args *a) { return conv(p, a, true); }

int ssm_conv_step(ssm *p, const void *x, int64_t x_stride, const uint8_t *done, int64_t done_stride, const float *w,
                  const float *bias, const void *history, void *history_out, void *y, int64_t y_stride, int64_t n)
{
    if (p == nullptr) return SSM_ENULL;
    if (n < 1) return SSM_EINVAL;                     // first: an empty batch comes without pointers
    if (x == nullptr || w == nullptr || history == nullptr || history_out == nullptr || y == nullptr) return SSM_ENULL;
    if (n > kMaxBlocks * 128 / p->channels || x_stride < 0 || done_stride < 0) return SSM_EINVAL;
    if (n > 1 && y_stride < p->channels) return SSM_EINVAL;
    const size_t e = element_bytes(p);
    if (!aligned(x, e) || !aligned(y, e) || !aligned(history, e) || !aligned(history_out, e) || !aligned(w, 4) ||
        !aligned(bias, 4))
        return SSM_EALIGN;
    ConvShape s = {};
    s.batch = n;
    s.channels = p->channels;
    s.width = p->width;
    s.sms = p->sms;
    const ConvParams k = {w, bias, nullptr, nullptr, nullptr};
    const OnDevice on(p->device);
    if (!on.ok()) return SSM_ECUDA;
    int launched;
    auto call = [&](auto zero) {
        using T = decltype(zero);
        return launch_conv_step<T>(s, k, static_cast<const T *>(x), x_stride, done, done_stride,
                                   static_cast<const T *>(history), static_cast<T *>(history_out),
                                   static_cast<T *>(y), y_stride, p->stream);
    };
    if (p->type == SSM_F32)
        launched = call(float());
    else
        launched = p->type == SSM_BF16 ? call(__nv_bfloat16()) : call(__half());
    if (launched < 0) {
        cudaGetLastError();
        return SSM_ECUDA;
    }
    p->launches += launched;
    return SSM_OK;
}

size_t ssm_scan_saved_bytes(const ssm *p, int64_t batch, int64_t time)
{
    if (p == nullptr || !sizes_ok(batch, time)) return 0;
    return static_cast<size_t>(batch) * div_up(time, kScanChunk) * quads_of(p->states) * p->channels * 16;
}

size_t ssm_scan_workspace_bytes(const ssm *p, int64_t batch, int64_t time, int backward)
{
    if (p == nullptr || !sizes_ok(batch, time)) return 0;
    return scan_scratch(scan_shape(p, batch, time, backward != 0), backward != 0).total;
}

int ssm_scan_forward(ssm *p, const ssm_scan_args *a) { return scan(p, a, false); }

int ssm_scan_backward(ssm *p, const ssm_scan_args *a) { return scan(p, a, true); }

int ssm_scan_step(ssm *p, const void *x, int64_t x_stride, const void *dt, int64_t dt_stride, const void *z,
                  int64_t z_stride, const void *b, int64_t b_stride, const void *c, int64_t c_stride,
                  const uint8_t *done, int64_t done_stride, const float *a, const float *d, const float *dt_bias,
                  const float *state, float *state_out, void *y, int64_t y_stride, int64_t n)
{
    if (p == nullptr) return SSM_ENULL;
    if (n < 1) return SSM_EINVAL;
    if (x == nullptr || dt == nullptr || b == nullptr || c == nullptr || a == nullptr || state == nullptr ||
        state_out == nullptr || y == nullptr)
        return SSM_ENULL;
    if (n > kMaxBlocks || x_stride < 0 || dt_stride < 0 || z_stride < 0 || b_stride < 0 || c_stride < 0 ||
        done_stride < 0 || (n > 1 && y_stride < p->channels))
        return SSM_EINVAL;
    const size_t e = element_bytes(p);
    for (const void *v : {x, dt, z, b, c, static_cast<const void *>(y)})
        if (!aligned(v, e)) return SSM_EALIGN;
    for (const float *v : {a, d, dt_bias})
        if (!aligned(v, 4)) return SSM_EALIGN;
    if (!aligned(state, 16) || !aligned(state_out, 16)) return SSM_EALIGN;
    const StepParams k = {a, d, dt_bias, state, state_out, done, x_stride, dt_stride, z_stride, b_stride, c_stride,
                          y_stride, done_stride, n, p->channels, p->states, p->channels / p->groups, p->sms};
    const OnDevice on(p->device);
    if (!on.ok()) return SSM_ECUDA;
    int launched;
    auto call = [&](auto zero) {
        using T = decltype(zero);
        return launch_scan_step<T>(k, static_cast<const T *>(x), static_cast<const T *>(dt),
                                   static_cast<const T *>(z), static_cast<const T *>(b), static_cast<const T *>(c),
                                   static_cast<T *>(y), p->stream);
    };
    if (p->type == SSM_F32)
        launched = call(float());
    else
        launched = p->type == SSM_BF16 ? call(__nv_bfloat16()) : call(__half());
    if (launched < 0) {
        cudaGetLastError();
        return SSM_ECUDA;
    }
    p->launches += launched;
    return SSM_OK;
}

int64_t ssm_launch_count(const ssm *p) { return p ? p->launches : 0; }

const char *ssm_strerror(int code)
{
    switch (code) {
    case SSM_OK: return "ok";
    case SSM_EINVAL: return "invalid size, stride or type";
    case SSM_ENULL: return "required pointer is NULL";
    case SSM_EALIGN: return "a pointer is not aligned";
    case SSM_ECUDA: return "CUDA runtime call or launch failed";
    case SSM_ENOMEM: return "allocation failed, or the workspace is too small";
    default: return "unknown error";
    }
}

}  // extern "C"
