// AdamW over many tensors at once.  Declared in include/cocod_adamw.h.
#include "cocod_adamw.h"
#include "cocod_adamw.cuh"
#include "cocod_internal.h"
#include "cocod_lm_internal.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

struct cocod_adamw {
    int n = 0, bits = 0, device = -1, quads = 1;
    bool flat = false;
    long long covered = 0;                 // flat: the values that the tensors cover one behind the other, 0 if they do not
    long long values = 0, launches = 0;
    std::vector<int> first_chunk;          // n + 1
    std::vector<int64_t> sizes;
    cocod::adamw::Tensor *tensors = nullptr;
    int *chunk_tensor = nullptr;
    cocod::adamw::Clock *clock = nullptr;
    cocod::adamw::State state{};
    double beta1 = 0, beta2 = 0;
    float eps = 0;
};

namespace {

using namespace cocod;
using namespace cocod::adamw;
using bf16 = __nv_bfloat16;

constexpr int SMALL = 64, LARGE = 1024;    // tensors in a launch's parameters

void adamw_free(cocod_adamw *h)
{
    void *ptrs[] = {h->tensors, h->chunk_tensor, h->clock};
    for (void *p : ptrs) if (p) cudaFree(p);
    delete h;
}

template <typename P, typename G, int BITS, typename W>
int launch_step(cocod_adamw *h, const Step &s, const W &where, int chunks, cudaStream_t stream)
{
    TRY_CUDA(launch_dependent(true, adamw_step<P, G, BITS, W>, dim3((unsigned)chunks), dim3(THREADS), 0, stream, s, where));
    return COCOD_OK;
}
template <typename W>
int launch_types(cocod_adamw *h, const Step &s, const W &where, int chunks, int param_type, int grad_type, cudaStream_t stream)
{
    const int form = (h->bits == 8 ? 4 : 0) + (param_type == COCOD_BF16 ? 2 : 0) + (grad_type == COCOD_BF16 ? 1 : 0);
    switch (form) {
    case 0: return launch_step<float, float, 32>(h, s, where, chunks, stream);
    case 1: return launch_step<float, bf16, 32>(h, s, where, chunks, stream);
    case 2: return launch_step<bf16, float, 32>(h, s, where, chunks, stream);
    case 3: return launch_step<bf16, bf16, 32>(h, s, where, chunks, stream);
    case 4: return launch_step<float, float, 8>(h, s, where, chunks, stream);
    case 5: return launch_step<float, bf16, 8>(h, s, where, chunks, stream);
    case 6: return launch_step<bf16, float, 8>(h, s, where, chunks, stream);
    default: return launch_step<bf16, bf16, 8>(h, s, where, chunks, stream);
    }
}
Step step_of(const cocod_adamw *h, const float *grad_scale)
{
    Step s{};
    s.tensors = h->tensors; s.chunk_tensor = h->chunk_tensor; s.clock = h->clock; s.state = h->state; s.grad_scale = grad_scale;
    s.beta1 = h->beta1; s.beta2 = h->beta2;
    s.b1 = (float)h->beta1; s.rest1 = (float)(1.0 - h->beta1); s.b2 = (float)h->beta2; s.rest2 = (float)(1.0 - h->beta2); s.eps = h->eps;
    s.quads = h->quads;
    s.advance = 1;
    return s;
}
// Values in a chunk, in units of APART.  What begins a chunk (its tensor, its addresses) is not hidden, so that long ones are better where there are
// enough of them for all SMs.  Small models: the shortest (50000 values: 10.3 us, chunks of 2048 12.3).  32 bits: 4 (187 M values: 768 us; chunks of 2048 834,
// of 8192 774; thread blocks that take one chunk after another 891).  8 bits, whose loads run ahead inside a chunk: up to 16, as long as every
// SM gets a dozen (150 M values: chunks of 16384 432 us, of 8192 469; 30 M: 106.5 and 110, of 32768 114).
int quads_of(int64_t values, int bits)
{
    const int64_t sms = std::max(1, sm_count());
    if (values <= 2 * APART * sms) return bits == 8 ? 2 : 1;
    if (bits == 32) return 4;
    int quads = 16;
    while (quads > 2 && values < 12 * sms * quads * APART) quads /= 2;
    return quads;
}
bool aligned(const void *p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

template <int CAPACITY>
int list_step(cocod_adamw *h, Step s, void *const *params, int param_type, const void *const *grads, int grad_type, void *const *copies, cudaStream_t stream)
{
    for (int t0 = 0; t0 < h->n; t0 += CAPACITY) {
        const int t1 = std::min(h->n, t0 + CAPACITY);
        Lists<CAPACITY> l;
        for (int i = t0; i < t1; ++i) {
            l.param[i - t0] = params[i];
            l.grad[i - t0] = grads[i];
            l.copy[i - t0] = copies ? copies[i] : nullptr;
        }
        s.first_tensor = t0; s.first_chunk = h->first_chunk[t0]; s.advance = t1 == h->n;
        if (int rc = launch_types(h, s, l, h->first_chunk[t1] - s.first_chunk, param_type, grad_type, stream)) return rc;
    }
    return COCOD_OK;
}

}  // namespace

extern "C" {

int64_t cocod_adamw_values(int n, const int64_t *sizes)
{
    if (n < 1 || n > COCOD_ADAMW_MAX_TENSORS || !sizes) return COCOD_ERR_INVALID;
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
        if (sizes[i] < 1 || sizes[i] >= (1ll << 40)) return COCOD_ERR_INVALID;
        total += ceil_div(sizes[i], BLOCK) * BLOCK;
        if (total >= (1ll << 40)) return COCOD_ERR_INVALID;
    }
    return total;
}

int cocod_adamw_create(cocod_adamw_handle **out, int n, const int64_t *sizes, const float *decay, const int64_t *starts, int state_bits, void *m, void *v,
                       float *m_units, float *v_units, float lr, double beta1, double beta2, float eps)
{
    const int64_t values = out ? cocod_adamw_values(n, sizes) : COCOD_ERR_INVALID;
    if (values < 0 || (state_bits != COCOD_ADAMW_8 && state_bits != COCOD_ADAMW_32) || !m || !v || !aligned16(m) || !aligned16(v) ||
        (state_bits == COCOD_ADAMW_8 && (!m_units || !v_units || !aligned(m_units, 4) || !aligned(v_units, 4))) || !std::isfinite(lr) || !(beta1 >= 0.0 && beta1 < 1.0) ||
        !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0f) || !std::isfinite(eps))
        return COCOD_ERR_INVALID;
    for (int i = 0; i < n; ++i)
        if ((decay && !std::isfinite(decay[i])) || (starts && (starts[i] < 0 || starts[i] >= (1ll << 40)))) return COCOD_ERR_INVALID;
    cocod_adamw *h = nullptr;
    try {
        const int quads = quads_of(values, state_bits);
        const int64_t chunk = quads * APART;
        int64_t chunks = 0;
        for (int i = 0; i < n; ++i) chunks += ceil_div(sizes[i], chunk);
        if (chunks > MAX_DIM) return COCOD_ERR_TOO_LARGE;
        h = new cocod_adamw();
        h->quads = quads;
        h->n = n; h->bits = state_bits; h->device = current_device(); h->flat = starts != nullptr; h->values = values;
        h->state = State{m, v, m_units, v_units};
        h->beta1 = beta1; h->beta2 = beta2; h->eps = eps;
        h->first_chunk.resize(n + 1);
        h->sizes.assign(sizes, sizes + n);
        std::vector<Tensor> tensors(n);
        std::vector<int> chunk_tensor(chunks);
        long long state = 0, covered = 0;
        bool gaps = !starts;
        int at = 0;
        for (int i = 0; i < n; ++i) {
            tensors[i] = Tensor{sizes[i], starts ? starts[i] : 0, state, at, decay ? decay[i] : 0.0f};
            gaps = gaps || starts[i] != covered;
            covered += sizes[i];
            h->first_chunk[i] = at;
            const int here = (int)ceil_div(sizes[i], chunk);
            std::fill_n(chunk_tensor.begin() + at, here, i);
            at += here;
            state += ceil_div(sizes[i], BLOCK) * BLOCK;
        }
        h->first_chunk[n] = at;
        h->covered = gaps ? 0 : covered;
        const Clock clock{1.0, 1.0, lr, (float)(1.0 / (1.0 - beta1)), (float)(1.0 / std::sqrt(1.0 - beta2)), 0u, 0};
        cudaError_t e = cudaMalloc((void **)&h->tensors, n * sizeof(Tensor));
        if (e == cudaSuccess) e = cudaMalloc((void **)&h->chunk_tensor, chunks * sizeof(int));
        if (e == cudaSuccess) e = cudaMalloc((void **)&h->clock, sizeof(Clock));
        // (steps come on any stream: the tables have to be there, and need not wait for other work)
        cudaStream_t s = nullptr;
        if (e == cudaSuccess) e = cudaStreamCreateWithFlags(&s, cudaStreamNonBlocking);
        if (e == cudaSuccess) e = cudaMemcpyAsync(h->tensors, tensors.data(), n * sizeof(Tensor), cudaMemcpyHostToDevice, s);
        if (e == cudaSuccess) e = cudaMemcpyAsync(h->chunk_tensor, chunk_tensor.data(), chunks * sizeof(int), cudaMemcpyHostToDevice, s);
        if (e == cudaSuccess) e = cudaMemcpyAsync(h->clock, &clock, sizeof(Clock), cudaMemcpyHostToDevice, s);
        if (e == cudaSuccess) e = cudaStreamSynchronize(s);
        if (s) cudaStreamDestroy(s);
        if (e != cudaSuccess) {
            cudaGetLastError();
            adamw_free(h);
            return e == cudaErrorMemoryAllocation ? COCOD_ERR_OOM : COCOD_ERR_CUDA;
        }
    } catch (const std::bad_alloc &) {
        if (h) adamw_free(h);
        return COCOD_ERR_OOM;
    }
    *out = h;
    return COCOD_OK;
}

int cocod_adamw_destroy(cocod_adamw_handle *h)
{
    if (!h) return COCOD_OK;
    const int now = current_device();
    if (now != h->device) cudaSetDevice(h->device);
    cudaDeviceSynchronize();
    if (now != h->device && now >= 0) cudaSetDevice(now);
    adamw_free(h);
    return COCOD_OK;
}

const int64_t *cocod_adamw_sizes(const cocod_adamw_handle *h, int *n)
{
    if (!h || !n) return nullptr;
    *n = h->n;
    return h->sizes.data();
}

int cocod_adamw_step(cocod_adamw_handle *h, void *const *params, int param_type, const void *const *grads, int grad_type, void *const *copies,
                     const float *grad_scale, cocod_stream_t stream)
{
    const int ps = size_of(param_type), gs = size_of(grad_type);
    if (!h || !ps || !gs || !params || !grads || (copies && param_type != COCOD_F32) || !aligned(grad_scale, 4)) return COCOD_ERR_INVALID;
    for (int i = 0; i < h->n; ++i)
        if (!params[i] || !aligned(params[i], ps) || !aligned(grads[i], gs) || (copies && !aligned(copies[i], 2))) return COCOD_ERR_INVALID;
    const Step s = step_of(h, grad_scale);
    return h->n <= SMALL ? list_step<SMALL>(h, s, params, param_type, grads, grad_type, copies, (cudaStream_t)stream)
                         : list_step<LARGE>(h, s, params, param_type, grads, grad_type, copies, (cudaStream_t)stream);
}

int cocod_adamw_flat_step(cocod_adamw_handle *h, const void *params_in, void *params_out, int param_type, const void *grads, int grad_type, void *copies,
                          const float *grad_scale, cocod_stream_t stream)
{
    const int ps = size_of(param_type), gs = size_of(grad_type);
    if (!h || !h->flat || !ps || !gs || !params_in || !params_out || !grads || (copies && param_type != COCOD_F32) || !aligned(params_in, ps) ||
        !aligned(params_out, ps) || !aligned(grads, gs) || !aligned(copies, 2) || !aligned(grad_scale, 4))
        return COCOD_ERR_INVALID;
    return launch_types(h, step_of(h, grad_scale), Flat{params_in, params_out, grads, copies}, h->first_chunk[h->n], param_type, grad_type, (cudaStream_t)stream);
}

int cocod_adamw_local_step(cocod_adamw_handle *h, cocod_handle *engine, const float *grads, const float *grad_scale)
{
    if (!h || !engine || !grads) return COCOD_ERR_INVALID;
    cocod_step_plan plan{};
    if (int rc = cocod_internal_plan_step(engine, &plan)) return rc;
    if (!h->flat || h->covered != (long long)plan.K * plan.P || h->device != plan.device) return COCOD_ERR_INVALID;
    if (int rc = cocod_adamw_flat_step(h, plan.x_in, plan.x_out, COCOD_F32, grads, COCOD_F32, plan.shadow, grad_scale, plan.compute)) return rc;
    return cocod_internal_finish_step(engine, 1);
}

int cocod_adamw_set_lr(cocod_adamw_handle *h, float lr, cocod_stream_t stream)
{
    if (!h || !std::isfinite(lr)) return COCOD_ERR_INVALID;
    TRY_CUDA(launch_dependent(true, adamw_set, dim3(1), dim3(1), 0, (cudaStream_t)stream, h->clock, 0, lr, 0ll, h->beta1, h->beta2));
    return COCOD_OK;
}

int cocod_adamw_set_step(cocod_adamw_handle *h, int64_t steps, cocod_stream_t stream)
{
    if (!h || steps < 0) return COCOD_ERR_INVALID;
    TRY_CUDA(launch_dependent(true, adamw_set, dim3(1), dim3(1), 0, (cudaStream_t)stream, h->clock, 1, 0.0f, (long long)steps, h->beta1, h->beta2));
    return COCOD_OK;
}

int cocod_adamw_get_step(cocod_adamw_handle *h, int64_t *steps, cocod_stream_t stream)
{
    if (!h || !steps) return COCOD_ERR_INVALID;
    const cudaStream_t s = (cudaStream_t)stream;
    long long got = 0;
    if (cudaMemcpyAsync(&got, &h->clock->steps, sizeof(got), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) {
        cudaGetLastError();
        return COCOD_ERR_CUDA;
    }
    *steps = got;
    return COCOD_OK;
}

int cocod_adamw_moments(cocod_adamw_handle *h, float *m, float *v, cocod_stream_t stream)
{
    if (!h || !m || !v || !aligned16(m) || !aligned16(v)) return COCOD_ERR_INVALID;
    const cudaStream_t s = (cudaStream_t)stream;
    if (h->bits == COCOD_ADAMW_32) {
        if (cudaMemcpyAsync(m, h->state.m, h->values * 4, cudaMemcpyDeviceToDevice, s) != cudaSuccess ||
            cudaMemcpyAsync(v, h->state.v, h->values * 4, cudaMemcpyDeviceToDevice, s) != cudaSuccess) {
            cudaGetLastError();
            return COCOD_ERR_CUDA;
        }
        return COCOD_OK;
    }
    const long long blocks = h->values / BLOCK;
    TRY_CUDA(launch_dependent(true, adamw_moments<true>, dim3((unsigned)std::min<long long>(ceil_div(blocks, THREADS / 16), 8ll * sm_count())), dim3(THREADS), 0, s,
                              h->state, blocks, m, v, static_cast<const float *>(nullptr), static_cast<const float *>(nullptr)));
    return COCOD_OK;
}

int cocod_adamw_load(cocod_adamw_handle *h, const float *m, const float *v, cocod_stream_t stream)
{
    if (!h || !m || !v || !aligned16(m) || !aligned16(v)) return COCOD_ERR_INVALID;
    const cudaStream_t s = (cudaStream_t)stream;
    if (h->bits == COCOD_ADAMW_32) {
        if (cudaMemcpyAsync(h->state.m, m, h->values * 4, cudaMemcpyDeviceToDevice, s) != cudaSuccess ||
            cudaMemcpyAsync(h->state.v, v, h->values * 4, cudaMemcpyDeviceToDevice, s) != cudaSuccess) {
            cudaGetLastError();
            return COCOD_ERR_CUDA;
        }
        return COCOD_OK;
    }
    const long long blocks = h->values / BLOCK;
    TRY_CUDA(launch_dependent(true, adamw_moments<false>, dim3((unsigned)std::min<long long>(ceil_div(blocks, THREADS / 16), 8ll * sm_count())), dim3(THREADS), 0, s,
                              h->state, blocks, static_cast<float *>(nullptr), static_cast<float *>(nullptr), m, v));
    return COCOD_OK;
}

int64_t cocod_adamw_launch_count(const cocod_adamw_handle *h) { return h ? h->launches : -1; }

}  // extern "C"
