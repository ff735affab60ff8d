// The C ABI declared in qlora.h: argument validation, workspace carving and kernel dispatch.  No kernel lives here.
#include <cuda_runtime.h>
#include <math.h>

#include <initializer_list>

#include "launch.h"
#include "qlora.h"

namespace {

using namespace qlora;

inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int check_bits(int bits) { return (bits == 2 || bits == 3 || bits == 4 || bits == 8) ? QLORA_OK : QLORA_ERR_UNSUPPORTED; }

int check_format(int bits, int K, int N) {
    if (K < 0 || N < 0) return QLORA_ERR_INVALID_ARG;
    if (check_bits(bits) != QLORA_OK) return QLORA_ERR_UNSUPPORTED;
    if (K % 32 != 0 || N % 8 != 0) return QLORA_ERR_UNSUPPORTED;
    return QLORA_OK;
}

int check_desc(const qlora_desc* d, bool need_lora) {
    if (d == nullptr) return QLORA_ERR_INVALID_ARG;
    const int rc = check_format(d->bits, d->K, d->N);
    if (rc != QLORA_OK) return rc;
    if (d->group_size <= 0) return QLORA_ERR_INVALID_ARG;
    if (d->group_size % 32 != 0 || d->K % d->group_size != 0) return QLORA_ERR_UNSUPPORTED;
    if (need_lora) {
        if (d->r < 0) return QLORA_ERR_INVALID_ARG;
        if (d->r % 8 != 0 || d->r > 64) return QLORA_ERR_UNSUPPORTED;
        if (!(d->alpha == d->alpha)) return QLORA_ERR_INVALID_ARG;   // NaN
    }
    return QLORA_OK;
}

size_t element_bytes(int dtype) { return dtype == QLORA_FP32 ? 4 : dtype == QLORA_E4M3 ? 1 : 2; }
bool element_aligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % element_bytes(dtype) == 0; }

int check_logits(int T, int V, long long row_stride, int dtype, float inv_temperature) {
    if (T < 0 || V < 0 || (T > 1 && row_stride < V)) return QLORA_ERR_INVALID_ARG;
    if (!(inv_temperature >= 0x1p-30f && inv_temperature <= 0x1p30f)) return QLORA_ERR_INVALID_ARG;
    if (dtype != QLORA_BF16 && dtype != QLORA_FP16 && dtype != QLORA_FP32) return QLORA_ERR_UNSUPPORTED;
    if (V == 0 || V > (1 << 24)) return QLORA_ERR_UNSUPPORTED;
    return QLORA_OK;
}

bool overlap(const void* a, size_t bytes_a, const void* b, size_t bytes_b) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return pa < pb + bytes_b && pb < pa + bytes_a;
}

// Whether two [T, V] tensors of rows that lie apart share memory.  (Different strides in the same stretch of memory: taken to.)
bool rows_overlap(const void* a, long long stride_a, const void* b, long long stride_b, int T, int V, size_t bytes) {
    typedef __int128 wide;                                            // (any stride that fits a long long)
    const wide pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b), size = bytes, length = V * size;
    if (pa + (T - 1) * size * stride_a + length <= pb || pb + (T - 1) * size * stride_b + length <= pa) return false;
    if (T == 1 || stride_a != stride_b) return true;
    const wide by = (pb > pa ? pb - pa : pa - pb) % (size * stride_a);   // (columns of one buffer may lie beside each other)
    return by < length || size * stride_a - by < length;
}

// `step`: the whole step (else only the gradients are used).
int check_adamw(const qlora_adamw_desc* d, bool step) {
    if (d == nullptr || d->n_tensors < 0 || (d->n_tensors > 0 && d->tensors == nullptr)) return QLORA_ERR_INVALID_ARG;
    if (!(d->beta1 >= 0.0 && d->beta1 < 1.0 && d->beta2 >= 0.0 && d->beta2 < 1.0)) return QLORA_ERR_INVALID_ARG;
    if (!(d->eps >= 1e-30 && d->eps < 1e30) || !(d->weight_decay >= 0.0 && d->weight_decay < 1e30)) return QLORA_ERR_INVALID_ARG;
    if (d->grad_type != QLORA_FP32 && d->grad_type != QLORA_BF16 && d->grad_type != QLORA_FP16) return QLORA_ERR_UNSUPPORTED;
    if (d->param_type != QLORA_FP32 && d->param_type != QLORA_BF16 && d->param_type != QLORA_FP16) return QLORA_ERR_UNSUPPORTED;
    if (d->state_type != QLORA_FP32 && d->state_type != QLORA_E4M3) return QLORA_ERR_UNSUPPORTED;
    const bool eight = d->state_type == QLORA_E4M3;
    for (int i = 0; i < d->n_tensors; ++i) {
        const qlora_adamw_tensor& t = d->tensors[i];
        if (t.n < 0) return QLORA_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        if (t.n > (1ll << 40)) return QLORA_ERR_UNSUPPORTED;
        if (!t.grad) return QLORA_ERR_INVALID_ARG;
        uintptr_t all = reinterpret_cast<uintptr_t>(t.grad);
        if (step) {
            if (!t.param || !t.m || !t.v || (t.m_scale != nullptr) != eight || (t.v_scale != nullptr) != eight) return QLORA_ERR_INVALID_ARG;
            if (t.master && d->param_type == QLORA_FP32) return QLORA_ERR_INVALID_ARG;
            for (const void* p : {(const void*)t.param, (const void*)t.master, (const void*)t.m, (const void*)t.v}) all |= reinterpret_cast<uintptr_t>(p);
            if ((reinterpret_cast<uintptr_t>(t.m_scale) | reinterpret_cast<uintptr_t>(t.v_scale)) & 3u) return QLORA_ERR_ALIGNMENT;
        }
        if (all & 15u) return QLORA_ERR_ALIGNMENT;
    }
    return QLORA_OK;
}

int check_adapters(const qlora_adapters_desc* d, int M) {
    if (d == nullptr || d->K < 0 || d->N < 0 || d->r < 0 || d->n_adapters < 0) return QLORA_ERR_INVALID_ARG;
    if (d->K == 0 || d->K % 32 != 0 || d->N == 0 || d->N % 8 != 0 || d->r % 8 != 0 || d->r == 0 || d->r > 64 || d->n_adapters > 65535) return QLORA_ERR_UNSUPPORTED;
    if (d->K > (1 << 24) || d->N > (1 << 24)) return QLORA_ERR_UNSUPPORTED;   // (elements of an adapter's matrix are counted in 32 bits)
    if (M < 0) return QLORA_ERR_INVALID_ARG;
    return M > (1 << 20) ? QLORA_ERR_UNSUPPORTED : QLORA_OK;
}
// Workspace of the calls on adapters: two [M, r] products, then the scratch of the gradients.
size_t adapters_low_bytes(const qlora_adapters_desc& d, int M) { return align_up((size_t)M * (size_t)d.r * sizeof(float), 256); }
size_t adapters_bytes(const qlora_adapters_desc& d, int M) {
    const size_t grads = 2 * adapters_low_bytes(d, M) + adapters_grad_scratch_bytes(M, d.K, d.N, d.r, d.n_adapters), products = adapters_scratch_bytes(M, d.r);
    return grads > products ? grads : products;
}

struct Workspace {
    size_t p0_off, p1_off, grad_off, sync_off, split_off, db_off;
    size_t required;   // what a call cannot do without
    size_t total;      // ... plus the optional areas, each used when the workspace reaches that far: the exchange area
                       // of split tiles, then the producers' parts of dB (qlora_bwd_input_db)
};

Workspace carve(const qlora_desc& d, int M) {
    Workspace w{};
    const size_t p = align_up((size_t)M * (size_t)d.r * sizeof(float), 256);
    w.p0_off = 0;
    w.p1_off = p;
    w.grad_off = 2 * p;
    w.sync_off = w.grad_off + align_up(lora_grad_scratch_bytes(M, d.K, d.N, d.r), 256);
    w.split_off = w.sync_off + 256;      // the counters of the tensor-core kernels: producer clusters, split tiles
    w.required = w.split_off;
    w.db_off = w.split_off + align_up(umma_split_scratch_bytes(d, M), 256);
    w.total = w.db_off + umma_db_part_bytes(d, M);
    return w;
}

}  // namespace

// What the layer calls cannot do without: qlora_workspace_bytes minus the exchange area of split tiles, which
// qlora_fwd / qlora_bwd_input use only when it is there (and qlora_bwd_lora never).
size_t qlora::required_workspace_bytes(const qlora_desc& d, int M) { return carve(d, M).required; }

extern "C" {

const char* qlora_status_string(int status) {
    switch (status) {
        case QLORA_OK: return "ok";
        case QLORA_ERR_INVALID_ARG: return "invalid argument";
        case QLORA_ERR_UNSUPPORTED: return "unsupported shape, bit width, group size or rank";
        case QLORA_ERR_ALIGNMENT: return "pointer not 16-byte aligned";
        case QLORA_ERR_WORKSPACE: return "workspace missing or too small";
        case QLORA_ERR_CUDA: return "CUDA call failed";
        case QLORA_ERR_TIMEOUT: return "bounded device-side wait gave up";
        case QLORA_ERR_STATIC_LIMIT: return "scratch need exceeds the library's built-in array";
        default: return "unknown status";
    }
}

int qlora_device_status(unsigned int* status_out, int clear) {
    if (status_out == nullptr) return QLORA_ERR_INVALID_ARG;
    if (cudaDeviceSynchronize() != cudaSuccess) return QLORA_ERR_CUDA;
    unsigned int head = 0;
    int rc = read_device_status(status_out, clear);
    if (rc == QLORA_OK) rc = read_head_status(&head, clear);
    if (rc != QLORA_OK) return rc;
    *status_out |= head << 1;
    return *status_out == 0 ? QLORA_OK : QLORA_ERR_TIMEOUT;
}

int qlora_selftest_bounded_wait(int limit_us, void* cuda_stream) {
    if (limit_us < 1 || limit_us > 1000000) return QLORA_ERR_INVALID_ARG;
    const int rc = launch_wait_probe(limit_us, (cudaStream_t)cuda_stream);
    return rc != QLORA_OK ? rc : launch_head_wait_probe(limit_us, (cudaStream_t)cuda_stream);
}

int qlora_workspace_bytes(const qlora_desc* desc, int M, size_t* out) {
    if (out == nullptr || M < 0) return QLORA_ERR_INVALID_ARG;
    const int rc = check_desc(desc, true);
    if (rc != QLORA_OK) return rc;
    *out = carve(*desc, M).total;
    return QLORA_OK;
}

int qlora_pack(int bits, int K, int N, const uint8_t* codes, int32_t* Q, void* cuda_stream) {
    const int rc = check_format(bits, K, N);
    if (rc != QLORA_OK) return rc;
    if (K == 0 || N == 0) return QLORA_OK;
    if (codes == nullptr || Q == nullptr) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(codes) || !aligned16(Q)) return QLORA_ERR_ALIGNMENT;
    return launch_pack(bits, K, N, codes, Q, (cudaStream_t)cuda_stream);
}

int qlora_unpack(int bits, int K, int N, const int32_t* Q, uint8_t* codes, void* cuda_stream) {
    const int rc = check_format(bits, K, N);
    if (rc != QLORA_OK) return rc;
    if (K == 0 || N == 0) return QLORA_OK;
    if (codes == nullptr || Q == nullptr) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(codes) || !aligned16(Q)) return QLORA_ERR_ALIGNMENT;
    return launch_unpack(bits, K, N, Q, codes, (cudaStream_t)cuda_stream);
}

int qlora_lrec_loss(int T, int V, const void* student_logits, const void* teacher_logits, const int32_t* labels, float lambda_kl,
                    float lambda_ce, float grad_scale, float* loss_tokens, void* dlogits, void* cuda_stream) {
    if (T < 0 || V < 0) return QLORA_ERR_INVALID_ARG;
    if (V == 0 || V % 8 != 0 || V > 32768) return QLORA_ERR_UNSUPPORTED;
    if (T == 0) return QLORA_OK;
    if (!student_logits || !teacher_logits || !loss_tokens) return QLORA_ERR_INVALID_ARG;
    if (!(lambda_kl == lambda_kl) || !(lambda_ce == lambda_ce) || !(grad_scale == grad_scale)) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(student_logits) || !aligned16(teacher_logits) || !aligned16(labels) || !aligned16(loss_tokens) ||
        !aligned16(dlogits))
        return QLORA_ERR_ALIGNMENT;
    return launch_lrec_loss(T, V, student_logits, teacher_logits, labels, lambda_kl, lambda_ce, grad_scale, loss_tokens, dlogits,
                            (cudaStream_t)cuda_stream);
}

int qlora_token_logprobs(int T, int V, long long row_stride, int dtype, const void* logits, const int32_t* tokens,
                         float inv_temperature, int k, float* logprobs, float* entropy, int32_t* top_ids,
                         float* top_logprobs, float* stats, void* cuda_stream) {
    const int rc = check_logits(T, V, row_stride, dtype, inv_temperature);
    if (rc != QLORA_OK) return rc;
    if (k < 0) return QLORA_ERR_INVALID_ARG;
    if (k > QLORA_MAX_TOP || k > V) return QLORA_ERR_UNSUPPORTED;
    if (T == 0) return QLORA_OK;
    if (!logits || (!logprobs && !entropy && !top_ids && !top_logprobs && !stats)) return QLORA_ERR_INVALID_ARG;
    if ((logprobs && !tokens) || ((top_ids || top_logprobs) != (k > 0))) return QLORA_ERR_INVALID_ARG;
    if (!element_aligned(logits, dtype) || !aligned4(tokens) || !aligned16(logprobs) || !aligned16(entropy) || !aligned16(top_ids) ||
        !aligned16(top_logprobs) || !aligned16(stats))
        return QLORA_ERR_ALIGNMENT;
    return launch_token_logprobs(T, V, row_stride, dtype, logits, tokens, inv_temperature, k, logprobs, entropy, top_ids, top_logprobs, stats,
                                 (cudaStream_t)cuda_stream);
}

int qlora_token_logprobs_bwd(int T, int V, long long row_stride, int dtype, const void* logits, const int32_t* tokens,
                             float inv_temperature, const float* stats, const float* d_logprobs, const float* d_entropy,
                             long long grad_stride, void* dlogits, void* cuda_stream) {
    const int rc = check_logits(T, V, row_stride, dtype, inv_temperature);
    if (rc != QLORA_OK) return rc;
    if (T > 1 && grad_stride < V) return QLORA_ERR_INVALID_ARG;
    if (T == 0) return QLORA_OK;
    if (!logits || !stats || !dlogits || (!d_logprobs && !d_entropy) || (d_logprobs && !tokens)) return QLORA_ERR_INVALID_ARG;
    const bool in_place = logits == dlogits && (T == 1 || row_stride == grad_stride);
    if (!in_place && rows_overlap(logits, row_stride, dlogits, grad_stride, T, V, element_bytes(dtype))) return QLORA_ERR_INVALID_ARG;
    if (!element_aligned(logits, dtype) || !element_aligned(dlogits, dtype) || !aligned4(tokens) || !aligned16(stats) ||
        !aligned16(d_logprobs) || !aligned16(d_entropy))
        return QLORA_ERR_ALIGNMENT;
    return launch_token_logprobs_bwd(T, V, row_stride, dtype, logits, tokens, inv_temperature, stats, d_logprobs, d_entropy, grad_stride, dlogits,
                                     (cudaStream_t)cuda_stream);
}

int qlora_grad_norm(const qlora_adamw_desc* desc, float prescale, float max_norm, float* out, void* workspace,
                    size_t workspace_bytes, void* cuda_stream) {
    const int rc = check_adamw(desc, false);
    if (rc != QLORA_OK) return rc;
    if (!(prescale == prescale) || !(max_norm == max_norm) || !out) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(out) || !aligned16(workspace)) return QLORA_ERR_ALIGNMENT;
    if (workspace == nullptr || workspace_bytes < QLORA_GRAD_NORM_WORKSPACE_BYTES) return QLORA_ERR_WORKSPACE;
    return launch_grad_norm(*desc, prescale, max_norm, out, workspace, (cudaStream_t)cuda_stream);
}

int qlora_adamw(const qlora_adamw_desc* desc, double lr, int step, const float* lr_dev, const int32_t* step_dev,
                const float* norm, void* cuda_stream) {
    const int rc = check_adamw(desc, true);
    if (rc != QLORA_OK) return rc;
    if ((!lr_dev && !(lr - lr == 0.0)) || (!step_dev && step < 1)) return QLORA_ERR_INVALID_ARG;      // a finite rate, steps from 1
    if (!aligned16(lr_dev) || !aligned16(step_dev) || !aligned16(norm)) return QLORA_ERR_ALIGNMENT;
    return launch_adamw(*desc, lr, step, lr_dev, step_dev, norm, (cudaStream_t)cuda_stream);
}

int qlora_adapters_workspace_bytes(const qlora_adapters_desc* desc, int M, size_t* out) {
    if (out == nullptr) return QLORA_ERR_INVALID_ARG;
    const int rc = check_adapters(desc, M);
    if (rc != QLORA_OK) return rc;
    *out = adapters_bytes(*desc, M);
    return QLORA_OK;
}

// Forward: In = X [M, K], Base and Out [M, N].  Backward: In = dY [M, N], Base and Out [M, K].
static int adapters_common(bool forward, const qlora_adapters_desc* desc, int M, const void* In, const int32_t* adapter_of, const void* A, const void* B,
                           const float* scales, const void* Base, void* Out, float* low, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const int rc = check_adapters(desc, M);
    if (rc != QLORA_OK) return rc;
    const qlora_adapters_desc& d = *desc;
    const int T = forward ? d.K : d.N, C = forward ? d.N : d.K;
    if (M == 0) return QLORA_OK;
    if (!In || !adapter_of || (d.n_adapters > 0 && (!A || !B || !scales)) || !Base || !Out) return QLORA_ERR_INVALID_ARG;
    if (Base != Out && rows_overlap(Base, C, Out, C, M, C, 2)) return QLORA_ERR_INVALID_ARG;
    if (overlap(In, (size_t)M * T * 2, Out, (size_t)M * C * 2)) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(In) || !aligned4(adapter_of) || !aligned16(A) || !aligned16(B) || !aligned4(scales) || !aligned16(Base) || !aligned16(Out) ||
        !aligned16(low) || !aligned16(workspace))
        return QLORA_ERR_ALIGNMENT;
    if (workspace == nullptr || workspace_bytes < adapters_scratch_bytes(M, d.r)) return QLORA_ERR_WORKSPACE;
    return launch_adapters(forward, M, T, C, d.r, d.n_adapters, In, adapter_of, forward ? A : B, forward ? B : A, scales, Base, Out, low, workspace,
                           (cudaStream_t)cuda_stream);
}

int qlora_adapters_fwd(const qlora_adapters_desc* desc, int M, const void* X, const int32_t* adapter_of, const void* A, const void* B, const float* scales,
                       const void* Y_base, void* Y, float* H_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return adapters_common(true, desc, M, X, adapter_of, A, B, scales, Y_base, Y, H_out, workspace, workspace_bytes, cuda_stream);
}

int qlora_adapters_bwd_input(const qlora_adapters_desc* desc, int M, const void* dY, const int32_t* adapter_of, const void* A, const void* B,
                             const float* scales, const void* dX_base, void* dX, float* G_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return adapters_common(false, desc, M, dY, adapter_of, A, B, scales, dX_base, dX, G_out, workspace, workspace_bytes, cuda_stream);
}

int qlora_adapters_bwd_lora(const qlora_adapters_desc* desc, int M, const void* X, const void* dY, const int32_t* adapter_of, const void* A, const void* B,
                            const float* scales, const float* H, const float* G, float* dA, float* dB, int accumulate, void* workspace,
                            size_t workspace_bytes, void* cuda_stream) {
    int rc = check_adapters(desc, M);
    if (rc != QLORA_OK) return rc;
    if (accumulate != 0 && accumulate != 1) return QLORA_ERR_INVALID_ARG;
    const qlora_adapters_desc& d = *desc;
    if (d.n_adapters == 0) return QLORA_OK;
    if (!dA || !dB || !scales) return QLORA_ERR_INVALID_ARG;
    if (M > 0 && (!X || !dY || !adapter_of || (!H && !A) || (!G && !B))) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(dY) || !aligned4(adapter_of) || !aligned16(A) || !aligned16(B) || !aligned4(scales) || !aligned16(H) || !aligned16(G) ||
        !aligned16(dA) || !aligned16(dB) || !aligned16(workspace))
        return QLORA_ERR_ALIGNMENT;
    if (workspace == nullptr || workspace_bytes < adapters_bytes(d, M)) return QLORA_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    void* scratch = static_cast<char*>(workspace) + 2 * adapters_low_bytes(d, M);   // (the gradients' is the larger)
    if (M > 0 && !H) {
        float* Hs = static_cast<float*>(workspace);
        rc = launch_adapters(true, M, d.K, 0, d.r, d.n_adapters, X, adapter_of, A, nullptr, scales, nullptr, nullptr, Hs, scratch, st);
        if (rc != QLORA_OK) return rc;
        H = Hs;
    }
    if (M > 0 && !G) {
        float* Gs = reinterpret_cast<float*>(static_cast<char*>(workspace) + adapters_low_bytes(d, M));
        rc = launch_adapters(false, M, d.N, 0, d.r, d.n_adapters, dY, adapter_of, B, nullptr, scales, nullptr, nullptr, Gs, scratch, st);
        if (rc != QLORA_OK) return rc;
        G = Gs;
    }
    return launch_adapters_grads(M, d.K, d.N, d.r, d.n_adapters, X, dY, adapter_of, scales, H, G, dA, dB, accumulate, scratch, st);
}

static int check_head(int T, int V, int D) {
    if (T < 0 || V < 0 || D < 0) return QLORA_ERR_INVALID_ARG;
    if (T > (1 << 24) || V == 0 || V > (1 << 24) || D < 64 || D % 8 != 0 || D > (1 << 20)) return QLORA_ERR_UNSUPPORTED;
    if (((long long)T / 256 + 1) * ((long long)V / 256 + 1 + D / 256 + 1) > (1 << 28)) return QLORA_ERR_UNSUPPORTED;   // (items of work are counted in 32 bits)
    return QLORA_OK;
}

int qlora_head_loss_workspace_bytes(int T, int V, int D, int gradient, size_t* out) {
    if (out == nullptr || (gradient != 0 && gradient != 1)) return QLORA_ERR_INVALID_ARG;
    const int rc = check_head(T, V, D);
    if (rc != QLORA_OK) return rc;
    *out = head_loss_workspace_bytes(T > 0 ? T : 1, V, D, gradient != 0);
    return QLORA_OK;
}

int qlora_head_loss(int T, int V, int D, const void* hidden, const void* head, const int32_t* labels, const float* d_loss, float* loss_tokens,
                    void* d_hidden, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const int rc = check_head(T, V, D);
    if (rc != QLORA_OK) return rc;
    if (T == 0) return QLORA_OK;
    if (!hidden || !head || !labels || !loss_tokens || (d_hidden != nullptr) != (d_loss != nullptr)) return QLORA_ERR_INVALID_ARG;
    if (d_hidden != nullptr && d_hidden != hidden && rows_overlap(hidden, D, d_hidden, D, T, D, 2)) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(hidden) || !aligned16(head) || !aligned4(labels) || !aligned4(d_loss) || !aligned4(loss_tokens) || !aligned16(d_hidden) || !aligned16(workspace))
        return QLORA_ERR_ALIGNMENT;
    if (d_loss != nullptr && overlap(d_loss, (size_t)T * 4, loss_tokens, (size_t)T * 4)) return QLORA_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < head_loss_workspace_bytes(T, V, D, d_hidden != nullptr)) return QLORA_ERR_WORKSPACE;
    return launch_head_loss(T, V, D, hidden, head, labels, d_loss, loss_tokens, d_hidden, workspace, (cudaStream_t)cuda_stream);
}

int qlora_gather_columns(int elem_bytes, int rows, int cols, const void* in, const int32_t* perm, void* out, void* cuda_stream) {
    if (rows < 0 || cols < 0) return QLORA_ERR_INVALID_ARG;
    if (elem_bytes != 2 && elem_bytes != 4) return QLORA_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return QLORA_OK;
    if (!in || !perm || !out || in == out) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(in) || !aligned16(perm) || !aligned16(out)) return QLORA_ERR_ALIGNMENT;
    return launch_gather_columns(elem_bytes, rows, cols, in, perm, out, (cudaStream_t)cuda_stream);
}

int qlora_dequant(const qlora_desc* desc, const int32_t* Q, const void* scales, const void* zeros, void* W,
                  void* cuda_stream) {
    const int rc = check_desc(desc, false);
    if (rc != QLORA_OK) return rc;
    if (desc->K == 0 || desc->N == 0) return QLORA_OK;
    if (!Q || !scales || !zeros || !W) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(Q) || !aligned16(scales) || !aligned16(zeros) || !aligned16(W)) return QLORA_ERR_ALIGNMENT;
    return launch_dequant(*desc, Q, scales, zeros, W, (cudaStream_t)cuda_stream);
}

int qlora_quantize_rtn(const qlora_desc* desc, const float* W, int32_t* Q, void* scales, void* zeros, void* cuda_stream) {
    const int rc = check_desc(desc, false);
    if (rc != QLORA_OK) return rc;
    if (desc->K == 0 || desc->N == 0) return QLORA_OK;
    if (!W || !Q || !scales || !zeros) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(W) || !aligned16(Q) || !aligned16(scales) || !aligned16(zeros)) return QLORA_ERR_ALIGNMENT;
    if ((long long)desc->K / desc->group_size > 65535) return QLORA_ERR_UNSUPPORTED;
    return launch_quantize_rtn(*desc, W, Q, scales, zeros, (cudaStream_t)cuda_stream);
}

// mask == NULL: the plain layer.  Otherwise LoRA dropout: the branch sees keep_scale * mask (.) X.
static int fwd_common(const qlora_desc* desc, int M, const void* X, const uint8_t* mask, float keep_scale, const int32_t* Q,
                      const void* scales, const void* zeros, const void* A, const void* B, void* Y, float* H_out,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
    int rc = check_desc(desc, true);
    if (rc != QLORA_OK) return rc;
    if (M < 0) return QLORA_ERR_INVALID_ARG;
    const qlora_desc& d = *desc;
    if (M == 0 || d.N == 0) return QLORA_OK;
    if (!X || !Q || !scales || !zeros || !Y) return QLORA_ERR_INVALID_ARG;
    if (d.r > 0 && (!A || !B)) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(Q) || !aligned16(scales) || !aligned16(zeros) || !aligned16(Y) ||
        !aligned16(A) || !aligned16(B) || !aligned16(H_out) || !aligned16(workspace))
        return QLORA_ERR_ALIGNMENT;
    const Workspace w = carve(d, M);
    if (workspace == nullptr || workspace_bytes < w.required) return QLORA_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    float* H = H_out ? H_out : reinterpret_cast<float*>(static_cast<char*>(workspace) + w.p0_off);
    unsigned int* sync = reinterpret_cast<unsigned int*>(static_cast<char*>(workspace) + w.sync_off);
    if (stream_supported(d, M, false)) {                              // up to 16 tokens: the weight-streaming kernels
        const bool fused = d.r > 0 && d.r <= 16 && mask == nullptr;   // the down-projection rides along inside the kernel
        if (d.r > 0 && !fused) {
            rc = launch_lora_down(M, d.K, d.r, true, X, A, H, st, mask, keep_scale);
            if (rc != QLORA_OK) return rc;
        }
        return launch_stream_gemm(d, M, false, X, Q, scales, zeros, A, B, H, !fused, Y, st);
    }
    // the tensor-core path computes H itself when given A (beside its tiles where SM pairs are idle, else ahead of them)
    const DownExtra dropout{mask, keep_scale, 0};
    if (umma_supported(d, M)) return launch_umma_gemm(d, M, false, X, Q, scales, zeros, B, H, Y, st, d.r > 0 ? A : nullptr, sync, static_cast<char*>(workspace) + w.split_off,
                                workspace_bytes - w.split_off, nullptr, mask != nullptr ? &dropout : nullptr);
    if (d.r > 0) {
        rc = launch_lora_down(M, d.K, d.r, true, X, A, H, st, mask, keep_scale);
        if (rc != QLORA_OK) return rc;
    }
    return launch_simt_gemm(d, M, false, X, Q, scales, zeros, B, H, Y, st);
}

// mask == NULL: the plain layer.  Otherwise LoRA dropout: the LoRA term of dX is keep_scale * mask (.) (s G A); the dense
// kernels then run without the branch (rank 0) and an elementwise pass adds the masked term.
static int bwd_input_common(const qlora_desc* desc, int M, const void* dY, const uint8_t* mask, float keep_scale,
                            const int32_t* Q, const void* scales, const void* zeros, const void* A, const void* B, void* dX,
                            float* G_out, void* workspace, size_t workspace_bytes, void* cuda_stream, DbFuse* db = nullptr) {
    int rc = check_desc(desc, true);
    if (rc != QLORA_OK) return rc;
    if (M < 0) return QLORA_ERR_INVALID_ARG;
    const qlora_desc& d = *desc;
    if (M == 0 || d.K == 0) return QLORA_OK;
    if (!dY || !Q || !scales || !zeros || !dX) return QLORA_ERR_INVALID_ARG;
    if (d.r > 0 && (!A || !B)) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(dY) || !aligned16(Q) || !aligned16(scales) || !aligned16(zeros) || !aligned16(dX) ||
        !aligned16(A) || !aligned16(B) || !aligned16(G_out) || !aligned16(workspace))
        return QLORA_ERR_ALIGNMENT;
    const Workspace w = carve(d, M);
    if (workspace == nullptr || workspace_bytes < w.required) return QLORA_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    float* G = G_out ? G_out : reinterpret_cast<float*>(static_cast<char*>(workspace) + w.p0_off);
    if (mask != nullptr && d.r > 0) {
        qlora_desc d0 = d;
        d0.r = 0;
        if (!stream_supported(d0, M, true) && umma_supported(d0, M)) {       // G beside the tiles where SM pairs are idle, else ahead of them
            const DownExtra g_only{nullptr, 1.0f, d.r};
            rc = launch_umma_gemm(d0, M, true, dY, Q, scales, zeros, A, G, dX, st, B, nullptr, nullptr, 0, nullptr, &g_only);
        } else {
            rc = launch_lora_down(M, d.N, d.r, false, dY, B, G, st);
            if (rc != QLORA_OK) return rc;
            rc = stream_supported(d0, M, true) ? launch_stream_gemm(d0, M, true, dY, Q, scales, zeros, B, A, G, true, dX, st)
                                               : launch_simt_gemm(d0, M, true, dY, Q, scales, zeros, A, G, dX, st);
        }
        if (rc != QLORA_OK) return rc;
        return launch_lora_masked_update(M, d.K, d.r, keep_scale * d.alpha / (float)d.r, G, A, mask, dX, st);
    }
    if (stream_supported(d, M, true)) {
        const bool fused = d.r > 0 && d.r <= 16;
        if (d.r > 0 && !fused) {
            rc = launch_lora_down(M, d.N, d.r, false, dY, B, G, st);
            if (rc != QLORA_OK) return rc;
        }
        return launch_stream_gemm(d, M, true, dY, Q, scales, zeros, B, A, G, !fused, dX, st);
    }
    unsigned int* sync = reinterpret_cast<unsigned int*>(static_cast<char*>(workspace) + w.sync_off);
    if (umma_supported(d, M)) {                                        // computes G (and takes dB on where it can)
        const size_t split_bytes = workspace_bytes < w.db_off ? workspace_bytes - w.split_off : w.db_off - w.split_off;
        if (db != nullptr) {
            db->part = reinterpret_cast<float*>(static_cast<char*>(workspace) + w.db_off);
            db->part_bytes = workspace_bytes > w.db_off ? workspace_bytes - w.db_off : 0;
        }
        return launch_umma_gemm(d, M, true, dY, Q, scales, zeros, A, G, dX, st, B, sync, static_cast<char*>(workspace) + w.split_off,
                                split_bytes, db);
    }
    if (d.r > 0) {
        rc = launch_lora_down(M, d.N, d.r, false, dY, B, G, st);
        if (rc != QLORA_OK) return rc;
    }
    return launch_simt_gemm(d, M, true, dY, Q, scales, zeros, A, G, dX, st);
}

// mask == NULL: the plain layer.  Otherwise LoRA dropout: H (if recomputed) and dA use keep_scale * mask (.) X.
static int bwd_lora_common(const qlora_desc* desc, int M, const void* X, const uint8_t* mask, float keep_scale, const void* dY,
                           const void* A, const void* B, const float* H, const float* G, float* dA, float* dB, int accumulate,
                           void* workspace, size_t workspace_bytes, void* cuda_stream) {
    int rc = check_desc(desc, true);
    if (rc != QLORA_OK) return rc;
    if (M < 0 || (accumulate != 0 && accumulate != 1)) return QLORA_ERR_INVALID_ARG;
    const qlora_desc& d = *desc;
    if (d.r == 0) return QLORA_OK;
    if (!dA) return QLORA_ERR_INVALID_ARG;
    const bool want_dB = dB != nullptr;                     // NULL: dB was computed by qlora_bwd_input_db; only dA is wanted
    if (M > 0 && (!X || (!dY && (want_dB || !G)))) return QLORA_ERR_INVALID_ARG;
    if (M > 0 && ((want_dB && !H && !A) || (!G && !B))) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(X) || !aligned16(dY) || !aligned16(A) || !aligned16(B) || !aligned16(H) || !aligned16(G) ||
        !aligned16(dA) || !aligned16(dB) || !aligned16(workspace))
        return QLORA_ERR_ALIGNMENT;
    const Workspace w = carve(d, M);
    if (workspace == nullptr || workspace_bytes < w.required) return QLORA_ERR_WORKSPACE;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    char* ws = static_cast<char*>(workspace);
    const float s = d.alpha / (float)d.r;
    if (M > 0 && !H && want_dB) {
        float* Hs = reinterpret_cast<float*>(ws + w.p0_off);
        rc = launch_lora_down(M, d.K, d.r, true, X, A, Hs, st, mask, keep_scale);
        if (rc != QLORA_OK) return rc;
        H = Hs;
    }
    if (M > 0 && !G) {
        float* Gs = reinterpret_cast<float*>(ws + w.p1_off);
        rc = launch_lora_down(M, d.N, d.r, false, dY, B, Gs, st);
        if (rc != QLORA_OK) return rc;
        G = Gs;
    }
    return launch_lora_grads(M, d.K, d.N, d.r, s, X, dY, H, G, dA, dB, accumulate, ws + w.grad_off, st, mask, keep_scale, want_dB ? 3 : 2);
}

static int check_dropout(const void* mask, float keep_scale, int M) {
    if (M > 0 && mask == nullptr) return QLORA_ERR_INVALID_ARG;
    if (!(keep_scale >= 1.0f) || !(keep_scale < 1e6f)) return QLORA_ERR_INVALID_ARG;   // 1 / (1 - p), p in [0, 1)
    if (!aligned16(mask)) return QLORA_ERR_ALIGNMENT;
    return QLORA_OK;
}

int qlora_fwd(const qlora_desc* desc, int M, const void* X, const int32_t* Q, const void* scales, const void* zeros,
              const void* A, const void* B, void* Y, float* H_out, void* workspace, size_t workspace_bytes,
              void* cuda_stream) {
    return fwd_common(desc, M, X, nullptr, 1.0f, Q, scales, zeros, A, B, Y, H_out, workspace, workspace_bytes, cuda_stream);
}

int qlora_bwd_input(const qlora_desc* desc, int M, const void* dY, const int32_t* Q, const void* scales,
                    const void* zeros, const void* A, const void* B, void* dX, float* G_out, void* workspace,
                    size_t workspace_bytes, void* cuda_stream) {
    return bwd_input_common(desc, M, dY, nullptr, 1.0f, Q, scales, zeros, A, B, dX, G_out, workspace, workspace_bytes, cuda_stream);
}

int qlora_bwd_input_db(const qlora_desc* desc, int M, const void* dY, const int32_t* Q, const void* scales,
                       const void* zeros, const void* A, const void* B, const float* H, void* dX, float* G_out, float* dB,
                       int accumulate, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (desc == nullptr) return QLORA_ERR_INVALID_ARG;
    if (accumulate != 0 && accumulate != 1) return QLORA_ERR_INVALID_ARG;
    if (desc->r > 0 && M > 0 && (!H || !dB)) return QLORA_ERR_INVALID_ARG;
    if (!aligned16(H) || !aligned16(dB)) return QLORA_ERR_ALIGNMENT;
    DbFuse db{H, dB, accumulate, nullptr, 0, false};
    int rc = bwd_input_common(desc, M, dY, nullptr, 1.0f, Q, scales, zeros, A, B, dX, G_out, workspace, workspace_bytes, cuda_stream,
                              desc->r > 0 ? &db : nullptr);
    if (rc != QLORA_OK || desc->r == 0 || db.done || M < 0) return rc;
    // the backward kernel of this shape has no producer clusters to do it: dB by the LoRA-gradient kernels (dY is read again)
    const qlora_desc& d = *desc;
    if (d.N == 0) return QLORA_OK;
    const Workspace w = carve(d, M);
    return launch_lora_grads(M, d.K, d.N, d.r, d.alpha / (float)d.r, nullptr, dY, H, nullptr, nullptr, dB, accumulate,
                             static_cast<char*>(workspace) + w.grad_off, (cudaStream_t)cuda_stream, nullptr, 1.0f, 1);
}

int qlora_bwd_input_db_on_producers(const qlora_desc* desc, int M) {
    const int rc = check_desc(desc, true);
    if (rc != QLORA_OK) return rc;
    if (M < 0) return QLORA_ERR_INVALID_ARG;
    return umma_db_on_producers(*desc, M) > 0 ? 1 : 0;
}

int qlora_bwd_lora(const qlora_desc* desc, int M, const void* X, const void* dY, const void* A, const void* B,
                   const float* H, const float* G, float* dA, float* dB, int accumulate, void* workspace,
                   size_t workspace_bytes, void* cuda_stream) {
    return bwd_lora_common(desc, M, X, nullptr, 1.0f, dY, A, B, H, G, dA, dB, accumulate, workspace, workspace_bytes, cuda_stream);
}

int qlora_fwd_dropout(const qlora_desc* desc, int M, const void* X, const uint8_t* mask, float keep_scale, const int32_t* Q,
                      const void* scales, const void* zeros, const void* A, const void* B, void* Y, float* H_out,
                      void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const int rc = check_dropout(mask, keep_scale, M);
    if (rc != QLORA_OK) return rc;
    return fwd_common(desc, M, X, mask, keep_scale, Q, scales, zeros, A, B, Y, H_out, workspace, workspace_bytes, cuda_stream);
}

int qlora_bwd_input_dropout(const qlora_desc* desc, int M, const void* dY, const uint8_t* mask, float keep_scale,
                            const int32_t* Q, const void* scales, const void* zeros, const void* A, const void* B, void* dX,
                            float* G_out, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const int rc = check_dropout(mask, keep_scale, M);
    if (rc != QLORA_OK) return rc;
    return bwd_input_common(desc, M, dY, mask, keep_scale, Q, scales, zeros, A, B, dX, G_out, workspace, workspace_bytes, cuda_stream);
}

int qlora_bwd_lora_dropout(const qlora_desc* desc, int M, const void* X, const uint8_t* mask, float keep_scale, const void* dY,
                           const void* A, const void* B, const float* H, const float* G, float* dA, float* dB, int accumulate,
                           void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const int rc = check_dropout(mask, keep_scale, M);
    if (rc != QLORA_OK) return rc;
    return bwd_lora_common(desc, M, X, mask, keep_scale, dY, A, B, H, G, dA, dB, accumulate, workspace, workspace_bytes, cuda_stream);
}

}  // extern "C"
