// The AdamW step over many tensors (include/tn_adamw.h): host side and C ABI. Kernels: kernels/adamw.hpp.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "../../include/tn_adamw.h"
#include "../../include/tn_fp8.h"

namespace {

#include "kernels/fp8_format.hpp"
#include "kernels/adamw.hpp"

static_assert(TN_ADAMW_BLOCK == kBlock, "states share the 8-bit format of rows");

constexpr int64_t kMostValues = int64_t(1) << 40;
constexpr int kNormGroups = 2048, kNormSums = 8192;      // workgroups of a launch of the norm, and of all of them (one each at the least)
constexpr int64_t kLaunchParts = int64_t(1) << 22;

int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, unsigned n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int launched() { return hipGetLastError() == hipSuccess ? TN_OK : TN_ERR_HIP; }
bool float_type(int32_t t) { return t == TN_DTYPE_F32 || t == TN_DTYPE_BF16; }
unsigned type_bytes(int32_t t) { return t == TN_DTYPE_F32 ? 4 : 2; }

}  // namespace

struct tn_adamw_s {
    int32_t n_tensors = 0, bits = 32;
    bool masters = false;                        // some parameter is in bf16
    std::vector<int64_t> sizes, part0;           // part0[i]: first part of tensor i; part0[n]: all parts
    TensorEntry* tensors = nullptr;              // device
    PartEntry* parts = nullptr;
    StepScalars* scalars = nullptr;
    void *first = nullptr, *second = nullptr;
    unsigned char *first_scales = nullptr, *second_scales = nullptr;
    float* master = nullptr;
    int64_t* count = nullptr;
    double beta1 = 0, beta2 = 0, eps = 0;
    uint32_t seed = 0;
    ~tn_adamw_s() {
        if (tensors) (void)hipFree(tensors);
        if (parts) (void)hipFree(parts);
        if (scalars) (void)hipFree(scalars);
    }
};

namespace {

AdamwArgs step_args(const tn_adamw_s& h) {
    AdamwArgs a{};
    a.tensors = h.tensors;
    a.parts = h.parts;
    a.first = h.first;
    a.second = h.second;
    a.first_scales = h.first_scales;
    a.second_scales = h.second_scales;
    a.master = h.master;
    a.scalars = h.scalars;
    a.beta1 = float(h.beta1);
    a.rest1 = float(1 - h.beta1);
    a.beta2 = float(h.beta2);
    a.rest2 = float(1 - h.beta2);
    a.least = h.beta1 * h.beta1 < h.beta2 ? float(std::sqrt((1 - h.beta2) * (1 - h.beta1 * h.beta1 / h.beta2)) / (1 - h.beta1)) : 0.f;
    a.eps = float(h.eps);
    return a;
}

int check_gradients(const tn_adamw_s& h, const void* const* grads, const int32_t* dtypes) {
    if (!grads || !dtypes) return TN_ERR_INVALID_ARG;
    for (int i = 0; i < h.n_tensors; ++i)
        if (!float_type(dtypes[i]) || (h.sizes[size_t(i)] && (!grads[i] || !aligned(grads[i], type_bytes(dtypes[i]))))) return TN_ERR_INVALID_ARG;
    return TN_OK;
}

// Runs of tensors whose gradients one launch takes: f(arguments, gradients, first part, parts)
template <typename F>
int for_launches(const tn_adamw_s& h, const void* const* grads, const int32_t* dtypes, F&& f) {
    int rc = TN_OK;
    for (int t0 = 0; t0 < h.n_tensors && rc == TN_OK; t0 += kLaunchTensors) {
        const int n = h.n_tensors - t0 < kLaunchTensors ? h.n_tensors - t0 : kLaunchTensors;
        Gradients g{};
        g.tensor0 = t0;
        for (int i = 0; i < n; ++i) {
            g.p[i] = grads[t0 + i];
            if (dtypes[t0 + i] == TN_DTYPE_BF16) g.bf16[i >> 5] |= 1u << (i & 31);
        }
        const int64_t p0 = h.part0[size_t(t0)], p1 = h.part0[size_t(t0 + n)];
        for (int64_t p = p0; p < p1 && rc == TN_OK; p += kLaunchParts) {
            AdamwArgs a = step_args(h);
            a.parts = h.parts + p;
            a.n_parts = p1 - p < kLaunchParts ? p1 - p : kLaunchParts;
            rc = f(a, g, p);
        }
    }
    return rc;
}

int64_t norm_launches(const tn_adamw_s& h) { return div_up(h.n_tensors, kLaunchTensors) + h.part0.back() / kLaunchParts; }
// Workgroups of a launch of the norm over these parts, as many as it has room for: launches follow each other, so that a short one is as long as what one workgroup
// does (1604 parts behind 27392 others: 16 us as a share of 2048 workgroups, 8 so)
int64_t norm_groups(const tn_adamw_s& h, int64_t parts) {
    const int64_t room = kNormSums / norm_launches(h), most = room < 1 ? 1 : room < kNormGroups ? room : kNormGroups;
    return parts < most ? parts : most;
}

int run_norm(const tn_adamw_s& h, const void* const* grads, const int32_t* dtypes, double* sums, int32_t* n_sums, hipStream_t stream) {
    int64_t done = 0;
    const int rc = for_launches(h, grads, dtypes, [&](const AdamwArgs& a, const Gradients& g, int64_t) {
        const int64_t groups = norm_groups(h, a.n_parts);
        gradient_norm_kernel<<<dim3(unsigned(groups)), dim3(256), 0, stream>>>(a, g, sums + done);
        done += groups;
        return launched();
    });
    *n_sums = int32_t(done);
    return rc;
}

int make_masters(const tn_adamw_s& h, hipStream_t stream) {
    if (!h.masters) return TN_OK;
    AdamwArgs a = step_args(h);
    a.n_parts = h.part0.back();
    const int64_t groups = a.n_parts < 4096 ? a.n_parts : 4096;
    adamw_master_kernel<<<dim3(unsigned(groups)), dim3(256), 0, stream>>>(a);
    return launched();
}

bool workspace_ok(tn_adamw_t h, const void* p, int64_t bytes) { return p && bytes >= tn_adamw_workspace(h) && aligned(p, 256); }

}  // namespace

extern "C" {

int64_t tn_adamw_state_values(int32_t n_tensors, const int64_t* sizes) {
    if (n_tensors < 1 || !sizes) return TN_ERR_INVALID_ARG;
    if (n_tensors > TN_ADAMW_MAX_TENSORS) return TN_ERR_UNSUPPORTED;
    int64_t all = 0;
    for (int i = 0; i < n_tensors; ++i) {
        if (sizes[i] < 0) return TN_ERR_INVALID_ARG;
        if (sizes[i] > kMostValues || (all += div_up(sizes[i], TN_ADAMW_BLOCK) * TN_ADAMW_BLOCK) > kMostValues) return TN_ERR_UNSUPPORTED;
    }
    return all;
}

int tn_adamw_create(tn_adamw_t* out, const tn_adamw_desc* d) {
    if (!out || !d || !d->dtypes || !d->params || !d->decays || !d->count || !aligned(d->count, 8)) return TN_ERR_INVALID_ARG;
    const int64_t values = tn_adamw_state_values(d->n_tensors, d->sizes);
    if (values < 0) return int(values);
    if ((d->state_bits != 32 && d->state_bits != 8) || !(d->beta1 >= 0 && d->beta1 < 1) || !(d->beta2 >= 0 && d->beta2 < 1) || !(d->eps >= 0)) return TN_ERR_INVALID_ARG;
    if (values > 0 && (!d->first || !d->second || !aligned(d->first, 256) || !aligned(d->second, 256))) return TN_ERR_INVALID_ARG;
    if (values > 0 && d->state_bits == 8 && (!d->first_scales || !d->second_scales)) return TN_ERR_INVALID_ARG;
    bool masters = false;
    for (int i = 0; i < d->n_tensors; ++i) {
        if (!float_type(d->dtypes[i]) || (d->sizes[i] && (!d->params[i] || !aligned(d->params[i], type_bytes(d->dtypes[i]))))) return TN_ERR_INVALID_ARG;
        masters = masters || (d->dtypes[i] == TN_DTYPE_BF16 && d->sizes[i]);
    }
    if (masters && (!d->master || !aligned(d->master, 256))) return TN_ERR_INVALID_ARG;

    tn_adamw_s* h = new (std::nothrow) tn_adamw_s;
    if (!h) return TN_ERR_ALLOC;
    int rc = TN_OK;
    std::vector<TensorEntry> tensors;
    std::vector<PartEntry> parts;
    try {
        h->sizes.assign(d->sizes, d->sizes + d->n_tensors);
        int64_t place = 0;
        for (int i = 0; i < d->n_tensors; ++i) {
            h->part0.push_back(int64_t(parts.size()));
            tensors.push_back({d->params[i], d->sizes[i], place, d->decays[i], d->dtypes[i] == TN_DTYPE_BF16});
            for (int64_t p = 0; p < div_up(d->sizes[i], kPartValues); ++p) parts.push_back({i, int32_t(p)});
            place += div_up(d->sizes[i], TN_ADAMW_BLOCK) * TN_ADAMW_BLOCK;
        }
        h->part0.push_back(int64_t(parts.size()));
    } catch (...) {
        rc = TN_ERR_ALLOC;
    }
    h->n_tensors = d->n_tensors;
    h->bits = d->state_bits;
    h->first = d->first;
    h->second = d->second;
    h->first_scales = static_cast<unsigned char*>(d->first_scales);
    h->second_scales = static_cast<unsigned char*>(d->second_scales);
    h->master = d->master;
    h->masters = masters;
    h->count = d->count;
    h->beta1 = d->beta1;
    h->beta2 = d->beta2;
    h->eps = d->eps;
    h->seed = d->seed;
    if (rc == TN_OK && (hipMalloc(reinterpret_cast<void**>(&h->tensors), tensors.size() * sizeof(TensorEntry)) != hipSuccess ||
                        hipMalloc(reinterpret_cast<void**>(&h->parts), (parts.size() + 1) * sizeof(PartEntry)) != hipSuccess ||
                        hipMalloc(reinterpret_cast<void**>(&h->scalars), sizeof(StepScalars)) != hipSuccess)) {
        (void)hipGetLastError();
        rc = TN_ERR_ALLOC;
    }
    const hipStream_t st = static_cast<hipStream_t>(d->stream);
    if (rc == TN_OK && (hipMemcpyAsync(h->tensors, tensors.data(), tensors.size() * sizeof(TensorEntry), hipMemcpyHostToDevice, st) != hipSuccess ||
                        (!parts.empty() && hipMemcpyAsync(h->parts, parts.data(), parts.size() * sizeof(PartEntry), hipMemcpyHostToDevice, st) != hipSuccess)))
        rc = TN_ERR_HIP;
    if (rc == TN_OK && d->init_master) rc = make_masters(*h, st);
    if (hipStreamSynchronize(st) != hipSuccess && rc == TN_OK) rc = TN_ERR_HIP;       // (the host's arrays go out of scope)
    if (rc != TN_OK) {
        delete h;
        return rc;
    }
    *out = h;
    return TN_OK;
}

int64_t tn_adamw_workspace(tn_adamw_t h) {
    if (!h) return TN_ERR_INVALID_ARG;
    return (kNormSums + norm_launches(*h)) * int64_t(sizeof(double));
}

int tn_adamw_gradient_norm(tn_adamw_t h, const void* const* grads, const int32_t* grad_dtypes, float* norm, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!h || !norm || !aligned(norm, 4) || !workspace_ok(h, workspace, workspace_bytes)) return TN_ERR_INVALID_ARG;
    int rc = check_gradients(*h, grads, grad_dtypes);
    if (rc != TN_OK) return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    PrepareArgs p{};
    p.sums = static_cast<double*>(workspace);
    p.norm = norm;
    rc = run_norm(*h, grads, grad_dtypes, static_cast<double*>(workspace), &p.n_sums, st);
    if (rc != TN_OK) return rc;
    adamw_prepare_kernel<<<dim3(1), dim3(1024), 0, st>>>(p);
    return launched();
}

int tn_adamw_step(tn_adamw_t h, const void* const* grads, const int32_t* grad_dtypes, double lr, const float* lr_device, double max_norm, float* norm,
                  int32_t norm_given, void* workspace, int64_t workspace_bytes, void* stream) {
    if (!h || !aligned(norm, 4) || !aligned(lr_device, 4) || max_norm != max_norm || (!lr_device && !(lr >= 0 && lr < 1e30))) return TN_ERR_INVALID_ARG;
    const bool clip = max_norm > 0, sums = clip && !norm_given;
    if ((clip && norm_given && !norm) || (sums && !workspace_ok(h, workspace, workspace_bytes))) return TN_ERR_INVALID_ARG;
    int rc = check_gradients(*h, grads, grad_dtypes);
    if (rc != TN_OK) return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    PrepareArgs p{};
    p.scalars = h->scalars;
    p.count = h->count;
    p.lr = lr;
    p.lr_device = lr_device;
    p.max_norm = max_norm;
    p.beta1 = h->beta1;
    p.beta2 = h->beta2;
    p.seed = h->seed;
    if (clip) p.norm = norm;
    if (sums) {
        p.sums = static_cast<double*>(workspace);
        rc = run_norm(*h, grads, grad_dtypes, static_cast<double*>(workspace), &p.n_sums, st);
        if (rc != TN_OK) return rc;
    }
    adamw_prepare_kernel<<<dim3(1), dim3(sums ? 1024 : 64), 0, st>>>(p);
    rc = launched();
    if (rc != TN_OK) return rc;
    return for_launches(*h, grads, grad_dtypes, [&](const AdamwArgs& a, const Gradients& g, int64_t) {
        const dim3 grid(unsigned(a.n_parts));
        if (h->bits == 32) adamw_step_kernel<32><<<grid, dim3(256), 0, st>>>(a, g);
        else adamw_step_kernel<8><<<grid, dim3(256), 0, st>>>(a, g);
        return launched();
    });
}

int tn_adamw_reset_master(tn_adamw_t h, void* stream) {
    if (!h) return TN_ERR_INVALID_ARG;
    return make_masters(*h, static_cast<hipStream_t>(stream));
}

int tn_adamw_destroy(tn_adamw_t h) {
    delete h;
    return TN_OK;
}

}  // extern "C"
