// Gradient lists: the plan that turns n nodes' lists of parameter gradients into pieces of equal work,
// its checks, and the entry points of the norm and the clipping.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>

#include "dlm_gradients.h"
#include "dlm_internal.h"
#include "dlm_launch.h"

namespace {

// Any array longer than this could not exist on the device; keeps the arithmetic of the checks in range.
constexpr int64_t kMaxElements = (int64_t)1 << 42;

int64_t element_bytes(int dtype) { return dtype == DLM_G_BF16 ? 2 : 4; }

// Bytes per piece.  32 KB give each of the 256 threads of a CTA 128 bytes to ask for at once; lists too small to give every
// SM four CTAs of that size are cut finer, down to 4 KB.
int64_t piece_bytes(int64_t total, int sms) {
    int64_t e = 32768;
    while (e > 4096 && e * 4 * std::max(1, sms) > total) e /= 2;
    return e;
}

template <typename T>
bool upload(T** dev, const std::vector<T>& host) {
    return cudaMalloc((void**)dev, host.size() * sizeof(T)) == cudaSuccess &&
           cudaMemcpy(*dev, host.data(), host.size() * sizeof(T), cudaMemcpyHostToDevice) == cudaSuccess;
}

int build(int n, int tensors, const int64_t* sizes, const int* dtypes, const void* const* data, const int64_t* offsets,
          dlm_gradients& list) {
    list.n = n;
    list.tensors = tensors;
    list.types = dtypes[0];
    list.offsets.resize(tensors);
    int64_t total = 0;
    std::vector<std::pair<int64_t, int64_t>> spans;
    for (int t = 0; t < tensors; ++t) {
        if (dtypes[t] != DLM_G_F32 && dtypes[t] != DLM_G_BF16) return DLM_ERR_KIND;
        if (sizes[t] < 0 || sizes[t] > kMaxElements || (offsets && (offsets[t] < 0 || offsets[t] > kMaxElements)))
            return DLM_ERR_SHAPE;
        list.offsets[t] = offsets ? offsets[t] : total;
        total += sizes[t];
        if (total > kMaxElements) return DLM_ERR_SHAPE;
        if (dtypes[t] != dtypes[0]) list.types = -1;
        if (sizes[t] > 0) {
            spans.push_back({list.offsets[t], list.offsets[t] + sizes[t]});
            list.columns = std::max(list.columns, list.offsets[t] + sizes[t]);
        }
    }
    list.elements = total;
    std::sort(spans.begin(), spans.end());
    for (size_t k = 1; k < spans.size(); ++k)
        if (spans[k].first < spans[k - 1].second) return DLM_ERR_ALIAS;  // two tensors claim a column
    for (int i = 0; i < n; ++i)
        for (int t = 0; t < tensors; ++t) {
            if (sizes[t] == 0) continue;
            const uintptr_t p = (uintptr_t)data[(size_t)i * tensors + t];
            if (!p) return DLM_ERR_NULL;
            if (p % element_bytes(dtypes[t])) return DLM_ERR_ALIGN;
            list.sources.push_back({p, p + (uintptr_t)(sizes[t] * element_bytes(dtypes[t]))});
        }
    std::sort(list.sources.begin(), list.sources.end());
    for (size_t k = 1; k < list.sources.size(); ++k)
        if (list.sources[k].first < list.sources[k - 1].second) return DLM_ERR_ALIAS;  // clipping in place would scale twice

    int devices = 0;
    if (cudaGetDeviceCount(&devices) != cudaSuccess || devices == 0) {
        cudaGetLastError();
        return DLM_OK;  // host-only handle: the layout can be read
    }
    if (cudaGetDevice(&list.device) != cudaSuccess) return DLM_ERR_CUDA;
    const dlm::DeviceInfo& info = dlm::device_info();
    if (!info.ok) return DLM_ERR_CUDA;
    int64_t per_node = 0;
    for (int t = 0; t < tensors; ++t) list.bytes += sizes[t] * element_bytes(dtypes[t]);
    const int64_t step_bytes = piece_bytes(list.bytes * n, info.sms);
    auto step_of = [&](int t) { return step_bytes / element_bytes(dtypes[t]); };
    // Pieces are cut where the source's addresses are multiples of 16 bytes, so that all but a tensor's ends are whole
    // 16-byte runs: a tensor that starts `skew` elements above such an address has its cuts that much earlier.  Every node
    // gets the same number of pieces, of which the last may be empty.
    auto most = [&](int t) { return 16 / element_bytes(dtypes[t]) - 1; };
    for (int t = 0; t < tensors; ++t)
        if (sizes[t] > 0) per_node += (sizes[t] + most(t) + step_of(t) - 1) / step_of(t);
    if (per_node * n > 0x3fffffff) return DLM_ERR_UNSUPPORTED;
    list.pieces = (int)per_node;
    std::vector<dlm_piece> pieces;
    pieces.reserve((size_t)per_node * n);
    for (int i = 0; i < n; ++i)
        for (int t = 0; t < tensors; ++t) {
            if (sizes[t] == 0) continue;
            const char* src = static_cast<const char*>(data[(size_t)i * tensors + t]);
            const int64_t e = element_bytes(dtypes[t]), step = step_of(t), skew = (int64_t)((uintptr_t)src % 16) / e;
            const int64_t parts = (sizes[t] + most(t) + step - 1) / step;
            for (int64_t k = 0; k < parts; ++k) {
                const int64_t lo = std::min(sizes[t], std::max<int64_t>(0, k * step - skew)), hi = std::min(sizes[t], (k + 1) * step - skew);
                pieces.push_back({src + lo * e, list.offsets[t] + lo, (int32_t)(hi - lo), dtypes[t] == DLM_G_BF16});
            }
        }
    if (pieces.empty()) return DLM_OK;
    if (!upload(&list.d_pieces, pieces)) return DLM_ERR_CUDA;
    if (total > DLM_SMALL_NODE) {
        if (cudaMalloc((void**)&list.d_scale, n * sizeof(float)) != cudaSuccess ||
            cudaMalloc((void**)&list.d_partial, (size_t)n * DLM_CLIP_CTAS_PER_SM * info.sms * DLM_CLIP_WARPS * sizeof(double)) != cudaSuccess) return DLM_ERR_CUDA;
    }
    return dlm::finish_uploads() ? DLM_OK : DLM_ERR_CUDA;
}

bool meets_a_source(const dlm_gradients& list, uintptr_t lo, uintptr_t hi) {
    // first source that ends after lo; the list is ascending and disjoint
    auto it = std::upper_bound(list.sources.begin(), list.sources.end(), lo,
                               [](uintptr_t v, const std::pair<uintptr_t, uintptr_t>& r) { return v < r.second; });
    return it != list.sources.end() && it->first < hi;
}

int check_call(const dlm_gradients* list, int kind, const float* norms) {
    if (!list || !norms) return DLM_ERR_NULL;
    if (kind != DLM_NORM_L2 && kind != DLM_NORM_MAX) return DLM_ERR_KIND;
    if ((uintptr_t)norms % 4) return DLM_ERR_ALIGN;
    if (meets_a_source(*list, (uintptr_t)norms, (uintptr_t)norms + (size_t)list->n * 4)) return DLM_ERR_ALIAS;
    int dev = -1;
    if (list->device < 0 || cudaGetDevice(&dev) != cudaSuccess || dev != list->device) return DLM_ERR_CUDA;
    return DLM_OK;
}

}  // namespace

extern "C" {

int gradients_build(int n, int tensors, const int64_t* sizes, const int* dtypes, const void* const* data,
                    const int64_t* offsets, dlm_gradients** out) {
    if (!sizes || !dtypes || !data || !out) return DLM_ERR_NULL;
    *out = nullptr;
    if (n < 1 || tensors < 1) return DLM_ERR_SHAPE;
    if (n > DLM_MAX_NODES) return DLM_ERR_UNSUPPORTED;
    dlm_gradients* list = nullptr;
    int rc = DLM_ERR_CUDA;
    try {
        list = new dlm_gradients;
        rc = build(n, tensors, sizes, dtypes, data, offsets, *list);
    } catch (...) {  // no memory for the plan
        rc = DLM_ERR_CUDA;
    }
    if (rc != DLM_OK) {
        gradients_destroy(list);
        return dlm::settled(rc);
    }
    *out = list;
    return DLM_OK;
}

int gradients_layout(const dlm_gradients* list, const int64_t** offsets, int64_t* columns) {
    if (!list) return DLM_ERR_NULL;
    if (offsets) *offsets = list->offsets.data();
    if (columns) *columns = list->columns;
    return DLM_OK;
}

int gradients_destroy(dlm_gradients* list) {
    if (!list) return DLM_OK;
    if (list->d_pieces) cudaFree(list->d_pieces);
    if (list->d_partial) cudaFree(list->d_partial);
    if (list->d_scale) cudaFree(list->d_scale);
    delete list;
    return DLM_OK;
}

int gradient_norm(dlm_gradients* list, int kind, float* norms, void* cuda_stream) {
    int rc = check_call(list, kind, norms);
    if (rc != DLM_OK) return rc;
    return dlm::settled(dlm_launch_gradients(*list, kind, 0.0f, norms, nullptr, DLM_G_F32, 0, cuda_stream));
}

int gradient_clip(dlm_gradients* list, int kind, float max_norm, float* norms, void* g, int g_dtype, int64_t ldg,
                  void* cuda_stream) {
    int rc = check_call(list, kind, norms);
    if (rc != DLM_OK) return rc;
    if (!std::isfinite(max_norm) || !(max_norm > 0.0f)) return DLM_ERR_HYPER;
    if (g) {
        if (g_dtype != DLM_G_F32 && g_dtype != DLM_G_BF16) return DLM_ERR_KIND;
        if (ldg < list->columns) return DLM_ERR_SHAPE;
        if (ldg > kMaxElements / list->n) return DLM_ERR_UNSUPPORTED;
        const size_t esz = g_dtype == DLM_G_BF16 ? 2 : 4;
        if ((uintptr_t)g % esz) return DLM_ERR_ALIGN;
        const uintptr_t lo = (uintptr_t)g, row = (uintptr_t)ldg * esz, width = (uintptr_t)list->columns * esz;
        const uintptr_t hi = lo + row * (list->n - 1) + width, nlo = (uintptr_t)norms, nhi = nlo + (size_t)list->n * 4;
        if (lo < nhi && nlo < hi) return DLM_ERR_ALIAS;
        if (meets_a_source(*list, lo, hi))  // a source between the rows (other columns of the same array) is no clash
            for (int i = 0; i < list->n; ++i)
                if (meets_a_source(*list, lo + row * i, lo + row * i + width)) return DLM_ERR_ALIAS;
    }
    return dlm::settled(dlm_launch_gradients(*list, kind, max_norm, norms, g, g_dtype, ldg, cuda_stream));
}

}  // extern "C"
