// extern "C" boundary of the operators around the products: argument checks.  Everything the kernels assume of sizes,
// types, pitches and addresses is established here, before any HIP call.
#include <cmath>
#include <exception>
#include <new>

#include "operators.h"

namespace {

using sparsert::set_error;

constexpr int64_t kProblemBytes = 1ll << 31;   // kernels address one problem's matrix with 32-bit byte offsets
constexpr int32_t kMaxRank = 256, kMost = 1 << 28;   // (a vector of floats as long stays under that, too)

int size_of(int32_t dtype) { return dtype == SPARSERT_F32 ? 4 : dtype == SPARSERT_F16 ? 2 : 1; }
bool floating(int32_t dtype) { return dtype == SPARSERT_F32 || dtype == SPARSERT_F16; }

template <typename... P> bool misaligned(uintptr_t mask, P... p) { return ((... | reinterpret_cast<uintptr_t>(p)) & mask) != 0; }

int check_sizes(int32_t rows, int32_t N, int32_t &batch, const int32_t *reserved, int n) {
    if (rows < 1 || N < 1) return set_error(SPARSERT_EINVAL, "sizes must be positive");
    if (rows >= kMost || N >= kMost) return set_error(SPARSERT_EUNSUPPORTED, "2^28 rows or tokens, or more");
    if (batch < 0 || batch > 65535) return set_error(SPARSERT_EINVAL, "batch must be 0..65535");
    if (batch == 0) batch = 1;
    for (int i = 0; i < n; ++i)
        if (reserved[i]) return set_error(SPARSERT_EINVAL, "reserved fields must be zero");
    return SPARSERT_OK;
}

int check_pitch(int32_t &ld, int32_t rows, int32_t N, int size, const char *name) {
    if (ld == 0) ld = N;
    if (ld < N) return set_error(SPARSERT_EINVAL, std::string(name) + " must be 0 or at least N");
    if ((int64_t)rows * ld * size >= kProblemBytes) return set_error(SPARSERT_EUNSUPPORTED, std::string("a matrix of 2 GiB or more (rows x ") + name + ")");
    return SPARSERT_OK;
}

int check_stream(void *stream) {
    return sparsert::stream_of_current_device(stream) ? SPARSERT_OK : set_error(SPARSERT_EINVAL, "the stream is not one of the current HIP device");
}

int check_norm(sparsert_norm &d) {
    if (int rc = check_sizes(d.K, d.N, d.batch, d.reserved, 3)) return rc;
    if (!floating(d.dtype)) return set_error(SPARSERT_EINVAL, "dtype must be F32 or F16");
    if (d.out_dtype != d.dtype && d.out_dtype != SPARSERT_I8) return set_error(SPARSERT_EINVAL, "out_dtype must be dtype or I8");
    if (!(d.eps > 0.0f) || !std::isfinite(d.eps)) return set_error(SPARSERT_EINVAL, "eps must be positive and finite");
    if (int rc = check_pitch(d.ldx, d.K, d.N, size_of(d.dtype), "ldx")) return rc;
    if (int rc = check_pitch(d.ldh, d.K, d.N, size_of(d.dtype), "ldh")) return rc;
    return check_pitch(d.ldy, d.K, d.N, size_of(d.out_dtype), "ldy");
}

int check_set(sparsert_adapter_set &d) {
    if (int rc = check_sizes(d.M, d.N, d.batch, d.reserved, 3)) return rc;
    if (int rc = check_sizes(d.K, d.N, d.batch, d.reserved, 0)) return rc;
    if (!floating(d.dtype)) return set_error(SPARSERT_EINVAL, "dtype must be F32 or F16");
    if (d.x_dtype != d.dtype && d.x_dtype != SPARSERT_I8) return set_error(SPARSERT_EINVAL, "x_dtype must be dtype or I8");
    if (d.rank < 1 || d.rank > kMaxRank) return set_error(SPARSERT_EINVAL, "rank must be 1..256");
    if (d.count < 1) return set_error(SPARSERT_EINVAL, "count must be positive");
    const int c_size = d.x_dtype == SPARSERT_I8 ? 4 : size_of(d.dtype);
    if (int rc = check_pitch(d.ldx, d.K, d.N, size_of(d.x_dtype), "ldx")) return rc;
    if (int rc = check_pitch(d.ldc, d.M, d.N, c_size, "ldc")) return rc;
    if (int rc = check_pitch(d.ldy, d.M, d.N, size_of(d.dtype), "ldy")) return rc;
    if ((int64_t)d.rank * (d.M > d.K ? d.M : d.K) * size_of(d.dtype) >= kProblemBytes) return set_error(SPARSERT_EUNSUPPORTED, "an adapter of 2 GiB or more");
    if ((int64_t)d.batch * d.N >= (1ll << 31)) return set_error(SPARSERT_EUNSUPPORTED, "2^31 tokens or more");
    return SPARSERT_OK;
}

// No exception crosses the C boundary (an error message may find no memory).
template <typename F> int guarded(F f) {
    try {
        std::string err;
        const int rc = f(err);
        return rc == SPARSERT_OK ? rc : err.empty() ? rc : set_error(rc, err);
    } catch (const std::bad_alloc &) {
        return SPARSERT_ENOMEM;
    } catch (const std::exception &) {
        return SPARSERT_EINVAL;
    }
}

}  // namespace

extern "C" {

int sparsert_rms_norm_workspace(const sparsert_norm *norm, size_t *bytes) {
    return guarded([&](std::string &) {
        if (!norm || !bytes) return set_error(SPARSERT_EINVAL, "norm or bytes is NULL");
        *bytes = 0;
        sparsert_norm d = *norm;
        if (int rc = check_norm(d)) return rc;
        *bytes = sparsert::norm_workspace(d);
        return (int)SPARSERT_OK;
    });
}

int sparsert_rms_norm(const sparsert_norm *norm, const void *X_dev, const void *R_dev, const float *gamma_dev, void *H_dev, void *Y_dev,
                      float *scale_dev, void *workspace_dev, size_t workspace_bytes, void *stream) {
    return guarded([&](std::string &err) {
        if (!norm) return set_error(SPARSERT_EINVAL, "norm is NULL");
        sparsert::NormCall c{*norm, X_dev, R_dev, gamma_dev, H_dev, Y_dev, scale_dev, static_cast<float *>(workspace_dev), stream};
        sparsert_norm &d = c.d;
        if (int rc = check_norm(d)) return rc;
        if (!X_dev || !Y_dev) return set_error(SPARSERT_EINVAL, "device pointer is NULL");
        if ((d.out_dtype == SPARSERT_I8) != (scale_dev != nullptr)) return set_error(SPARSERT_EINVAL, "scale_dev goes with an int8 result, and only with one");
        if (misaligned(15, X_dev, R_dev, H_dev, Y_dev, workspace_dev)) return set_error(SPARSERT_EINVAL, "matrices and workspace must be 16-byte aligned");
        if (misaligned(3, gamma_dev, scale_dev)) return set_error(SPARSERT_EINVAL, "vectors must be 4-byte aligned");
        if (Y_dev == H_dev) return set_error(SPARSERT_EINVAL, "Y and H must be two buffers");
        if (H_dev == X_dev && d.ldh != d.ldx) return set_error(SPARSERT_EINVAL, "H may be X only at the same pitch");
        if (Y_dev == X_dev && (d.out_dtype != d.dtype || d.ldy != d.ldx)) return set_error(SPARSERT_EINVAL, "Y may be X only with its type and pitch");
        if (Y_dev == R_dev && (d.out_dtype != d.dtype || d.ldy != d.ldh)) return set_error(SPARSERT_EINVAL, "Y may be R only with its type and pitch");
        if (workspace_dev && workspace_bytes < sparsert::norm_workspace(d)) return set_error(SPARSERT_EINVAL, "the workspace is smaller than sparsert_rms_norm_workspace says");
        if (int rc = check_stream(stream)) return rc;
        return sparsert::launch_norm(c, err);
    });
}

int sparsert_dequantize(const sparsert_dequant *dequant, const int32_t *C_dev, const float *row_scale_dev, const float *col_scale_dev,
                        void *Y_dev, void *stream) {
    return guarded([&](std::string &err) {
        if (!dequant) return set_error(SPARSERT_EINVAL, "dequant is NULL");
        sparsert::DequantCall c{*dequant, C_dev, row_scale_dev, col_scale_dev, Y_dev, stream};
        sparsert_dequant &d = c.d;
        if (int rc = check_sizes(d.M, d.N, d.batch, d.reserved, 2)) return rc;
        if (!floating(d.dtype)) return set_error(SPARSERT_EINVAL, "dtype must be F32 or F16");
        if (int rc = check_pitch(d.ldc, d.M, d.N, 4, "ldc")) return rc;
        if (int rc = check_pitch(d.ldy, d.M, d.N, size_of(d.dtype), "ldy")) return rc;
        if (!C_dev || !Y_dev) return set_error(SPARSERT_EINVAL, "device pointer is NULL");
        if (misaligned(15, C_dev, Y_dev)) return set_error(SPARSERT_EINVAL, "matrices must be 16-byte aligned");
        if (misaligned(3, row_scale_dev, col_scale_dev)) return set_error(SPARSERT_EINVAL, "vectors must be 4-byte aligned");
        if (Y_dev == C_dev && (d.dtype != SPARSERT_F32 || d.ldy != d.ldc)) return set_error(SPARSERT_EINVAL, "Y may be C only as F32 at the same pitch");
        if (int rc = check_stream(stream)) return rc;
        return sparsert::launch_dequantize(c, err);
    });
}

int sparsert_adapters_workspace(const sparsert_adapter_set *set, size_t *bytes) {
    return guarded([&](std::string &) {
        if (!set || !bytes) return set_error(SPARSERT_EINVAL, "set or bytes is NULL");
        *bytes = 0;
        sparsert_adapter_set d = *set;
        if (int rc = check_set(d)) return rc;
        *bytes = sparsert::adapters_workspace(d);
        return (int)SPARSERT_OK;
    });
}

int sparsert_adapters(const sparsert_adapter_set *set, const void *X_dev, const void *down_dev, const void *up_dev, const int32_t *index_dev,
                      const float *alpha_dev, const void *C_dev, const float *row_scale_dev, const float *col_scale_dev, void *Y_dev,
                      void *workspace_dev, size_t workspace_bytes, void *stream) {
    return guarded([&](std::string &err) {
        if (!set) return set_error(SPARSERT_EINVAL, "set is NULL");
        sparsert::AdaptersCall c{*set, X_dev, down_dev, up_dev, index_dev, alpha_dev, C_dev, row_scale_dev, col_scale_dev, Y_dev, workspace_dev, stream};
        sparsert_adapter_set &d = c.d;
        if (int rc = check_set(d)) return rc;
        if (!X_dev || !down_dev || !up_dev || !index_dev || !C_dev || !Y_dev) return set_error(SPARSERT_EINVAL, "device pointer is NULL");
        if (misaligned(15, X_dev, down_dev, up_dev, C_dev, Y_dev, workspace_dev)) return set_error(SPARSERT_EINVAL, "matrices and workspace must be 16-byte aligned");
        if (misaligned(3, index_dev, alpha_dev, row_scale_dev, col_scale_dev)) return set_error(SPARSERT_EINVAL, "vectors must be 4-byte aligned");
        if (d.x_dtype != SPARSERT_I8 && (row_scale_dev || col_scale_dev)) return set_error(SPARSERT_EINVAL, "scales go with int8 X only");
        if (Y_dev == C_dev && (d.ldy != d.ldc || (d.x_dtype == SPARSERT_I8 && d.dtype != SPARSERT_F32)))
            return set_error(SPARSERT_EINVAL, "Y may be C only with elements of its size and at the same pitch");
        if (Y_dev == X_dev || workspace_dev == Y_dev) return set_error(SPARSERT_EINVAL, "Y overlaps X or the workspace");
        const size_t need = sparsert::adapters_workspace(d);
        if (need && !workspace_dev) return set_error(SPARSERT_EINVAL, "workspace_dev is NULL");
        if (workspace_bytes < need) return set_error(SPARSERT_EINVAL, "the workspace is smaller than sparsert_adapters_workspace says");
        if (int rc = check_stream(stream)) return rc;
        return sparsert::launch_adapters(c, err);
    });
}

}  // extern "C"
