// distill_host.hpp -- C ABI of the distillation loss (declared in pnn.h).  Included by pnn.hip after
// groups_host.hpp, whose helpers it uses.

namespace {

// Parts of a row: with fewer rows than four workgroups per CU a row is split until there are as many,
// as long as a part keeps 2,048 classes, one 8-value load a thread.  Loss + gradient in us, whole rows against parts,
// in fp32: one row of 131,072 classes 15 + 29 against 6 + 6, 32 rows 16 + 32 against 8 + 11; 32,000 classes, 32 rows 7 + 13
// against 8 + 8, 256 rows 9 + 18 against 12 + 15, 768 rows 19 + 35 against 22 + 34; 8,192 classes, 64 rows 5 + 8 against
// 7 + 7.  (The join makes the loss alone slower from about 100 rows on; both together are level or better in parts.)
void distill_parts(int64_t n, int32_t classes, int* S, int* part) {
    int64_t s = n > 0 ? (1024 + n - 1) / n : 1;
    s = std::max<int64_t>(1, std::min<int64_t>(s, classes / 2048));
    const int64_t p = round_up((classes + s - 1) / s, 8);
    *part = (int)p;
    *S = (int)((classes + p - 1) / p);
}

// 16 lanes, one wave or a workgroup per row.  Loss + gradient in us in fp32: 128 classes, lanes against a wave 3 + 4
// against 4 + 6 for 64 rows, 9 + 16 against 35 + 46 for 60,000; a wave against a workgroup, 512 classes 4 + 5 against 5 + 5
// for 64 rows, 36 + 51 against 99 + 122 for 60,000; 2,048 classes 4 + 8 against 5 + 7 and 87 + 259 against 138 + 241; 4,096
// classes 5 + 10 against 7 + 7 and 172 + 477 against 182 + 425 (bf16 98 + 247 against 153 + 262).
enum { DL_LANES, DL_WAVE, DL_BLOCK };
int distill_width(int64_t n, int32_t classes, int32_t k) {
    if (classes <= DL_TINY && k <= DL_TINY_TOP) return DL_LANES;
    if (classes <= 2048 && k <= DL_WAVE_TOP) return DL_WAVE;
    return DL_BLOCK;
}

pnn_status check_distill(int64_t n, int32_t classes) {
    if (n < 0 || n > INT32_MAX) return fail(nullptr, PNN_ESHAPE, "n = %lld (must be in 0..2^31 - 1)", (long long)n);
    if (classes < 1 || classes > (1 << 30)) return fail(nullptr, PNN_EINVAL, "classes = %d (must be in 1..2^30)", classes);
    return PNN_OK;
}

int64_t distill_bytes(int64_t n, int32_t classes) {
    int S, part;
    distill_parts(n, classes, &S, &part);
    return n * 16 * (S > 1 ? S + 1 : 1);
}

pnn_status check_distill(const pnn_distill* a, const void* stats, int64_t stats_bytes) {
    if (!a) return fail(nullptr, PNN_EINVAL, "the arguments are NULL");
    TRY(check_distill(a->n, a->classes));
    if (a->top < 0 || a->top > DL_MAX_TOP) return fail(nullptr, PNN_EINVAL, "top = %d (must be in 0..%d)", a->top, DL_MAX_TOP);
    if (!(a->temperature >= 1e-6f && a->temperature <= 1e6f))
        return fail(nullptr, PNN_EINVAL, "temperature = %g (must be in 1e-6..1e6)", a->temperature);
    if (!(a->alpha >= 0.0f && a->alpha <= 1.0f)) return fail(nullptr, PNN_EINVAL, "alpha = %g (must be in 0..1)", a->alpha);
    if (a->n == 0) return PNN_OK;
    TRY(check_rows("z_dev", a->z_dev, a->z_ld, a->classes, a->type));
    if (a->alpha < 1.0f && a->top > 0 && (!a->idx_dev || !a->t_dev)) return fail(nullptr, PNN_EINVAL, "idx_dev / t_dev is NULL");
    if (a->alpha > 0.0f && !a->y_dev) return fail(nullptr, PNN_EINVAL, "alpha = %g needs y_dev", a->alpha);
    if ((((uintptr_t)a->idx_dev | (uintptr_t)a->y_dev) & 3) != 0 || ((uintptr_t)a->t_dev & (type_size(a->type) - 1)) != 0)
        return fail(nullptr, PNN_EINVAL, "idx_dev, t_dev or y_dev is not aligned to its type");
    if (!stats || !aligned16(stats)) return fail(nullptr, PNN_EINVAL, "stats_dev is NULL or not 16-byte aligned");
    if (stats_bytes < distill_bytes(a->n, a->classes))
        return fail(nullptr, PNN_ESHAPE, "stats_dev needs %lld bytes and has %lld", (long long)distill_bytes(a->n, a->classes),
                    (long long)stats_bytes);
    return PNN_OK;
}

DistillArgs distill_args(const pnn_distill* a, void* stats, int width) {
    const double log2e = 1.4426950408889634, T = a->temperature, alpha = a->alpha;
    DistillArgs d;
    memset(&d, 0, sizeof d);
    d.z = a->z_dev; d.ldz = a->z_ld; d.n = a->n; d.V = a->classes; d.k = a->top;
    d.idx = a->idx_dev; d.t = a->t_dev; d.y = alpha > 0.0 ? a->y_dev : nullptr;
    d.ct = (float)(log2e / T); d.cs = (float)log2e; d.inv_t = (float)(1.0 / T);
    d.wt = a->top > 0 ? (float)((1.0 - alpha) * T * T) : 0.0f; d.ws = (float)alpha;
    d.gt = (float)((1.0 - alpha) * T); d.gs = (float)alpha;
    if (d.wt == 0.0f) d.ct = d.cs;  // the label alone: the one sum is at 1
    d.rows_per = 1;
    d.S = 1; d.part = a->classes;
    if (width == DL_BLOCK) distill_parts(a->n, a->classes, &d.S, &d.part);
    d.stats = (float4*)stats;
    d.parts = (float4*)stats + a->n;
    return d;
}

// the sums that a call needs: one; two; two whose second is that of the first's squares
int distill_mode(const pnn_distill* a) {
    if (a->top == 0 || a->alpha == 0.0f || a->alpha == 1.0f || a->temperature == 1.0f) return 1;
    return a->temperature == 2.0f ? 3 : 2;
}

// f(d, workgroups) for as many rows at a time as a launch holds workgroups of 256 threads
template <typename F>
pnn_status distill_launches(DistillArgs d, int width, const char* what, F f) {
    const int64_t most = MAX_THREADS / 256, per = width == DL_LANES ? 16 : width == DL_WAVE ? 4 : 1;  // rows of a workgroup
    const int64_t rows = width == DL_BLOCK ? std::max<int64_t>(1, most / d.S) : most * per;
    for (d.row0 = 0; d.row0 < d.n; d.row0 += rows) {
        const int64_t m = std::min(rows, d.n - d.row0);
        f(d, (unsigned)(width == DL_BLOCK ? m * d.S : (m + per - 1) / per), (unsigned)m);
        TRY(launched(what));
    }
    return PNN_OK;
}

template <typename T, int MODE>
pnn_status launch_distill_loss(const DistillArgs& a, int width, hipStream_t s) {
    return distill_launches(a, width, "distillation loss", [&](const DistillArgs& d, unsigned blocks, unsigned rows) {
        if (width == DL_LANES) {
            if (d.V <= 16) distill_loss_tiny_kernel<T, MODE, 1><<<blocks, 256, 0, s>>>(d);
            else distill_loss_tiny_kernel<T, MODE, DL_TINY / 16><<<blocks, 256, 0, s>>>(d);
        } else if (width == DL_WAVE) {
            distill_loss_kernel<T, MODE, 1><<<blocks, 256, 0, s>>>(d);
        } else {
            distill_loss_kernel<T, MODE, 4><<<blocks, 256, 0, s>>>(d);
            if (d.S > 1) distill_join_kernel<T, MODE><<<rows, 64, 0, s>>>(d);
        }
    });
}

template <typename T, int MODE>
pnn_status launch_distill_grad(const DistillArgs& a, int width, hipStream_t s) {
    return distill_launches(a, width, "distillation gradient", [&](const DistillArgs& d, unsigned blocks, unsigned) {
        if (width == DL_LANES) {
            if (d.V <= 16) distill_grad_tiny_kernel<T, 1><<<blocks, 256, 0, s>>>(d);
            else distill_grad_tiny_kernel<T, DL_TINY / 16><<<blocks, 256, 0, s>>>(d);
        } else if (width == DL_WAVE) {
            distill_grad_kernel<T, MODE, 1><<<blocks, 256, 0, s>>>(d);
        } else {
            distill_grad_kernel<T, MODE, 4><<<blocks, 256, 0, s>>>(d);
        }
    });
}

template <typename T>
pnn_status run_distill_loss(const DistillArgs& d, int mode, int width, hipStream_t s) {
    return mode == 1 ? launch_distill_loss<T, 1>(d, width, s)
                     : mode == 2 ? launch_distill_loss<T, 2>(d, width, s) : launch_distill_loss<T, 3>(d, width, s);
}
template <typename T>
pnn_status run_distill_grad(const DistillArgs& d, int mode, int width, hipStream_t s) {
    return mode == 1 ? launch_distill_grad<T, 1>(d, width, s)
                     : mode == 2 ? launch_distill_grad<T, 2>(d, width, s) : launch_distill_grad<T, 3>(d, width, s);
}

}  // namespace

extern "C" {

pnn_status pnn_distill_bytes(int64_t n, int32_t classes, int64_t* bytes) {
    TRY(check_distill(n, classes));
    if (!bytes) return fail(nullptr, PNN_EINVAL, "bytes is NULL");
    *bytes = distill_bytes(n, classes);
    return PNN_OK;
}

pnn_status pnn_distill_loss(const pnn_distill* a, float* loss_dev, void* stats_dev, int64_t stats_bytes, void* hip_stream) {
    TRY(check_distill(a, stats_dev, stats_bytes));
    if (a->n == 0) return PNN_OK;
    if (!loss_dev || ((uintptr_t)loss_dev & 3) != 0) return fail(nullptr, PNN_EINVAL, "loss_dev is NULL or not aligned to its type");
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    const int width = distill_width(a->n, a->classes, a->top);
    DistillArgs d = distill_args(a, stats_dev, width);
    d.loss = loss_dev;
    const int mode = distill_mode(a);
    return a->type == PNN_FP32 ? run_distill_loss<float>(d, mode, width, s) : run_distill_loss<bf16_t>(d, mode, width, s);
}

pnn_status pnn_distill_grad(const pnn_distill* a, const float* g_dev, const void* stats_dev, int64_t stats_bytes, void* dz_dev,
                            int64_t dz_ld, void* hip_stream) {
    TRY(check_distill(a, stats_dev, stats_bytes));
    if (a->n == 0) return PNN_OK;
    TRY(check_rows("dz_dev", dz_dev, dz_ld, a->classes, a->type));
    if (((uintptr_t)g_dev & 3) != 0) return fail(nullptr, PNN_EINVAL, "g_dev is not aligned to its type");
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    const int width = distill_width(a->n, a->classes, a->top);
    DistillArgs d = distill_args(a, const_cast<void*>(stats_dev), width);
    d.g = g_dev; d.dz = dz_dev; d.lddz = dz_ld;
    // The gradient is streamed where the logits, read again by row, and it exceed the 256 MB memory-side cache together.
    // Loss and gradient in us, cached -> streamed, and with a reader of the gradient: 32,000 classes in bf16, 131 MB
    // 79 -> 79, 129 -> 125; 147 MB 94 -> 93, 166 -> 146; 262 MB 186 -> 161, 273 -> 269; 16,000 classes in fp32, 98 MB
    // 57 -> 66, 87 -> 95; 131 MB 77 -> 84, 131 -> 131; 147 MB 86 -> 92, 164 -> 146; 262 MB 183 -> 159, 271 -> 264.
    d.stream = a->n * a->classes * (int64_t)type_size(a->type) > (int64_t(128) << 20);
    const int mode = distill_mode(a);
    return a->type == PNN_FP32 ? run_distill_grad<float>(d, mode, width, s) : run_distill_grad<bf16_t>(d, mode, width, s);
}

}  // extern "C"
