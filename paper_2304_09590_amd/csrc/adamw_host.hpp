// adamw_host.hpp -- C ABI of the AdamW step (declared in pnn.h).  Included by pnn.hip after route_host.hpp, whose
// helpers it uses.

namespace {

pnn_status check_adamw(const pnn_adamw* a) {
    if (!a) return fail(nullptr, PNN_EINVAL, "the arguments are NULL");
    if (a->bits != 32 && a->bits != 8) return fail(nullptr, PNN_EINVAL, "bits = %d (must be 32 or 8)", a->bits);
    if (a->g_type != PNN_FP32 && a->g_type != PNN_BF16_MIXED) return fail(nullptr, PNN_EINVAL, "unknown type %d of the gradients", a->g_type);
    if (!(a->beta1 >= 0.0 && a->beta1 < 1.0 && a->beta2 >= 0.0 && a->beta2 < 1.0))
        return fail(nullptr, PNN_EINVAL, "beta1 = %g, beta2 = %g (must be in [0, 1))", a->beta1, a->beta2);
    if ((float)a->beta1 >= 1.0f || (float)a->beta2 >= 1.0f) return fail(nullptr, PNN_EINVAL, "a beta is 1 in fp32");
    if (!(a->eps >= 1e-30 && a->eps <= 1.0)) return fail(nullptr, PNN_EINVAL, "eps = %g (must be in 1e-30..1)", a->eps);
    if (!(a->weight_decay >= 0.0 && a->weight_decay <= 1e6)) return fail(nullptr, PNN_EINVAL, "weight_decay = %g (must be in 0..1e6)", a->weight_decay);
    if (!a->lr_dev && !(a->lr >= 0.0 && a->lr <= 1e6)) return fail(nullptr, PNN_EINVAL, "lr = %g (must be in 0..1e6)", a->lr);
    if (misaligned4(a->lr_dev)) return fail(nullptr, PNN_EINVAL, "lr_dev is not aligned to its type");
    if (!a->steps_dev || misaligned4(a->steps_dev)) return fail(nullptr, PNN_EINVAL, "steps_dev is NULL or not aligned to its type");
    return PNN_OK;
}

pnn_status check_adamw(const pnn_adamw* a, const pnn_adamw_tensor& t, int32_t i) {
    if (t.n < 0 || t.n > (int64_t(1) << 40)) return fail(nullptr, PNN_ESHAPE, "tensor %d has %lld values (must be in 0..2^40)", i, (long long)t.n);
    if (t.n == 0) return PNN_OK;
    if (!t.p_dev || !t.g_dev || !t.m_dev || !t.v_dev) return fail(nullptr, PNN_EINVAL, "tensor %d: p_dev, g_dev, m_dev or v_dev is NULL", i);
    if (misaligned4(t.p_dev) || ((uintptr_t)t.g_dev & (type_size(a->g_type) - 1)) != 0 || ((uintptr_t)t.copy_dev & 1) != 0)
        return fail(nullptr, PNN_EINVAL, "tensor %d: p_dev, g_dev or copy_dev is not aligned to its type", i);
    if (a->bits == 32) {
        if (misaligned4(t.m_dev) || misaligned4(t.v_dev)) return fail(nullptr, PNN_EINVAL, "tensor %d: m_dev or v_dev is not aligned to its type", i);
    } else if (!t.m_scale_dev || !t.v_scale_dev || misaligned4(t.m_scale_dev) || misaligned4(t.v_scale_dev)) {
        return fail(nullptr, PNN_EINVAL, "tensor %d: m_scale_dev or v_scale_dev is NULL or not aligned to its type", i);
    }
    return PNN_OK;
}

template <int BITS, typename TG>
pnn_status launch_adamw(const AdamArgs& a, hipStream_t s) {
    // (a call without values still counts its step)
    const unsigned blocks = std::max(1u, std::min(a.first[a.count], 2048u));
    adamw_kernel<BITS, TG><<<blocks, 256, 0, s>>>(a);
    return launched("the AdamW step");
}

}  // namespace

extern "C" {

pnn_status pnn_adamw_step(const pnn_adamw* a, const pnn_adamw_tensor* tensors, int32_t count, void* hip_stream) {
    TRY(check_adamw(a));
    if (count < 0) return fail(nullptr, PNN_ESHAPE, "count = %d < 0", count);
    if (count > 0 && !tensors) return fail(nullptr, PNN_EINVAL, "tensors is NULL");
    for (int32_t i = 0; i < count; ++i) TRY(check_adamw(a, tensors[i], i));
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    AdamArgs d;
    memset(&d, 0, sizeof d);
    d.b1 = (float)a->beta1; d.c1 = (float)(1.0 - a->beta1);
    d.b2 = (float)a->beta2; d.c2 = (float)(1.0 - a->beta2);
    d.ln1 = (float)std::log(a->beta1); d.ln2 = (float)std::log(a->beta2);  // (-inf for a beta of 0: nothing is left after a step)
    d.lr = (float)a->lr; d.eps = (float)a->eps; d.decay = (float)a->weight_decay;
    d.lr_dev = a->lr_dev; d.seed = a->seed; d.steps = a->steps_dev;
    int32_t i = 0;
    do {  // as many tensors a launch as its arguments hold, and chunks as 31 bits count
        d.number = i;
        d.count = 0;
        int64_t chunks = 0;
        while (i < count && d.count < AD_TENSORS) {
            const pnn_adamw_tensor& t = tensors[i];
            const int64_t more = (t.n + AD_CHUNK - 1) / AD_CHUNK;
            if (chunks + more > INT32_MAX) break;  // (one tensor has at most 2^28)
            d.t[d.count] = {t.p_dev, t.g_dev, t.m_dev, t.v_dev, t.m_scale_dev, t.v_scale_dev, t.copy_dev, t.n};
            d.first[d.count++] = (uint32_t)chunks;
            chunks += more;
            ++i;
        }
        d.first[d.count] = (uint32_t)chunks;
        d.last = i == count;
        if (a->bits == 32) TRY((a->g_type == PNN_FP32 ? launch_adamw<32, float>(d, s) : launch_adamw<32, bf16_t>(d, s)));
        else TRY((a->g_type == PNN_FP32 ? launch_adamw<8, float>(d, s) : launch_adamw<8, bf16_t>(d, s)));
    } while (i < count);
    return PNN_OK;
}

pnn_status pnn_adamw_values(const uint8_t* m_dev, const uint8_t* v_dev, const float* m_scale_dev, const float* v_scale_dev, int64_t n,
                            float* m_out_dev, float* v_out_dev, void* hip_stream) {
    if (n < 0 || n > (int64_t(1) << 40)) return fail(nullptr, PNN_ESHAPE, "n = %lld (must be in 0..2^40)", (long long)n);
    if (n == 0) return PNN_OK;
    if (!m_dev || !v_dev || !m_scale_dev || !v_scale_dev || !m_out_dev || !v_out_dev) return fail(nullptr, PNN_EINVAL, "a state or a result is NULL");
    if (misaligned4(m_scale_dev) || misaligned4(v_scale_dev) || misaligned4(m_out_dev) || misaligned4(v_out_dev))
        return fail(nullptr, PNN_EINVAL, "a scale or a result is not aligned to its type");
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    adamw_values_kernel<<<(unsigned)std::min<int64_t>((n + 1023) / 1024, 8192), 256, 0, s>>>(m_dev, v_dev, m_scale_dev, v_scale_dev, n,
                                                                                          m_out_dev, v_out_dev);
    return launched("the values of 8-bit states");
}

}  // extern "C"
