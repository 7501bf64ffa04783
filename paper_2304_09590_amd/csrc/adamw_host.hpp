// adamw_host.hpp -- C ABI of the AdamW step (declared in pnn.h).  Included by pnn.hip after route_host.hpp, whose
// helpers it uses.

namespace {

pnn_status check_adamw(int32_t bits, int32_t g_type) {
    if (bits != 32 && bits != 8) return fail(nullptr, PNN_EINVAL, "bits = %d (must be 32 or 8)", bits);
    if (g_type != PNN_FP32 && g_type != PNN_BF16_MIXED) return fail(nullptr, PNN_EINVAL, "unknown type %d of the gradients", g_type);
    return PNN_OK;
}

pnn_status check_adamw(const pnn_adamw* a) {
    if (!a) return fail(nullptr, PNN_EINVAL, "the arguments are NULL");
    TRY(check_adamw(a->bits, a->g_type));
    if (a->chunks < 0 || a->chunks > INT32_MAX) return fail(nullptr, PNN_EINVAL, "chunks = %lld", (long long)a->chunks);
    if (a->chunks > 0 && (!a->plan_dev || !aligned16(a->plan_dev))) return fail(nullptr, PNN_EINVAL, "plan_dev is NULL or not 16-byte aligned");
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

pnn_status check_adamw(const pnn_adamw_tensor& t, int32_t i, int32_t bits, int32_t g_type) {
    if (t.n == 0) return PNN_OK;
    if (!t.p_dev || !t.g_dev || !t.m_dev || !t.v_dev) return fail(nullptr, PNN_EINVAL, "tensor %d: p_dev, g_dev, m_dev or v_dev is NULL", i);
    if (misaligned4(t.p_dev) || ((uintptr_t)t.g_dev & (type_size(g_type) - 1)) != 0 || ((uintptr_t)t.copy_dev & 1) != 0)
        return fail(nullptr, PNN_EINVAL, "tensor %d: p_dev, g_dev or copy_dev is not aligned to its type", i);
    if (bits == 32) {
        if (misaligned4(t.m_dev) || misaligned4(t.v_dev)) return fail(nullptr, PNN_EINVAL, "tensor %d: m_dev or v_dev is not aligned to its type", i);
    } else if (!t.m_scale_dev || !t.v_scale_dev || misaligned4(t.m_scale_dev) || misaligned4(t.v_scale_dev)) {
        return fail(nullptr, PNN_EINVAL, "tensor %d: m_scale_dev or v_scale_dev is NULL or not aligned to its type", i);
    }
    return PNN_OK;
}

// chunks of the tensors, checked
pnn_status adamw_chunks(const pnn_adamw_tensor* tensors, int32_t count, int64_t* chunks) {
    if (count < 0) return fail(nullptr, PNN_ESHAPE, "count = %d < 0", count);
    if (count > 0 && !tensors) return fail(nullptr, PNN_EINVAL, "tensors is NULL");
    *chunks = 0;
    for (int32_t i = 0; i < count; ++i) {
        const int64_t n = tensors[i].n;
        if (n < 0 || n > (int64_t(1) << 40)) return fail(nullptr, PNN_ESHAPE, "tensor %d has %lld values (must be in 0..2^40)", i, (long long)n);
        *chunks += (n + AD_CHUNK - 1) / AD_CHUNK;
        if (*chunks > INT32_MAX) return fail(nullptr, PNN_ESHAPE, "the tensors have more than 2^43 values");
    }
    return PNN_OK;
}

// 16 waves a workgroup, a block each, where there are no more chunks than CUs; else four waves that take four blocks
// each, with a workgroup for each chunk.  Us for 32 bits, 16 waves against four: 0.1 million values 4.5, 5.2; 1 million 7.0,
// 7.6; 2 million 9.8, 10.1; 4 million 21.5, 20.4; for 8 bits 6.8, 8.9; 9.1, 11.1; 14.5, 14.2; 27.3, 22.9.
template <int BITS, typename TG>
void launch_adamw(const AdamArgs& a, hipStream_t s) {
    // (a call without values still counts its step)
    if (a.chunks <= 256) adamw_kernel<BITS, TG, 16><<<std::max(1u, a.chunks), 1024, 0, s>>>(a);
    else adamw_kernel<BITS, TG, 4><<<std::min(a.chunks, 16384u), 256, 0, s>>>(a);
}

}  // namespace

extern "C" {

pnn_status pnn_adamw_bytes(const pnn_adamw_tensor* tensors, int32_t count, int64_t* bytes, int64_t* chunks) {
    int64_t c = 0;
    TRY(adamw_chunks(tensors, count, &c));
    if (!bytes || !chunks) return fail(nullptr, PNN_EINVAL, "bytes or chunks is NULL");
    *bytes = AD_HEAD + c * (int64_t)sizeof(AdamChunk);
    *chunks = c;
    return PNN_OK;
}

pnn_status pnn_adamw_plan(const pnn_adamw_tensor* tensors, int32_t count, int32_t bits, int32_t g_type, void* plan_dev,
                          int64_t plan_bytes, void* hip_stream) {
    int64_t chunks = 0;
    TRY(adamw_chunks(tensors, count, &chunks));
    TRY(check_adamw(bits, g_type));
    for (int32_t i = 0; i < count; ++i) TRY(check_adamw(tensors[i], i, bits, g_type));
    if (chunks == 0) return PNN_OK;
    if (!plan_dev || !aligned16(plan_dev)) return fail(nullptr, PNN_EINVAL, "plan_dev is NULL or not 16-byte aligned");
    const int64_t need = AD_HEAD + chunks * (int64_t)sizeof(AdamChunk);
    if (plan_bytes < need) return fail(nullptr, PNN_ESHAPE, "the plan needs %lld bytes and has %lld", (long long)need, (long long)plan_bytes);
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    AdamPlanArgs d;
    memset(&d, 0, sizeof d);
    d.state_size = bits / 8;
    d.g_size = (int)type_size(g_type);
    d.places = (uint32_t*)plan_dev;
    d.plan = (AdamChunk*)((char*)plan_dev + AD_HEAD);
    for (int32_t i = 0; i < count;) {  // as many tensors a launch as its arguments hold
        d.number = i;
        uint32_t at = 0;
        for (d.count = 0; i < count && d.count < AD_TENSORS; ++i) {
            const pnn_adamw_tensor& t = tensors[i];
            d.t[d.count] = {t.p_dev, t.g_dev, t.m_dev, t.v_dev, t.m_scale_dev, t.v_scale_dev, t.copy_dev, t.n};
            d.first[d.count++] = at;
            at += (uint32_t)((t.n + AD_CHUNK - 1) / AD_CHUNK);
        }
        d.first[d.count] = at;
        if (at > 0) {
            adamw_plan_kernel<<<std::min((at + 255) / 256, 4096u), 256, 0, s>>>(d);
            TRY(launched("an AdamW plan"));
            d.places = nullptr;
        }
        d.plan += at;
    }
    return PNN_OK;
}

pnn_status pnn_adamw_step(const pnn_adamw* a, void* hip_stream) {
    TRY(check_adamw(a));
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    AdamArgs d;
    memset(&d, 0, sizeof d);
    d.places = (uint32_t*)a->plan_dev;
    d.plan = (const AdamChunk*)((const char*)a->plan_dev + AD_HEAD); d.chunks = (uint32_t)a->chunks;
    d.b1 = (float)a->beta1; d.c1 = (float)(1.0 - a->beta1);
    d.b2 = (float)a->beta2; d.c2 = (float)(1.0 - a->beta2);
    d.ln1 = (float)std::log(a->beta1); d.ln2 = (float)std::log(a->beta2);  // (-inf for a beta of 0: nothing is left after a step)
    d.lr = (float)a->lr; d.eps = (float)a->eps; d.decay = (float)a->weight_decay;
    d.lr_dev = a->lr_dev; d.seed = a->seed; d.steps = a->steps_dev;
    if (a->bits == 32) {
        if (a->g_type == PNN_FP32) launch_adamw<32, float>(d, s);
        else launch_adamw<32, bf16_t>(d, s);
    } else {
        if (a->g_type == PNN_FP32) launch_adamw<8, float>(d, s);
        else launch_adamw<8, bf16_t>(d, s);
    }
    return launched("the AdamW step");
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
