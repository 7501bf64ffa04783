// codes_host.hpp -- C ABI of rows as 8-bit codes and of their grouped product (declared in pnn.h).  Included by
// pnn.hip after groups_host.hpp, whose helpers it uses.

namespace {

// sums of 127 x 127 fit 32 bits up to here
constexpr int32_t CODES_MAX_INPUTS = 1 << 17;

pnn_status check_codes(const char* name, const int8_t* p, int64_t ld, int64_t width) {
    if (!p) return fail(nullptr, PNN_EINVAL, "%s is NULL", name);
    if (!aligned16(p) || ld % 16 != 0 || ld < width || ld >= (int64_t(1) << 31))
        return fail(nullptr, PNN_EINVAL, "rows of %s start at multiples of 16 bytes (they are %lld apart and %lld wide)", name,
                    (long long)ld, (long long)width);
    return PNN_OK;
}

pnn_status check_scale(const char* name, const float* p) {
    if (!p || ((uintptr_t)p & 3) != 0) return fail(nullptr, PNN_EINVAL, "%s is NULL or not aligned to its type", name);
    return PNN_OK;
}

// Threads of a row, 16 values each at a time: as many as it fills.  Us for 16, 64, 128 and 256: 16,384 rows of 200 in fp32 4.4, 9.1,
// 13.8, 22; of 1,024 - , 16, 18, 24; of 2,048 -, 27, 28, 29 (in bf16 27, 26, 29); of 4,096 -, 78, 58, 56 (46, 41, 40); 64 rows
// of 1,024 in fp32 -, 3.3, 3.2, 3.3, of 4,096 -, 5.8, 4.1, 3.2.
template <typename T>
void launch_codes(const CodesArgs& c, hipStream_t s) {
    const int threads = c.width <= 256 ? 16 : c.width <= 1024 ? 64 : c.width <= 2048 ? 128 : 256, each = 256 / threads;
    const unsigned blocks = (unsigned)std::min<int64_t>((c.n + each - 1) / each, 2048);
    if (threads == 16) codes_kernel<T, 16><<<blocks, 256, 0, s>>>(c);
    else if (threads == 64) codes_kernel<T, 64><<<blocks, 256, 0, s>>>(c);
    else if (threads == 128) codes_kernel<T, 128><<<blocks, 256, 0, s>>>(c);
    else codes_kernel<T, 256><<<blocks, 256, 0, s>>>(c);
}

}  // namespace

extern "C" {

pnn_status pnn_quantize_rows(const void* x_dev, int64_t x_ld, int32_t type, int64_t n, int32_t width, int8_t* q_dev, int64_t q_ld,
                             float* scale_dev, void* hip_stream) {
    if (n < 0) return fail(nullptr, PNN_ESHAPE, "n = %lld < 0", (long long)n);
    if (width < 1 || width > GROUP_MAX_WIDTH) return fail(nullptr, PNN_EINVAL, "width = %d (must be in 1..%d)", width, GROUP_MAX_WIDTH);
    if (n == 0) return PNN_OK;
    TRY(check_rows("x_dev", x_dev, x_ld, width, type));
    TRY(check_codes("q_dev", q_dev, q_ld, round_up(width, 16)));
    TRY(check_scale("scale_dev", scale_dev));
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    const CodesArgs c = {x_dev, x_ld, n, width, q_dev, q_ld, scale_dev};
    if (type == PNN_FP32) launch_codes<float>(c, s);
    else launch_codes<bf16_t>(c, s);
    return launched("quantizing rows");
}

pnn_status pnn_grouped_forward_int8(const pnn_groups* groups, const pnn_group_codes* layer, const int8_t* x_dev, int64_t x_ld,
                                    const float* x_scale_dev, int32_t act, void* y_dev, int64_t y_ld, int32_t y_type, void* hip_stream) {
    TRY(check_groups(groups));
    if (!layer) return fail(nullptr, PNN_EINVAL, "layer is NULL");
    if (layer->inputs < 16 || layer->inputs > CODES_MAX_INPUTS || layer->inputs % 16 != 0)
        return fail(nullptr, PNN_EINVAL, "a layer of %d inputs (must be a multiple of 16 in 16..%d)", layer->inputs, CODES_MAX_INPUTS);
    if (layer->outputs < 1 || layer->outputs > GROUP_MAX_WIDTH)
        return fail(nullptr, PNN_EINVAL, "a layer of %d outputs (must be in 1..%d)", layer->outputs, GROUP_MAX_WIDTH);
    TRY(check_codes("w_dev", layer->w_dev, layer->w_ld, layer->inputs));
    if (layer->w_net < 0 || layer->w_net % 16 != 0 || layer->scale_net < 0 || layer->b_net < 0)
        return fail(nullptr, PNN_EINVAL, "strides between networks are >= 0, w_net a multiple of 16");
    TRY(check_scale("scale_dev", layer->scale_dev));
    if (((uintptr_t)layer->b_dev & 3) != 0) return fail(nullptr, PNN_EINVAL, "b_dev is not aligned to its type");
    TRY(check_act(act));
    if (groups->n == 0) return PNN_OK;
    TRY(check_codes("x_dev", x_dev, x_ld, layer->inputs));
    TRY(check_scale("x_scale_dev", x_scale_dev));
    TRY(check_rows("y_dev", y_dev, y_ld, layer->outputs, y_type));
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    GroupGemm a = group_base(groups);  // (widths and distances in two codes)
    a.M = layer->outputs; a.Kx = layer->inputs / 2;
    a.p = x_dev; a.ldp = x_ld / 2; a.pdiv = div_by(groups->per_row);
    a.w = layer->w_dev; a.wnet = layer->w_net / 2; a.ldw = layer->w_ld / 2;
    a.b = layer->b_dev; a.bnet = layer->b_net;
    a.sx = x_scale_dev; a.sw = layer->scale_dev; a.swnet = layer->scale_net;
    a.act = act;
    a.y = y_dev; a.ldy = y_ld;
    return y_type == PNN_FP32 ? run_group_pairs<GR_FWD, codes_t, float>(a, groups, s) : run_group_pairs<GR_FWD, codes_t, bf16_t>(a, groups, s);
}

}  // extern "C"
