// route_host.hpp -- C ABI of the router and of combining (declared in pnn.h).  Included by pnn.hip after
// groups_host.hpp, whose helpers it uses.

namespace {

pnn_status check_route(int64_t n, int32_t networks) {
    if (n < 0 || n > INT32_MAX) return fail(nullptr, PNN_ESHAPE, "n = %lld (must be in 0..2^31 - 1)", (long long)n);
    if (networks < 1 || networks > GR_MAX_NETS)
        return fail(nullptr, PNN_EINVAL, "networks = %d (must be in 1..%d)", networks, GR_MAX_NETS);
    return PNN_OK;
}

pnn_status check_route(const pnn_router* a) {
    if (!a) return fail(nullptr, PNN_EINVAL, "the arguments are NULL");
    TRY(check_route(a->n, a->networks));
    if (a->per_row < 1 || a->per_row > RT_MAX_TOP || a->per_row > a->networks)
        return fail(nullptr, PNN_EINVAL, "per_row = %d (must be in 1..%d and at most the %d networks)", a->per_row, RT_MAX_TOP, a->networks);
    TRY(check_groups(a->n, a->per_row, a->networks));
    if (a->n == 0) return PNN_OK;
    return check_rows("s_dev", a->s_dev, a->s_ld, a->networks, a->type);
}

bool misaligned4(const void* p) { return ((uintptr_t)p & 3) != 0; }

// rows that a wave takes at a time: those of up to 256 scores lie on 16 lanes
int route_rows(int32_t networks) { return networks <= 256 ? 4 : 1; }

int route_blocks(int64_t n, int32_t networks) {
    const int64_t each = RT_THREADS / 64 * route_rows(networks);
    return (int)std::max<int64_t>(1, std::min<int64_t>((n + each - 1) / each, RT_MAX_BLOCKS));
}

RouteArgs route_args(const pnn_router* a) {
    RouteArgs r;
    memset(&r, 0, sizeof r);
    r.s = a->s_dev; r.lds = a->s_ld; r.n = a->n;
    r.K = a->networks; r.k = a->per_row; r.normalize = a->normalize != 0;
    return r;
}

// f(scores of a lane, lanes of a row) by the number of networks
template <typename F>
void route_by_width(int32_t K, F f) {
    using std::integral_constant;
    if (K <= 16) f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
    else if (K <= 64) f(integral_constant<int, 16>{}, integral_constant<int, 4>{});
    else if (K <= 128) f(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    else if (K <= 256) f(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    else if (K <= 512) f(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    else f(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

pnn_status check_combine(const pnn_combine* a) {
    if (!a) return fail(nullptr, PNN_EINVAL, "the arguments are NULL");
    TRY(check_groups(a->n, a->per_row, a->networks));
    if (a->width < 1 || a->width > GROUP_MAX_WIDTH)
        return fail(nullptr, PNN_EINVAL, "width = %d (must be in 1..%d)", a->width, GROUP_MAX_WIDTH);
    if (a->n == 0) return PNN_OK;
    TRY(check_rows("y_dev", a->y_dev, a->y_ld, a->width, a->type));
    if (!a->ids_dev || !a->w_dev) return fail(nullptr, PNN_EINVAL, "ids_dev / w_dev is NULL");
    if (misaligned4(a->ids_dev) || misaligned4(a->w_dev)) return fail(nullptr, PNN_EINVAL, "ids_dev or w_dev is not aligned to its type");
    return PNN_OK;
}

CombineArgs combine_args(const pnn_combine* a, unsigned* blocks) {
    CombineArgs c;
    memset(&c, 0, sizeof c);
    c.y = a->y_dev; c.ldy = a->y_ld; c.n = a->n;
    c.per_row = a->per_row; c.M = a->width; c.K = a->networks;
    c.ids = a->ids_dev; c.w = a->w_dev;
    c.threads = row_threads((a->width + 7) / 8);
    const int each = 256 / c.threads;
    *blocks = (unsigned)std::min<int64_t>((a->n + each - 1) / each, 8192);
    return c;
}

}  // namespace

extern "C" {

pnn_status pnn_route_bytes(int64_t n, int32_t networks, int64_t* bytes) {
    TRY(check_route(n, networks));
    if (!bytes) return fail(nullptr, PNN_EINVAL, "bytes is NULL");
    *bytes = 4 * (round_up((int64_t)route_blocks(n, networks) * (2 * networks + 1), 4) + 2 * (GR_MAX_NETS / RT_JOIN + 1) + 2);
    return PNN_OK;
}

pnn_status pnn_route(const pnn_router* a, int32_t* ids_dev, float* gates_dev, int32_t* counts_dev, float* loss_dev,
                     void* ws_dev, int64_t ws_bytes, void* hip_stream) {
    TRY(check_route(a));
    if ((counts_dev == nullptr) != (loss_dev == nullptr)) return fail(nullptr, PNN_EINVAL, "counts_dev and loss_dev go together");
    if (a->n > 0 && (!ids_dev || !gates_dev)) return fail(nullptr, PNN_EINVAL, "ids_dev / gates_dev is NULL");
    if (misaligned4(ids_dev) || misaligned4(gates_dev) || misaligned4(counts_dev) || misaligned4(loss_dev))
        return fail(nullptr, PNN_EINVAL, "ids_dev, gates_dev, counts_dev or loss_dev is not aligned to its type");
    if (counts_dev) {
        int64_t need = 0;
        TRY(pnn_route_bytes(a->n, a->networks, &need));
        TRY(check_ws(ws_dev, ws_bytes, need));
    } else if (a->n == 0) {
        return PNN_OK;
    }
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    RouteArgs r = route_args(a);
    r.ids = ids_dev; r.gates = gates_dev;
    r.counts = counts_dev; r.loss = loss_dev;
    const int64_t each = RT_THREADS / 64 * route_rows(a->networks);
    // (without sums to join, as many workgroups as rows keep busy)
    r.blocks = counts_dev ? route_blocks(a->n, a->networks) : (int)std::min<int64_t>((a->n + each - 1) / each, 4096);
    r.part = (float*)ws_dev;
    r.part_counts = (int32_t*)ws_dev + (int64_t)r.blocks * a->networks;
    r.dots = (float*)ws_dev + round_up((int64_t)r.blocks * (2 * a->networks + 1), 4);
    r.arrived = (int32_t*)r.dots + 2 * (GR_MAX_NETS / RT_JOIN + 1);
    route_by_width(a->networks, [&](auto L, auto V) {
        if (a->type == PNN_FP32) route_kernel<float, L(), V()><<<r.blocks, RT_THREADS, 0, s>>>(r);
        else route_kernel<bf16_t, L(), V()><<<r.blocks, RT_THREADS, 0, s>>>(r);
    });
    TRY(launched("routing"));
    if (!counts_dev || r.blocks == 1) return PNN_OK;  // (a workgroup that is alone has it all)
    route_join_kernel<<<a->networks / RT_JOIN + 1, 256, 0, s>>>(r);
    return launched("the balance loss");
}

pnn_status pnn_route_grad(const pnn_router* a, const int32_t* ids_dev, const int32_t* counts_dev, const float* dgates_dev,
                          const float* dloss_dev, void* ds_dev, int64_t ds_ld, void* hip_stream) {
    TRY(check_route(a));
    if (a->n == 0) return PNN_OK;
    TRY(check_rows("ds_dev", ds_dev, ds_ld, a->networks, a->type));
    if (dgates_dev && !ids_dev) return fail(nullptr, PNN_EINVAL, "dgates_dev needs ids_dev");
    if (dloss_dev && !counts_dev) return fail(nullptr, PNN_EINVAL, "dloss_dev needs counts_dev");
    if (misaligned4(ids_dev) || misaligned4(counts_dev) || misaligned4(dgates_dev) || misaligned4(dloss_dev))
        return fail(nullptr, PNN_EINVAL, "ids_dev, counts_dev, dgates_dev or dloss_dev is not aligned to its type");
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    RouteArgs r = route_args(a);
    r.ids = const_cast<int32_t*>(ids_dev); r.counts = const_cast<int32_t*>(counts_dev);
    r.dgates = dgates_dev; r.dloss = dloss_dev;
    r.ds = ds_dev; r.ldds = ds_ld;
    const int64_t each = 4 * route_rows(a->networks);
    const unsigned blocks = (unsigned)std::min<int64_t>((a->n + each - 1) / each, 2048);
    route_by_width(a->networks, [&](auto L, auto V) {
        if (a->type == PNN_FP32) route_grad_kernel<float, L(), V()><<<blocks, 256, 0, s>>>(r);
        else route_grad_kernel<bf16_t, L(), V()><<<blocks, 256, 0, s>>>(r);
    });
    return launched("the router's gradient");
}

pnn_status pnn_combine_rows(const pnn_combine* a, void* out_dev, int64_t out_ld, int32_t out_type, void* hip_stream) {
    TRY(check_combine(a));
    if (a->n == 0) return PNN_OK;
    TRY(check_rows("out_dev", out_dev, out_ld, a->width, out_type));
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    unsigned blocks;
    CombineArgs c = combine_args(a, &blocks);
    c.out = out_dev; c.ldo = out_ld;
    if (a->type == PNN_FP32) {
        if (out_type == PNN_FP32) combine_kernel<float, float><<<blocks, 256, 0, s>>>(c);
        else combine_kernel<float, bf16_t><<<blocks, 256, 0, s>>>(c);
    } else {
        if (out_type == PNN_FP32) combine_kernel<bf16_t, float><<<blocks, 256, 0, s>>>(c);
        else combine_kernel<bf16_t, bf16_t><<<blocks, 256, 0, s>>>(c);
    }
    return launched("combining");
}

pnn_status pnn_combine_grad(const pnn_combine* a, const void* g_dev, int64_t g_ld, int32_t g_type, void* dy_dev, int64_t dy_ld,
                            float* dw_dev, void* hip_stream) {
    TRY(check_combine(a));
    if (a->n == 0) return PNN_OK;
    TRY(check_rows("g_dev", g_dev, g_ld, a->width, g_type));
    TRY(check_rows("dy_dev", dy_dev, dy_ld, a->width, a->type));
    if (!dw_dev || misaligned4(dw_dev)) return fail(nullptr, PNN_EINVAL, "dw_dev is NULL or not aligned to its type");
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    unsigned blocks;
    CombineArgs c = combine_args(a, &blocks);
    c.g = g_dev; c.ldg = g_ld; c.dy = dy_dev; c.lddy = dy_ld; c.dw = dw_dev;
    if (a->type == PNN_FP32) {
        if (g_type == PNN_FP32) combine_grad_kernel<float, float><<<blocks, 256, 0, s>>>(c);
        else combine_grad_kernel<float, bf16_t><<<blocks, 256, 0, s>>>(c);
    } else {
        if (g_type == PNN_FP32) combine_grad_kernel<bf16_t, float><<<blocks, 256, 0, s>>>(c);
        else combine_grad_kernel<bf16_t, bf16_t><<<blocks, 256, 0, s>>>(c);
    }
    return launched("the gradients of combining");
}

}  // extern "C"
