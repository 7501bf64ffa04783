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

// Lanes of a row.  Few lanes share the exchanges of a choice among several rows, many have fewer scores each to look at.
// Us with counts, two and eight choices: 60,000 rows of 250 on 16 lanes 18, 26, on 64 32, 73; of 40 10, 19 against
// 22, 45; of 500 on 32 lanes 29, 48, on 64 38, 79; 8,000 rows of 500 7.2, 9.6 against 7.6, 13.0; 1,000 rows of 500 6.7, 9.1
// against 5.1, 7.8; of 250 on 16 lanes 6.8, 9.0, on 64 7.6, 7.7.  (1,000 scores on 32 lanes do not fit the registers.)
int route_lanes(int64_t n, int32_t K) { return K <= 256 ? 16 : K <= 512 && n > 4096 ? 32 : 64; }
// The gradient has no choices, and a wave its networks' weights to begin with.  Us on 16 lanes against 64: 60,000 rows of 250 26,
// 28, of 40 12, 19; 16,000 rows 12.0, 11.4 and 6.1, 6.8; 8,000 rows 8.7, 7.3 and 4.9, 4.7; 1,000 rows 6.7, 3.8 and 4.5, 3.1.
int route_grad_lanes(int64_t n, int32_t K) { return K <= 256 && n > 8192 ? 16 : 64; }

int64_t route_rows(int lanes) { return RT_THREADS / 64 * (64 / lanes); }  // of a workgroup, at a time
int route_blocks(int64_t n, int32_t K) {
    const int64_t each = route_rows(route_lanes(n, K));
    return (int)std::max<int64_t>(1, std::min<int64_t>((n + each - 1) / each, RT_MAX_BLOCKS));
}

RouteArgs route_args(const pnn_router* a) {
    RouteArgs r;
    memset(&r, 0, sizeof r);
    r.s = a->s_dev; r.lds = a->s_ld; r.n = a->n;
    r.K = a->networks; r.k = a->per_row; r.normalize = a->normalize != 0;
    return r;
}

template <typename T>
void launch_route(const RouteArgs& r, hipStream_t s) {
    const int lanes = route_lanes(r.n, r.K);
#define PNN_ROUTE(L, V) route_kernel<T, L, V><<<r.blocks, RT_THREADS, 0, s>>>(r)
    if (r.K <= 16) PNN_ROUTE(16, 1);
    else if (r.K <= 64) PNN_ROUTE(16, 4);
    else if (r.K <= 128) PNN_ROUTE(16, 8);
    else if (r.K <= 256) PNN_ROUTE(16, 16);
    else if (lanes == 32) PNN_ROUTE(32, 16);
    else if (r.K <= 512) PNN_ROUTE(64, 8);
    else PNN_ROUTE(64, 16);
#undef PNN_ROUTE
}

template <typename T>
void launch_route_grad(const RouteArgs& r, hipStream_t s) {
    const int lanes = route_grad_lanes(r.n, r.K);
    const int64_t each = 4 * (64 / lanes);
    // (us with 1,024 workgroups against 2,048: 60,000 rows of 250 26, 29, of 1,000 93, 101; of 500 45, 42)
    const unsigned blocks = (unsigned)std::min<int64_t>((r.n + each - 1) / each, r.K > 256 && r.K <= 512 ? 2048 : 1024);
#define PNN_ROUTE(L, V) route_grad_kernel<T, L, V><<<blocks, 256, 0, s>>>(r)
    if (lanes == 16) {
        if (r.K <= 16) PNN_ROUTE(16, 1);
        else if (r.K <= 64) PNN_ROUTE(16, 4);
        else if (r.K <= 128) PNN_ROUTE(16, 8);
        else PNN_ROUTE(16, 16);
    } else {
        if (r.K <= 64) PNN_ROUTE(64, 1);
        else if (r.K <= 256) PNN_ROUTE(64, 4);
        else if (r.K <= 512) PNN_ROUTE(64, 8);
        else PNN_ROUTE(64, 16);
    }
#undef PNN_ROUTE
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
    r.blocks = route_blocks(a->n, a->networks);
    if (!counts_dev && a->networks <= 128) {  // (without sums to join: small rows keep more than one workgroup a CU busy)
        const int64_t each = route_rows(route_lanes(a->n, a->networks));
        r.blocks = (int)std::min<int64_t>((a->n + each - 1) / each, 4096);
    }
    r.part = (float*)ws_dev;
    r.part_counts = (int32_t*)ws_dev + (int64_t)r.blocks * a->networks;
    r.dots = (float*)ws_dev + round_up((int64_t)r.blocks * (2 * a->networks + 1), 4);
    r.arrived = (int32_t*)r.dots + 2 * (GR_MAX_NETS / RT_JOIN + 1);
    if (a->type == PNN_FP32) launch_route<float>(r, s);
    else launch_route<bf16_t>(r, s);
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
    if (a->type == PNN_FP32) launch_route_grad<float>(r, s);
    else launch_route_grad<bf16_t>(r, s);
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
