// groups_host.hpp -- C ABI of the grouping and of the grouped products (declared in pnn.h).
// Included by pnn.hip, whose helpers it uses.

namespace {

// The device that a stream belongs to is the current one for the time of a call (the null stream
// takes the current device as it is).
struct OnDeviceOf {
    int before = -1;
    explicit OnDeviceOf(hipStream_t s) {
        hipDevice_t dev = -1;
        int cur = -1;
        if (!s) return;
        if (hipStreamGetDevice(s, &dev) != hipSuccess || hipGetDevice(&cur) != hipSuccess) {
            (void)hipGetLastError();  // (the launch itself will tell)
            return;
        }
        if (dev != cur && hipSetDevice(dev) == hipSuccess) before = cur;
    }
    ~OnDeviceOf() { if (before >= 0) (void)hipSetDevice(before); }
};

pnn_status launched(const char* what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(nullptr, PNN_EHIP, "%s failed to launch: %s", what, hipGetErrorString(e));
    return PNN_OK;
}

// lets a kernel have that much dynamic LDS, once per device (set: the devices on which it may)
pnn_status lds_of(const void* kernel, int bytes, std::atomic<uint64_t>& set) {
    int dev = 0;
    (void)hipGetDevice(&dev);
    const uint64_t bit = dev < 64 ? uint64_t(1) << dev : 0;
    if (bit && (set.load(std::memory_order_relaxed) & bit)) return PNN_OK;
    const hipError_t e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != hipSuccess) return fail(nullptr, PNN_EHIP, "hipFuncSetAttribute failed: %s", hipGetErrorString(e));
    set.fetch_or(bit, std::memory_order_relaxed);
    return PNN_OK;
}

constexpr int64_t GROUP_MAX_PAIRS = int64_t(1) << 30;
constexpr int32_t GROUP_MAX_WIDTH = 1 << 20;

pnn_status check_groups(int64_t n, int32_t per_row, int32_t networks) {
    if (n < 0) return fail(nullptr, PNN_ESHAPE, "n = %lld < 0", (long long)n);
    if (per_row < 1) return fail(nullptr, PNN_EINVAL, "per_row = %d (must be >= 1)", per_row);
    if (networks < 1 || networks > GR_MAX_NETS)
        return fail(nullptr, PNN_EINVAL, "networks = %d (must be in 1..%d)", networks, GR_MAX_NETS);
    if (n > GROUP_MAX_PAIRS / per_row)
        return fail(nullptr, PNN_ESHAPE, "%lld rows of %d networks are more than 2^30 pairs", (long long)n, per_row);
    return PNN_OK;
}

pnn_status check_groups(const pnn_groups* g) {
    if (!g) return fail(nullptr, PNN_EINVAL, "groups is NULL");
    TRY(check_groups(g->n, g->per_row, g->networks));
    if (g->n > 0 && !g->plan_dev) return fail(nullptr, PNN_EINVAL, "plan_dev is NULL");
    if (((uintptr_t)g->plan_dev & 15) != 0) return fail(nullptr, PNN_EINVAL, "plan_dev is not 16-byte aligned");
    return PNN_OK;
}

size_t type_size(int32_t type) { return type == PNN_FP32 ? 4 : 2; }

// a matrix argument: present, its rows at least as far apart as they are wide, aligned to its type
pnn_status check_rows(const char* name, const void* p, int64_t ld, int64_t width, int32_t type) {
    if (!p) return fail(nullptr, PNN_EINVAL, "%s is NULL", name);
    if (type != PNN_FP32 && type != PNN_BF16_MIXED) return fail(nullptr, PNN_EINVAL, "unknown type %d of %s", type, name);
    if (((uintptr_t)p & (type_size(type) - 1)) != 0) return fail(nullptr, PNN_EINVAL, "%s is not aligned to its type", name);
    if (ld < width) return fail(nullptr, PNN_EINVAL, "the rows of %s are %lld apart and %lld wide", name, (long long)ld, (long long)width);
    return PNN_OK;
}

pnn_status check_layer(const pnn_group_layer* l, bool weights) {
    if (!l) return fail(nullptr, PNN_EINVAL, "layer is NULL");
    if (l->inputs < 1 || l->inputs > GROUP_MAX_WIDTH || l->outputs < 1 || l->outputs > GROUP_MAX_WIDTH)
        return fail(nullptr, PNN_EINVAL, "a layer of %d inputs and %d outputs (each must be in 1..%d)", l->inputs, l->outputs,
                    GROUP_MAX_WIDTH);
    if (l->type != PNN_FP32 && l->type != PNN_BF16_MIXED) return fail(nullptr, PNN_EINVAL, "unknown type %d of a layer", l->type);
    if (!weights) return PNN_OK;
    TRY(check_rows("w_dev", l->w_dev, l->w_ld, l->inputs, l->type));
    if (l->w_net < 0 || l->b_net < 0) return fail(nullptr, PNN_EINVAL, "negative stride between networks");
    if (((uintptr_t)l->b_dev & 3) != 0) return fail(nullptr, PNN_EINVAL, "b_dev is not aligned to its type");
    return PNN_OK;
}

pnn_status check_act(int32_t act) {
    if (act < -1 || act > PNN_LEAKY_RELU)
        return fail(nullptr, PNN_EINVAL, "activation %d (-1 for none, or an elementwise pnn_act)", act);
    return PNN_OK;
}

GroupGemm group_base(const pnn_groups* g) {
    const GroupPlan p = group_plan(g->n, g->per_row, g->networks);
    const int32_t* w = (const int32_t*)g->plan_dev;
    GroupGemm a;
    memset(&a, 0, sizeof a);
    a.off = w;
    a.pairs = w + p.o_pairs;
    a.K = g->networks;
    a.N = (int)p.P;
    a.pdiv = a.wdiv = div_by(1);
    a.act = -1;
    a.splits = 1;
    return a;
}

// a launch holds less than 2^32 threads
constexpr int64_t MAX_THREADS = (int64_t(1) << 32) - 1;
pnn_status grid_fits(int64_t blocks, int threads) {
    if (blocks > MAX_THREADS / threads)
        return fail(nullptr, PNN_ESHAPE, "%lld workgroups are more than a launch takes", (long long)blocks);
    return PNN_OK;
}

// The kernels' tiles.  Large ones read operands less often; small ones are more, which hides the latency of
// short products and unequal groups.
enum { FEW, TILE64, TILE128, RING_SMALL, RING, RING_HUGE };
constexpr int64_t GROUP_FILL = 512;  // workgroups that fill the device: two on each of 256 CUs

// Parts that a group's pairs are cut into for a weight gradient, and the ring's tile: 256 x 256 where groups
// are long and cutting them into parts of 512 pairs fills the device; else 256 x 128; else 128 x 64, groups cut
// into parts of 256.  In us for tiles of 256 x 256, 256 x 128, 128 x 64 on whole groups: 2048 x 2048, 16 networks, 32,768
// pairs 298, 313, 508, 8,192 pairs 116, 111, 165; 784 x 512, 64 networks, 4,096 pairs 36, 33, 37; 512 x 512, 8
// networks, 2,000 pairs 16, 13, 9.  784 x 256, 60,000 pairs: one network whole 1,377, 1,146, 634, in 64 parts 88, 102,
// 116; four networks whole 358, 295, 164, in 29, 29 and 58 parts 84, 92, 158.  Parts are written and read again,
// which costs more than it gains where whole groups nearly fill the device: 1024 x 1024, 16 networks, 16,384 pairs in
// the rule's two parts 93, whole 47; 784 x 512, 16 networks, 60,000 pairs in its four parts 114, whole 101; 512 x 512,
// 8 networks, 8,000 pairs in its two (128 x 64) 25, whole 17.  Through registers (fp32), tiles of 64 and of 128 on whole
// groups: 501 x 203, 24 networks, 1,501 pairs 10, 15; 784 x 1024, 256 networks, 32,768 pairs 601, 540.
// The parts follow the mean: a group that holds most pairs is cut no finer than an even one would be.  784 x
// 1024, 256 networks, 32,768 pairs: even 336, half of them in one network 512, all in one 745 (fp32 530, 1,408, 2,619).
void group_weights_plan(int64_t P, int32_t K, int32_t inputs, int32_t outputs, int* kind, int* splits) {
    auto tiles = [&](int bm, int bn) { return (int64_t)K * ((inputs + bm - 1) / bm) * ((outputs + bn - 1) / bn); };
    const int64_t mean = P / K;
    auto cut = [&](int64_t t, int64_t rows) { return std::max<int64_t>(1, std::min<int64_t>({(GROUP_FILL + t - 1) / t, mean / rows, 64})); };
    int64_t t = tiles(256, 256), s = cut(t, 512);
    if (mean >= 512 && t * s >= GROUP_FILL / 2) {
        *kind = RING_HUGE;
        *splits = (int)s;
        return;
    }
    t = tiles(256, 128);
    if (t >= GROUP_FILL / 2) {
        *kind = RING;
        *splits = 1;
        return;
    }
    *kind = RING_SMALL;
    *splits = (int)cut(tiles(128, 64), 256);
}

// the ring kernels' copies: 16 bytes each, whole inside a row
bool ring_ok(const void* p, int64_t ld, int64_t net, int width) {
    return aligned16(p) && ld % 8 == 0 && ld < (int64_t(1) << 31) && net % 8 == 0 && width % 8 == 0;
}

template <int DIR, typename TO, int BM, int BN, int WM, int WN, int NST, bool AHEAD>
pnn_status launch_ring(const GroupGemm& a, int64_t blocks, hipStream_t s) {
    const int lds = NST * (BM + BN) * 32 * 2 + (DIR == GR_DW ? WM * WN * 2 * (NST - 1) * 256 : 0);
    TRY(grid_fits(blocks, 64 * WM * WN));
    static std::atomic<uint64_t> set{0};
    TRY(lds_of((const void*)group_ring_kernel<DIR, TO, BM, BN, WM, WN, NST, AHEAD>, lds, set));
    group_ring_kernel<DIR, TO, BM, BN, WM, WN, NST, AHEAD><<<(unsigned)blocks, 64 * WM * WN, lds, s>>>(a);
    return launched(DIR == GR_FWD ? "grouped forward" : DIR == GR_DX ? "grouped input gradient" : "grouped weight gradient");
}

// Which kernel multiplies pairs: tiles of 16 re-read the weights for each of them, those of 64 to 256 multiply
// what is not there.  Kernels in us, tiles of 16 against the larger ones that the rule would take.  fp32 at 1, 8, 16, 20
// pairs a network: 64 networks 784 -> 512 15, 23, 27, 34 against 26, 28, 29, 30, its input gradient 18, 29, 36, 44
// against 24, 27, 29, 29; 32 networks 1001 -> 999 19, 30, 35, 41 against 34, 37, 37, 37, its input gradient 25, 33, 43, 54
// against 37, 37, 40, 40.  bf16 at 1, 2, 4, 8: 784 -> 512 8, 11, 13, 14 against 9, 10, 11, 12, its input gradient 13,
// 13, 14, 15 against 10, 11, 12, 12; 32 networks 2048 -> 4096 64, 95, 106, 121 against 74, 105, 118, 108, its input
// gradient 68, 88, 93, 97 against 69, 93, 98, 101; 1001 -> 999 17, 22, 23, 26 against 19, 19, 19, 19, its input gradient 40,
// 41, 42, 42 against 31, 31, 31, 28.  One limit a type serves both directions: it costs a bf16 input gradient of
// narrow or unaligned layers a quarter at one and two pairs, and a wide forward product a tenth at three and four.
// Tiles of 64 against 128: fp32 8 networks 512 -> 512 8,000 pairs 34, 45, 16,000 pairs 61, 61; 256 networks 784 -> 1024
// 32,768 pairs 453, 397; bf16 of one value more each way 27, 26; 46, 38; 317, 253.  The ring's 128 x 64, 256 x 128, 256 x
// 256: 8 networks 1024 -> 1024 8,000 pairs 35, 35, 31, 16,000 pairs 59, 55, 60; 64 networks 784 -> 512 32,000 pairs 62, 51,
// 57; 16 networks 2048 -> 2048 8,192 pairs 124, 96, 106, 32,768 pairs 447, 293, 277; 4 networks 2048 -> 2048 8,000 pairs
// 112, 73, 61.  (256 x 256 is taken too early for short contractions: 8 networks 512 -> 512, 32,000 pairs 34, 27, 40.)
int group_pairs_kind(const pnn_groups* g, int M, bool bf16, bool ring) {
    const int64_t P = g->n * g->per_row, mean = P / g->networks;
    if (mean <= (bf16 ? 2 : 16)) return FEW;
    // (half of a network's last tile is empty in the mean)
    auto tiles = [&](int bm, int bn) { return (int64_t)((M + bm - 1) / bm) * (P / bn + g->networks / 2); };
    if (!ring) return tiles(128, 128) >= GROUP_FILL ? TILE128 : TILE64;
    if (mean >= 512 && tiles(256, 256) >= GROUP_FILL / 2) return RING_HUGE;
    return tiles(256, 128) >= GROUP_FILL ? RING : RING_SMALL;
}

template <int DIR, typename T, typename TO>
pnn_status run_group_pairs(GroupGemm& a, const pnn_groups* g, hipStream_t s) {
    const int kind = group_pairs_kind(g, a.M, sizeof(T) == 2, sizeof(T) == 2 && ring_ok(a.w, a.ldw, a.wnet, DIR == GR_FWD ? a.Kx : a.M) && ring_ok(a.p, a.ldp, 0, a.Kx));
    const GroupPlan p = group_plan(g->n, g->per_row, g->networks);
    const int height = kind == FEW ? 0 : kind == TILE64 || kind == RING_SMALL ? 1 : kind == RING_HUGE ? 3 : 2;
    a.tiles = (const int2*)((const int32_t*)g->plan_dev + p.o_tiles[height]);
    a.n_tiles = (const int32_t*)g->plan_dev + p.o_count + height;
    auto blocks = [&](int band) { return (a.M + band - 1) / band * p.most[height]; };
    // Large bf16 results are streamed: written past the caches they evict nothing of what the next workgroups read.
    // Forward in us, cached -> streamed, and with the next layer, which reads the result: 2048 x 2048, 134 MB 314 ->
    // 263, 641 -> 603; 67 MB 157 -> 154, 357 -> 370; 1024 x 1024, 134 MB 171 -> 148, 356 -> 328; 17 MB 38 -> 38,
    // 75 -> 78.
    a.stream = sizeof(TO) == 2 && p.P * a.M * (int64_t)sizeof(TO) >= (int64_t(96) << 20);
    if constexpr (sizeof(T) == 2) {
        if (kind == RING_HUGE) return launch_ring<DIR, TO, 256, 256, 2, 4, 4, true>(a, blocks(256), s);
        if (kind == RING) return launch_ring<DIR, TO, 256, 128, 2, 2, 3, false>(a, blocks(256), s);
        if (kind == RING_SMALL) return launch_ring<DIR, TO, 128, 64, 2, 2, 4, false>(a, blocks(128), s);
    }
    const int64_t all = blocks(kind == TILE128 ? 128 : kind == TILE64 ? 64 : DIR == GR_FWD ? GS_OUT : sizeof(T) == 4 ? 64 : 128);
    TRY(grid_fits(all, 256));
    if (kind == TILE128) group_tile_kernel<DIR, T, TO, 128><<<(unsigned)all, 256, 0, s>>>(a);
    else if (kind == TILE64) group_tile_kernel<DIR, T, TO, 64><<<(unsigned)all, 256, 0, s>>>(a);
    else if constexpr (DIR == GR_FWD) group_few_fwd_kernel<T, TO><<<(unsigned)all, 256, 0, s>>>(a);
    else group_few_dx_kernel<T, TO><<<(unsigned)all, 256, 0, s>>>(a);
    return launched(DIR == GR_FWD ? "grouped forward" : "grouped input gradient");
}

template <int DIR>
pnn_status run_group_pairs(GroupGemm& a, const pnn_groups* g, int32_t type, int32_t out_type, hipStream_t s) {
    if (type == PNN_FP32)
        return out_type == PNN_FP32 ? run_group_pairs<DIR, float, float>(a, g, s) : run_group_pairs<DIR, float, bf16_t>(a, g, s);
    return out_type == PNN_FP32 ? run_group_pairs<DIR, bf16_t, float>(a, g, s) : run_group_pairs<DIR, bf16_t, bf16_t>(a, g, s);
}

// weight gradient (lr = 0), or the update y -= lr / pairs * gradient
pnn_status run_group_weights(const pnn_groups* g, int32_t inputs, int32_t outputs, int32_t type, const void* dy, int64_t dy_ld,
                             const void* x, int64_t x_ld, int xdiv, float* dw, int64_t dw_net, int64_t dw_ld, float* db,
                             int64_t db_net, float lr, bf16_t* shadow, void* ws, hipStream_t s) {
    GroupGemm a = group_base(g);
    int S, kind;
    group_weights_plan((int64_t)g->n * g->per_row, g->networks, inputs, outputs, &kind, &S);
    a.M = inputs; a.N = outputs;
    a.p = dy; a.ldp = dy_ld;
    a.w = x; a.ldw = x_ld; a.wdiv = div_by(xdiv);
    a.splits = S;
    float* dbpart = (float*)ws + (int64_t)S * g->networks * inputs * outputs;
    if (S > 1) {
        a.y = ws; a.ldy = inputs; a.ynet = (int64_t)inputs * outputs;
        a.db = db ? dbpart : nullptr; a.dbnet = outputs;
    } else {
        a.y = dw; a.ldy = dw_ld; a.ynet = dw_net;
        a.db = db; a.dbnet = db_net;
        a.lr = lr; a.shadow = shadow;
    }
    auto blocks = [&](int bm, int bn) {
        return group_dw_blocks((int64_t)((inputs + bm - 1) / bm) * ((outputs + bn - 1) / bn), (int64_t)S * g->networks);
    };
    if (type != PNN_FP32 && ring_ok(x, x_ld, 0, inputs) && ring_ok(dy, dy_ld, 0, outputs)) {
        if (kind == RING_HUGE) TRY((launch_ring<GR_DW, float, 256, 256, 2, 4, 4, true>(a, blocks(256, 256), s)));
        else if (kind == RING) TRY((launch_ring<GR_DW, float, 256, 128, 2, 2, 3, false>(a, blocks(256, 128), s)));
        else TRY((launch_ring<GR_DW, float, 128, 64, 2, 2, 4, false>(a, blocks(128, 64), s)));
    } else {
        const bool small = blocks(128, 128) < GROUP_FILL;
        const int64_t all = small ? blocks(64, 64) : blocks(128, 128);
        TRY(grid_fits(all, 256));
        if (type == PNN_FP32) {
            if (small) group_tile_kernel<GR_DW, float, float, 64><<<(unsigned)all, 256, 0, s>>>(a);
            else group_tile_kernel<GR_DW, float, float, 128><<<(unsigned)all, 256, 0, s>>>(a);
        } else {
            if (small) group_tile_kernel<GR_DW, bf16_t, float, 64><<<(unsigned)all, 256, 0, s>>>(a);
            else group_tile_kernel<GR_DW, bf16_t, float, 128><<<(unsigned)all, 256, 0, s>>>(a);
        }
        TRY(launched("grouped weight gradient"));
    }
    if (S > 1) {
        GroupJoin j = {a.off, (const float*)ws, dbpart, g->networks, inputs, outputs, S, dw, dw_ld, dw_net, db, db_net, lr, shadow,
                       row_threads((inputs + 7) / 8)};
        const int64_t rows = (int64_t)g->networks * outputs, each = 256 / j.threads;
        group_join_kernel<<<(unsigned)std::min<int64_t>((rows + each - 1) / each, 8192), 256, 0, s>>>(j);
        TRY(launched("sum of a grouped weight gradient"));
    }
    return PNN_OK;
}

int64_t group_input_ws(const pnn_groups* g, int32_t inputs) {
    return g->per_row > 1 ? g->n * g->per_row * (int64_t)inputs * 4 : 0;
}
int64_t group_weights_ws(const pnn_groups* g, int32_t inputs, int32_t outputs) {
    int S, kind;
    group_weights_plan(g->n * g->per_row, g->networks, inputs, outputs, &kind, &S);
    return S > 1 ? (int64_t)S * g->networks * outputs * ((int64_t)inputs + 1) * 4 : 0;
}

pnn_status check_ws(const void* ws, int64_t have, int64_t need) {
    if (need == 0) return PNN_OK;
    if (!ws || have < need) return fail(nullptr, PNN_ESHAPE, "the call needs %lld bytes of workspace and has %lld", (long long)need, (long long)(ws ? have : 0));
    if (!aligned16(ws)) return fail(nullptr, PNN_EINVAL, "ws_dev is not 16-byte aligned");
    return PNN_OK;
}

}  // namespace

extern "C" {

pnn_status pnn_group_bytes(int64_t n, int32_t per_row, int32_t networks, int64_t* bytes) {
    TRY(check_groups(n, per_row, networks));
    if (!bytes) return fail(nullptr, PNN_EINVAL, "bytes is NULL");
    *bytes = group_plan(n, per_row, networks).words * 4;
    return PNN_OK;
}

pnn_status pnn_group_rows(const int32_t* ids_dev, int64_t n, int32_t per_row, int32_t networks, void* plan_dev,
                          int64_t plan_bytes, void* hip_stream) {
    TRY(check_groups(n, per_row, networks));
    const GroupPlan p = group_plan(n, per_row, networks);
    if (!plan_dev || (n > 0 && !ids_dev)) return fail(nullptr, PNN_EINVAL, "ids_dev / plan_dev is NULL");
    if (!aligned16(plan_dev)) return fail(nullptr, PNN_EINVAL, "plan_dev is not 16-byte aligned");
    if (((uintptr_t)ids_dev & 3) != 0) return fail(nullptr, PNN_EINVAL, "ids_dev is not aligned to its type");
    if (plan_bytes < p.words * 4)
        return fail(nullptr, PNN_ESHAPE, "the plan needs %lld bytes and has %lld", (long long)p.words * 4, (long long)plan_bytes);
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    int32_t* w = (int32_t*)plan_dev;
    GroupArgs a = {ids_dev, w, w + p.o_pairs, w + p.o_count, w + p.o_hist,
                   {(int2*)(w + p.o_tiles[0]), (int2*)(w + p.o_tiles[1]), (int2*)(w + p.o_tiles[2]), (int2*)(w + p.o_tiles[3])},
                   per_row > 1 ? (uint8_t*)(w + p.o_kept) : nullptr, p.P, p.chunk, p.K, p.blocks};
    if (p.blocks > 1) {
        group_count_kernel<<<(unsigned)p.blocks, GR_THREADS, 0, s>>>(a);
        TRY(launched("counting the groups"));
    }
    const int lds = (int)group_lds(p.K);
    if (p.blocks <= 1) {
        static std::atomic<uint64_t> set{0};
        TRY(lds_of((const void*)group_place_kernel<GR_ALONE / GR_THREADS>, (int)group_lds(GR_MAX_NETS), set));
        group_place_kernel<GR_ALONE / GR_THREADS><<<1, GR_THREADS, lds, s>>>(a);
    } else {
        static std::atomic<uint64_t> set{0};
        TRY(lds_of((const void*)group_place_kernel<GR_CHUNK / GR_THREADS>, (int)group_lds(GR_MAX_NETS), set));
        group_place_kernel<GR_CHUNK / GR_THREADS><<<(unsigned)p.blocks, GR_THREADS, lds, s>>>(a);
    }
    return launched("placing the groups");
}

pnn_status pnn_grouped_forward(const pnn_groups* groups, const pnn_group_layer* layer, const void* x_dev, int64_t x_ld,
                               int32_t act, void* y_dev, int64_t y_ld, int32_t y_type, void* hip_stream) {
    TRY(check_groups(groups));
    TRY(check_layer(layer, true));
    TRY(check_act(act));
    if (groups->n == 0) return PNN_OK;
    TRY(check_rows("x_dev", x_dev, x_ld, layer->inputs, layer->type));
    TRY(check_rows("y_dev", y_dev, y_ld, layer->outputs, y_type));
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    GroupGemm a = group_base(groups);
    a.M = layer->outputs; a.Kx = layer->inputs;
    a.p = x_dev; a.ldp = x_ld; a.pdiv = div_by(groups->per_row);
    a.w = layer->w_dev; a.wnet = layer->w_net; a.ldw = layer->w_ld;
    a.b = layer->b_dev; a.bnet = layer->b_net;
    a.act = act;
    a.y = y_dev; a.ldy = y_ld;
    return run_group_pairs<GR_FWD>(a, groups, layer->type, y_type, s);
}

pnn_status pnn_grouped_workspace(const pnn_groups* groups, const pnn_group_layer* layer, int64_t* input_bytes,
                                 int64_t* weights_bytes) {
    if (!groups) return fail(nullptr, PNN_EINVAL, "groups is NULL");
    TRY(check_groups(groups->n, groups->per_row, groups->networks));
    TRY(check_layer(layer, false));
    if (input_bytes) *input_bytes = group_input_ws(groups, layer->inputs);
    if (weights_bytes) *weights_bytes = group_weights_ws(groups, layer->inputs, layer->outputs);
    return PNN_OK;
}

pnn_status pnn_grouped_backward_input(const pnn_groups* groups, const pnn_group_layer* layer, const void* dy_dev, int64_t dy_ld,
                                      const void* a_dev, int64_t a_ld, int32_t act, void* dx_dev, int64_t dx_ld,
                                      int32_t dx_type, void* ws_dev, int64_t ws_bytes, void* hip_stream) {
    TRY(check_groups(groups));
    TRY(check_layer(layer, true));
    TRY(check_act(act));
    if (groups->n == 0) return PNN_OK;
    TRY(check_rows("dy_dev", dy_dev, dy_ld, layer->outputs, layer->type));
    TRY(check_rows("dx_dev", dx_dev, dx_ld, layer->inputs, dx_type));
    if (act >= 0) TRY(check_rows("a_dev", a_dev, a_ld, layer->inputs, layer->type));
    TRY(check_ws(ws_dev, ws_bytes, group_input_ws(groups, layer->inputs)));
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    const bool sum = groups->per_row > 1;
    GroupGemm a = group_base(groups);
    a.M = layer->inputs; a.Kx = layer->outputs;
    a.p = dy_dev; a.ldp = dy_ld;
    a.w = layer->w_dev; a.wnet = layer->w_net; a.ldw = layer->w_ld;
    if (!sum) {
        a.a = act >= 0 ? a_dev : nullptr; a.lda = a_ld; a.act = act;
        a.y = dx_dev; a.ldy = dx_ld;
        return run_group_pairs<GR_DX>(a, groups, layer->type, dx_type, s);
    }
    a.y = ws_dev; a.ldy = layer->inputs;
    TRY(run_group_pairs<GR_DX>(a, groups, layer->type, PNN_FP32, s));
    const int threads = row_threads((layer->inputs + 7) / 8), each = 256 / threads;
    const unsigned blocks = (unsigned)std::min<int64_t>((groups->n + each - 1) / each, 8192);
    const float* part = (const float*)ws_dev;
    const uint8_t* kept = (const uint8_t*)((const int32_t*)groups->plan_dev + group_plan(groups->n, groups->per_row, groups->networks).o_kept);
    const void* ad = act >= 0 ? a_dev : nullptr;
#define PNN_SUM_PAIRS(T, TO) \
    group_sum_pairs_kernel<T, TO><<<blocks, 256, 0, s>>>(part, groups->n, groups->per_row, layer->inputs, kept, (const T*)ad, a_ld, act, (TO*)dx_dev, dx_ld, threads)
    if (layer->type == PNN_FP32) { if (dx_type == PNN_FP32) PNN_SUM_PAIRS(float, float); else PNN_SUM_PAIRS(float, bf16_t); }
    else { if (dx_type == PNN_FP32) PNN_SUM_PAIRS(bf16_t, float); else PNN_SUM_PAIRS(bf16_t, bf16_t); }
#undef PNN_SUM_PAIRS
    return launched("sum over the pairs of a row");
}

pnn_status pnn_grouped_backward_weights(const pnn_groups* groups, const pnn_group_layer* layer, const void* dy_dev,
                                        int64_t dy_ld, const void* x_dev, int64_t x_ld, float* dw_dev, int64_t dw_net,
                                        int64_t dw_ld, float* db_dev, int64_t db_net, void* ws_dev, int64_t ws_bytes,
                                        void* hip_stream) {
    TRY(check_groups(groups));
    TRY(check_layer(layer, false));
    if (!groups->plan_dev) return fail(nullptr, PNN_EINVAL, "plan_dev is NULL");  // (no rows still give zeros)
    if (groups->n > 0) {
        TRY(check_rows("dy_dev", dy_dev, dy_ld, layer->outputs, layer->type));
        TRY(check_rows("x_dev", x_dev, x_ld, layer->inputs, layer->type));
    }
    TRY(check_rows("dw_dev", dw_dev, dw_ld, layer->inputs, PNN_FP32));
    if (((uintptr_t)db_dev & 3) != 0) return fail(nullptr, PNN_EINVAL, "db_dev is not aligned to its type");
    // (one network's rows after another's, or all networks' share of a row before the next row)
    const __int128 M = layer->inputs, after = (layer->outputs - 1) * (__int128)dw_ld + M;  // (strides of any size)
    if (groups->networks > 1 && dw_net < after && (dw_net < M || dw_ld - M < (groups->networks - 1) * (__int128)dw_net))
        return fail(nullptr, PNN_EINVAL, "the networks of dw_dev overlap");
    if (db_dev && db_net < layer->outputs && groups->networks > 1) return fail(nullptr, PNN_EINVAL, "the networks of db_dev overlap");
    TRY(check_ws(ws_dev, ws_bytes, group_weights_ws(groups, layer->inputs, layer->outputs)));
    hipStream_t s = (hipStream_t)hip_stream;
    OnDeviceOf dev(s);
    return run_group_weights(groups, layer->inputs, layer->outputs, layer->type, dy_dev, dy_ld, x_dev, x_ld, groups->per_row, dw_dev,
                             dw_net, dw_ld, db_dev, db_net, 0.0f, nullptr, ws_dev, s);
}

}  // extern "C"
