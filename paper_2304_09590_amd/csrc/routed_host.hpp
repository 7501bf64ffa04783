// routed_host.hpp -- answers and training steps of a handle whose rows name their child networks
// (declared in pnn.h), made of the grouped products and the distillation loss.  Included by pnn.hip
// after both.

namespace {

// rows of one chunk of answers: about as many pairs as keep every CU busy
constexpr int64_t ROUTED_CHUNK = 65536;

// pieces of the handle's workspace, 256 bytes apart; without a base they only add up
struct Carve {
    char* base;
    int64_t used = 0;
    template <typename T> T* take(int64_t elems) {
        T* p = base ? (T*)(base + used) : nullptr;
        used += round_up(elems * (int64_t)sizeof(T), 256);
        return p;
    }
};

// a status of a call without a handle, reported on the handle
pnn_status of_handle(pnn_net* n, pnn_status st) {
    if (st == PNN_OK) return st;
    if (st == PNN_EHIP) n->broken = true;
    n->err = g_init_error;
    return st;
}
#define TRY_NET(net, x) TRY(of_handle(net, (x)))

pnn_status routed_usable(pnn_net* n, const float* x_dev, const int32_t* ids_dev, int64_t rows, int32_t per_row, hipStream_t s) {
    TRY_NET(n, check_groups(rows, per_row, n->cfg.replicas));
    if (rows == 0) return PNN_OK;
    if (!x_dev || !ids_dev) return fail(n, PNN_EINVAL, "x_dev / ids_dev is NULL");
    if (!aligned16(x_dev)) return fail(n, PNN_EINVAL, "x_dev is not 16-byte aligned");
    TRY(check_abort(n, true, s));
    // (recorded, the copy of the merged network would be made at every replay, and not before the first)
    if (n->bcast_pending && capturing(s))
        return fail(n, PNN_EHIP, "a merge has left its broadcast to the next call: make one outside the recording first");
    return settle(n, s);
}

pnn_status routed_grow(pnn_net* n, int64_t need, hipStream_t s) {
    const size_t had = n->routed_bytes;
    TRY(grow(n, s, &n->routed_ws, &n->routed_bytes, (size_t)need));
    if (n->routed_bytes != had) HIP_TRY(n, hipStreamSynchronize(nullptr));  // (a new workspace is cleared there)
    return PNN_OK;
}

// one layer of all CNs as the grouped products take it
pnn_group_layer routed_layer(const pnn_net* n, int l) {
    pnn_group_layer g;
    g.inputs = n->sizes[l]; g.outputs = n->sizes[l + 1];
    g.type = n->bf16 ? PNN_BF16_MIXED : PNN_FP32;
    g.w_dev = n->bf16 ? (const void*)(n->shadow + n->off_w[l]) : (const void*)(n->theta + n->off_w[l]);
    g.w_net = n->pstride; g.w_ld = n->sizes[l];
    g.b_dev = n->theta + n->off_b[l]; g.b_net = n->pstride;
    return g;
}

void rows_to_bf16(const float* src, bf16_t* dst, int64_t values, hipStream_t s) {
    rows_to_bf16_kernel<<<(unsigned)std::min<int64_t>((values + 2047) / 2048, 65536), 256, 0, s>>>(src, dst, values);
}

// the rows as the first layer's products take them
pnn_status routed_rows(pnn_net* n, const float* x, bf16_t* xb, int64_t rows, const void** xin, hipStream_t s) {
    *xin = x;
    if (!n->bf16) return PNN_OK;
    Launch lc(n, s, "routed_rows");
    rows_to_bf16(x, xb, rows * n->sizes[0], s);
    *xin = xb;
    return lc.done();
}

// activations of the hidden layers (act[l], l = 1 .. L - 1) and the output layer's sums z, a pair each
pnn_status routed_forward(pnn_net* n, const pnn_groups& g, const pnn_groups& pairs, const void* x, void* const* act, float* z,
                          hipStream_t s) {
    for (int l = 0; l < n->L; ++l) {
        const pnn_group_layer layer = routed_layer(n, l);
        const bool last = l == n->L - 1;
        Launch lc(n, s, "routed_forward");
        TRY_NET(n, pnn_grouped_forward(l == 0 ? &g : &pairs, &layer, l == 0 ? x : act[l], layer.inputs, last ? -1 : n->act[l],
                                       last ? z : act[l + 1], layer.outputs, last ? PNN_FP32 : layer.type, s));
        TRY(lc.done());
    }
    return PNN_OK;
}

}  // namespace

extern "C" {

pnn_status pnn_infer_routed(pnn_net* n, const float* x_dev, int64_t rows, const int32_t* ids_dev, int32_t per_row,
                            const float* weights_dev, int32_t* pred_dev, float* out_dev, void* hip_stream) {
    TRY(usable(n));
    hipStream_t s = (hipStream_t)hip_stream;
    TRY(routed_usable(n, x_dev, ids_dev, rows, per_row, s));
    if (rows == 0) return PNN_OK;
    if (!pred_dev) return fail(n, PNN_EINVAL, "pred_dev is NULL");
    const int64_t most = std::min(rows, std::max<int64_t>(1, ROUTED_CHUNK / per_row));
    const int64_t plan_words = group_plan(most, per_row, n->cfg.replicas).words, P = most * per_row;
    void* act[9] = {nullptr};
    int32_t* plan = nullptr;
    bf16_t* xb = nullptr;
    float* z = nullptr;
    auto lay = [&](char* base) {
        Carve c{base};
        plan = c.take<int32_t>(plan_words);
        xb = c.take<bf16_t>(n->bf16 ? most * n->sizes[0] : 0);
        for (int l = 1; l < n->L; ++l) act[l] = c.take<char>(P * n->sizes[l] * (n->bf16 ? 2 : 4));
        z = c.take<float>(P * n->sizes[n->L]);
        return c.used;
    };
    TRY(routed_grow(n, lay(nullptr), s));
    lay(n->routed_ws);
    for (int64_t r0 = 0; r0 < rows; r0 += most) {
        const int64_t m = std::min(most, rows - r0);
        const int32_t* ids = ids_dev + r0 * per_row;
        const pnn_groups g = {plan, m, per_row, n->cfg.replicas}, pairs = {plan, m * per_row, 1, n->cfg.replicas};
        {
            Launch lc(n, s, "routed_group");
            TRY_NET(n, pnn_group_rows(ids, m, per_row, n->cfg.replicas, plan, plan_words * 4, s));
            TRY(lc.done());
        }
        const void* xin = nullptr;
        TRY(routed_rows(n, x_dev + r0 * n->sizes[0], xb, m, &xin, s));
        TRY(routed_forward(n, g, pairs, xin, act, z, s));
        Launch lc(n, s, "routed_answer");
        routed_answer_kernel<<<(unsigned)((m + 255) / 256), 256, 0, s>>>(
            z, ids, weights_dev ? weights_dev + r0 * per_row : nullptr, m, per_row, n->cfg.replicas, n->sizes[n->L],
            n->act[n->L - 1], pred_dev + r0, out_dev ? out_dev + r0 * n->sizes[n->L] : nullptr);
        TRY(lc.done());
    }
    return PNN_OK;
}

pnn_status pnn_train_routed(pnn_net* n, const float* x_dev, int64_t rows, const int32_t* ids_dev, int32_t per_row,
                            const int32_t* idx_dev, const float* t_dev, int32_t top, const int32_t* y_dev, float temperature,
                            float alpha, float* loss_dev, void* hip_stream) {
    TRY(usable(n));
    hipStream_t s = (hipStream_t)hip_stream;
    const int L = n->L, O = n->sizes[L], K = n->cfg.replicas;
    if (n->act[L - 1] != PNN_SOFTMAX) return fail(n, PNN_EINVAL, "a teacher's logits train softmax outputs only");
    TRY(routed_usable(n, x_dev, ids_dev, rows, per_row, s));
    if (rows == 0) return PNN_OK;
    const int64_t P = rows * per_row;
    pnn_distill d = {nullptr, O, PNN_FP32, O, P, idx_dev, t_dev, top, y_dev, temperature, alpha};
    d.z_dev = x_dev;  // (a stand-in until the workspace is there: the other arguments are checked first)
    TRY_NET(n, check_distill(&d, x_dev, INT64_MAX));
    const int64_t plan_words = group_plan(rows, per_row, K).words;
    const pnn_groups shape = {nullptr, P, 1, K};
    const int64_t el = n->bf16 ? 2 : 4, stats_bytes = distill_bytes(P, O);
    int64_t widest = O, split = 0;
    for (int l = 1; l < L; ++l) widest = std::max<int64_t>(widest, n->sizes[l]);
    for (int l = 0; l < L; ++l) split = std::max(split, group_weights_ws(&shape, n->sizes[l], n->sizes[l + 1]));
    void *act[9] = {nullptr}, *err[2] = {nullptr};
    int32_t* plan = nullptr;
    bf16_t* xb = nullptr;
    float *z = nullptr, *stats = nullptr, *loss = nullptr;
    char* ws = nullptr;
    auto lay = [&](char* base) {
        Carve c{base};
        plan = c.take<int32_t>(plan_words);
        xb = c.take<bf16_t>(n->bf16 ? rows * n->sizes[0] : 0);
        for (int l = 1; l < L; ++l) act[l] = c.take<char>(P * n->sizes[l] * el);
        z = c.take<float>(P * O);
        stats = (float*)c.take<char>(stats_bytes);
        loss = c.take<float>(loss_dev ? 0 : P);
        for (auto& e : err) e = c.take<char>(P * widest * el);
        ws = c.take<char>(split);
        return c.used;
    };
    TRY(routed_grow(n, lay(nullptr), s));
    lay(n->routed_ws);
    const pnn_groups g = {plan, rows, per_row, K}, pairs = {plan, P, 1, K};
    {
        Launch lc(n, s, "routed_group");
        TRY_NET(n, pnn_group_rows(ids_dev, rows, per_row, K, plan, plan_words * 4, s));
        TRY(lc.done());
    }
    const void* xin = nullptr;
    TRY(routed_rows(n, x_dev, xb, rows, &xin, s));
    TRY(routed_forward(n, g, pairs, xin, act, z, s));
    void* delta = z;  // the output errors replace the sums, or stand beside them in bf16
    {
        Launch lc(n, s, "routed_loss");
        d.z_dev = z;
        const int width = distill_width(P, O, top);
        DistillArgs a = distill_args(&d, stats, width);
        a.rows_per = per_row; a.ids = ids_dev; a.K = K;
        a.loss = loss_dev ? loss_dev : loss;
        const int mode = distill_mode(&d);
        TRY_NET(n, run_distill_loss<float>(a, mode, width, s));
        a.dz = z; a.lddz = O;
        TRY_NET(n, run_distill_grad<float>(a, mode, width, s));
        if (n->bf16) {
            rows_to_bf16(z, (bf16_t*)err[0], P * O, s);
            delta = err[0];
        }
        TRY(lc.done());
    }
    for (int l = L - 1; l >= 0; --l) {
        const pnn_group_layer layer = routed_layer(n, l);
        void* below = delta == err[0] ? err[1] : err[0];
        if (l > 0) {  // with the weights from before the update
            Launch lc(n, s, "routed_errors");
            TRY_NET(n, pnn_grouped_backward_input(&pairs, &layer, delta, layer.outputs, act[l], layer.inputs, n->act[l - 1], below,
                                                  layer.inputs, layer.type, nullptr, 0, s));
            TRY(lc.done());
        }
        if (n->cfg.lr != 0.0f) {
            Launch lc(n, s, "routed_update");
            TRY_NET(n, run_group_weights(l == 0 ? &g : &pairs, layer.inputs, layer.outputs, layer.type, delta, layer.outputs,
                                         l == 0 ? xin : act[l], layer.inputs, l == 0 ? per_row : 1, n->theta + n->off_w[l],
                                         n->pstride, layer.inputs, n->theta + n->off_b[l], n->pstride, n->cfg.lr,
                                         n->bf16 ? n->shadow + n->off_w[l] : nullptr, ws, s));
            TRY(lc.done());
        }
        delta = below;
    }
    return PNN_OK;
}

}  // extern "C"
