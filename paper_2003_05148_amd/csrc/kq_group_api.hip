// C ABI of the 4-bit fully-connected layer and the 8-bit checkpoints: argument checks and launches.
// As everywhere in the library, the arguments are checked before HIP is touched and nothing is allocated.
#include "kq_group.h"

using namespace kq;

namespace {

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
bool valid_type(int32_t t) { return t == KQ_T_F32 || t == KQ_T_BF16 || t == KQ_T_F16; }
bool valid_act(int32_t t) { return t == KQ_T_BF16 || t == KQ_T_F16; }
uintptr_t type_bytes(int32_t t) { return t == KQ_T_F32 ? 4 : 2; }
bool valid_tensor(const void* p, int32_t type, int64_t ld, int64_t cols) {
    return p != nullptr && aligned(p, type_bytes(type)) && ld >= cols && ld <= (int64_t(1) << 40);
}

kq_status hip_status(hipError_t e) { return e == hipSuccess ? KQ_OK : KQ_ERR_HIP; }

int log2_group(int32_t group) { return group == 32 ? 5 : group == 64 ? 6 : group == 128 ? 7 : -1; }

kq_status check_size(int64_t n, int64_t k) {
    if (n < 1 || k < 1) return KQ_ERR_ARG;
    if (n > KQ_GROUP_MAX_FEATURES || k > KQ_GROUP_MAX_FEATURES || n * k > KQ_GROUP_MAX_VALUES) return KQ_ERR_UNSUPPORTED;
    return KQ_OK;
}
// m rows of n and of k values (0 for a matrix that the call does not have)
kq_status check_rows(int64_t m, int64_t n, int64_t k) {
    if (m < 0) return KQ_ERR_ARG;
    if (m > KQ_GROUP_MAX_ROWS || m * n > KQ_GROUP_MAX_VALUES || m * k > KQ_GROUP_MAX_VALUES) return KQ_ERR_UNSUPPORTED;
    return KQ_OK;
}

// the packed weights of a call; scales may be left out (need_scales false)
kq_status make_weights(GroupWeights& w, const uint8_t* codes, const void* scales, const void* levels, int64_t n,
                       int64_t k, int32_t group, bool need_scales) {
    const kq_status st = check_size(n, k);
    if (st != KQ_OK) return st;
    if (log2_group(group) < 0) return KQ_ERR_UNSUPPORTED;
    if (!codes || !aligned(codes, 16) || (need_scales && (!scales || !aligned(scales, 2))) || !aligned(levels, 2))
        return KQ_ERR_ARG;
    w.codes = codes;
    w.scales = (const uint16_t*)scales;
    w.levels = (const uint16_t*)levels;
    w.n = (int)n;
    w.k = (int)k;
    w.log_group = log2_group(group);
    w.groups = (int)ceil_div64(k, group);
    w.ktiles = (int)ceil_div64(k, kTileCols);
    w.ntiles = (int)ceil_div64(n, kTileRows);
    return KQ_OK;
}

kq_status check_ws(void* ws, size_t ws_bytes, size_t need) {
    if (need == 0) return KQ_OK;
    if (ws == nullptr || !aligned(ws, 256) || ws_bytes < need) return KQ_ERR_WORKSPACE;
    return KQ_OK;
}

kq_status check_checkpoint(int32_t type, int64_t m, int64_t k) {
    if (k < 1) return KQ_ERR_ARG;
    if (!valid_type(type) || k > KQ_GROUP_MAX_FEATURES) return KQ_ERR_UNSUPPORTED;
    return check_rows(m, 0, k);
}

}  // namespace

extern "C" {

size_t kq_group_code_bytes(int64_t n, int64_t k) {
    if (check_size(n, k) != KQ_OK) return 0;
    return (size_t)ceil_div64(n, kTileRows) * (size_t)ceil_div64(k, kTileCols) * kTileBytes;
}

kq_status kq_quantize_groups(const void* W, int32_t type, int64_t ldw, int64_t n, int64_t k, int32_t group,
                             const void* levels, uint8_t* codes, void* scales, void* stream) {
    GroupWeights w;
    const kq_status st = make_weights(w, codes, scales, levels, n, k, group, true);
    if (st != KQ_OK) return st;
    if (!valid_type(type)) return KQ_ERR_UNSUPPORTED;
    if (!valid_tensor(W, type, ldw, k)) return KQ_ERR_ARG;
    const QuantizeParams p = {W, ldw, type, w.n, w.k, w.log_group, w.groups, w.ktiles, w.levels, codes, (uint16_t*)scales};
    return hip_status(launch_quantize_groups(p, (hipStream_t)stream));
}

kq_status kq_reconstruct_groups(const uint8_t* codes, const void* scales, const void* levels, int64_t n, int64_t k,
                                int32_t group, int32_t type, void* W_hat, int64_t ldw, void* stream) {
    ReconstructGroupsParams p;
    const kq_status st = make_weights(p.w, codes, scales, levels, n, k, group, true);
    if (st != KQ_OK) return st;
    if (!valid_type(type)) return KQ_ERR_UNSUPPORTED;
    if (!valid_tensor(W_hat, type, ldw, k)) return KQ_ERR_ARG;
    p.type = type;
    p.W_hat = W_hat;
    p.ldw = ldw;
    return hip_status(launch_reconstruct_groups(p, (hipStream_t)stream));
}

size_t kq_group_linear_workspace_bytes(const void* X, int64_t ldx, int64_t m, int64_t n, int64_t k) {
    if (m < 1 || check_size(n, k) != KQ_OK || check_rows(m, n, k) != KQ_OK) return 0;
    return m <= kMatvecRows ? matvec_plan((int)m, n, k).ws_bytes : gemm_plan(Product::Linear, X, ldx, n, m, k, 0).ws_bytes;
}

kq_status kq_group_linear(const void* X, int32_t type, int64_t ldx, int64_t m, int64_t n, int64_t k,
                          const uint8_t* codes, const void* scales, const void* levels, int32_t group,
                          const float* bias, void* Y, int64_t ldy, void* ws, size_t ws_bytes, void* stream) {
    GemmParams p = {};
    kq_status st = make_weights(p.w, codes, scales, levels, n, k, group, true);
    if (st != KQ_OK) return st;
    if (!valid_act(type)) return KQ_ERR_UNSUPPORTED;
    if ((st = check_rows(m, n, k)) != KQ_OK) return st;
    if (!aligned(bias, 4)) return KQ_ERR_ARG;
    if (m == 0) return KQ_OK;
    if (!valid_tensor(X, type, ldx, k) || !valid_tensor(Y, type, ldy, n)) return KQ_ERR_ARG;
    if (m <= kMatvecRows) {
        const MatvecPlan plan = matvec_plan((int)m, n, k);
        if ((st = check_ws(ws, ws_bytes, plan.ws_bytes)) != KQ_OK) return st;
        MatvecParams v = {};
        v.w = p.w;
        v.X = X;
        v.ldx = ldx;
        v.m = (int)m;
        v.bias = bias;
        v.Y = Y;
        v.ldy = ldy;
        v.part = plan.ws_bytes ? (float*)ws : nullptr;
        return hip_status(launch_matvec(type == KQ_T_BF16, plan, v, (hipStream_t)stream));
    }
    const GemmPlan plan = gemm_plan(Product::Linear, X, ldx, n, m, k, 0);
    if ((st = check_ws(ws, ws_bytes, plan.ws_bytes)) != KQ_OK) return st;
    p.B = X;
    p.ldb = ldx;
    p.I = n;
    p.J = m;
    p.C = k;
    p.bias = bias;
    p.out = Y;
    p.ldo = ldy;
    return hip_status(launch_gemm(Product::Linear, type == KQ_T_BF16, plan, p, ws, (hipStream_t)stream));
}

size_t kq_group_linear_grad_input_workspace_bytes(const void* dY, int64_t ldy, int64_t m, int64_t n, int64_t k) {
    if (m < 1 || check_size(n, k) != KQ_OK || check_rows(m, n, k) != KQ_OK) return 0;
    return gemm_plan(Product::GradInput, dY, ldy, k, m, n, 0).ws_bytes;
}

kq_status kq_group_linear_grad_input(const void* dY, int32_t type, int64_t ldy, int64_t m, int64_t n, int64_t k,
                                     const uint8_t* codes, const void* scales, const void* levels, int32_t group,
                                     void* dX, int64_t ldx, void* ws, size_t ws_bytes, void* stream) {
    GemmParams p = {};
    kq_status st = make_weights(p.w, codes, scales, levels, n, k, group, true);
    if (st != KQ_OK) return st;
    if (!valid_act(type)) return KQ_ERR_UNSUPPORTED;
    if ((st = check_rows(m, n, k)) != KQ_OK) return st;
    if (m == 0) return KQ_OK;
    if (!valid_tensor(dY, type, ldy, n) || !valid_tensor(dX, type, ldx, k)) return KQ_ERR_ARG;
    const GemmPlan plan = gemm_plan(Product::GradInput, dY, ldy, k, m, n, 0);
    if ((st = check_ws(ws, ws_bytes, plan.ws_bytes)) != KQ_OK) return st;
    p.B = dY;
    p.ldb = ldy;
    p.I = k;
    p.J = m;
    p.C = n;
    p.out = dX;
    p.ldo = ldx;
    return hip_status(launch_gemm(Product::GradInput, type == KQ_T_BF16, plan, p, ws, (hipStream_t)stream));
}

kq_status kq_checkpoint_pack(const void* X, int32_t type, int64_t ldx, int64_t m, int64_t k, int8_t* q, uint8_t* exps,
                             void* stream) {
    const kq_status st = check_checkpoint(type, m, k);
    if (st != KQ_OK) return st;
    if (m == 0) return KQ_OK;
    if (!valid_tensor(X, type, ldx, k) || !q || !aligned(q, 16) || !exps) return KQ_ERR_ARG;
    const CheckpointParams p = {const_cast<void*>(X), ldx, type, m, (int)k, ceil_div((int)k, kCkGroup) * kCkGroup, q, exps};
    return hip_status(launch_checkpoint_pack(p, (hipStream_t)stream));
}

kq_status kq_checkpoint_restore(const int8_t* q, const uint8_t* exps, int64_t m, int64_t k, int32_t type, void* X_hat,
                                int64_t ldx, void* stream) {
    const kq_status st = check_checkpoint(type, m, k);
    if (st != KQ_OK) return st;
    if (m == 0) return KQ_OK;
    if (!valid_tensor(X_hat, type, ldx, k) || !q || !aligned(q, 16) || !exps) return KQ_ERR_ARG;
    const CheckpointParams p = {X_hat, ldx, type, m, (int)k, ceil_div((int)k, kCkGroup) * kCkGroup,
                                const_cast<int8_t*>(q), const_cast<uint8_t*>(exps)};
    return hip_status(launch_checkpoint_restore(p, (hipStream_t)stream));
}

size_t kq_checkpoint_grad_workspace_bytes(int64_t m, int64_t n, int64_t k, int32_t group) {
    if (check_size(n, k) != KQ_OK || check_rows(m, n, k) != KQ_OK || (group != 0 && log2_group(group) < 0)) return 0;
    if (group == 0) return gemm_plan(Product::GradWeight, nullptr, 0, k, n, m, 0).ws_bytes;
    return gemm_plan(Product::GradScales, nullptr, 0, k, n, m, (int)ceil_div64(k, group)).ws_bytes;
}

namespace {
kq_status checkpoint_grad(Product mode, GemmParams& p, const void* dY, int32_t type, int64_t ldy, int64_t m, int64_t n,
                          int64_t k, const int8_t* q, const uint8_t* exps, void* out, int64_t ldo, float* dbias, void* ws,
                          size_t ws_bytes, hipStream_t stream) {
    if (!valid_act(type)) return KQ_ERR_UNSUPPORTED;
    kq_status st = check_rows(m, n, k);
    if (st != KQ_OK) return st;
    if (!out || !aligned(out, 4) || ldo < 1 || ldo > (int64_t(1) << 40) || !aligned(dbias, 4)) return KQ_ERR_ARG;
    // without rows there is nothing to read, and the gradients are zero
    if (m > 0 && (!valid_tensor(dY, type, ldy, n) || !q || !aligned(q, 16) || !exps)) return KQ_ERR_ARG;
    const GemmPlan plan = gemm_plan(mode, nullptr, 0, k, n, m, p.w.groups);
    if ((st = check_ws(ws, ws_bytes, plan.ws_bytes)) != KQ_OK) return st;
    p.B = dY;
    p.ldb = ldy;
    p.q = q;
    p.exps = exps;
    p.kq = ceil_div((int)k, kCkGroup) * kCkGroup;
    p.I = k;
    p.J = n;
    p.C = m;
    p.out = out;
    p.ldo = ldo;
    p.dbias = dbias;
    return hip_status(launch_gemm(mode, type == KQ_T_BF16, plan, p, ws, stream));
}
}  // namespace

kq_status kq_checkpoint_grad_scales(const void* dY, int32_t type, int64_t ldy, int64_t m, int64_t n, int64_t k,
                                    const int8_t* q, const uint8_t* exps, const uint8_t* codes, const void* levels,
                                    int32_t group, float* dscales, float* dbias, void* ws, size_t ws_bytes,
                                    void* stream) {
    GemmParams p = {};
    const kq_status st = make_weights(p.w, codes, nullptr, levels, n, k, group, false);
    if (st != KQ_OK) return st;
    return checkpoint_grad(Product::GradScales, p, dY, type, ldy, m, n, k, q, exps, dscales, p.w.groups, dbias, ws,
                           ws_bytes, (hipStream_t)stream);
}

kq_status kq_checkpoint_grad_weight(const void* dY, int32_t type, int64_t ldy, int64_t m, int64_t n, int64_t k,
                                    const int8_t* q, const uint8_t* exps, float* dW, int64_t lddw, float* dbias,
                                    void* ws, size_t ws_bytes, void* stream) {
    GemmParams p = {};
    const kq_status st = check_size(n, k);
    if (st != KQ_OK) return st;
    if (lddw < k) return KQ_ERR_ARG;
    return checkpoint_grad(Product::GradWeight, p, dY, type, ldy, m, n, k, q, exps, dW, lddw, dbias, ws, ws_bytes,
                           (hipStream_t)stream);
}

}  // extern "C"
