// C ABI of the 8-bit fully-connected layer: argument checks and launches.  As everywhere in the library, the
// arguments are checked before HIP is touched and nothing is allocated.
#include "kq_block.h"

using namespace kq;

namespace {

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
bool plain_type(int32_t t) { return t == KQ_T_F32 || t == KQ_T_BF16 || t == KQ_T_F16; }
bool valid_tensor(const void* p, int32_t type, int64_t ld, int64_t cols) {
    return p != nullptr && aligned(p, type == KQ_T_F32 ? 4 : 2) && ld >= cols && ld <= (int64_t(1) << 40);
}
bool valid_blocks(const uint8_t* values, const uint8_t* exps) { return values && aligned(values, 16) && exps; }
kq_status hip_status(hipError_t e) { return e == hipSuccess ? KQ_OK : KQ_ERR_HIP; }

kq_status check_matrix(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 1) return KQ_ERR_ARG;
    if (rows > KQ_GROUP_MAX_FEATURES || cols > KQ_GROUP_MAX_FEATURES || rows * cols > KQ_GROUP_MAX_VALUES) return KQ_ERR_UNSUPPORTED;
    return KQ_OK;
}
// a weight [n][k] and m rows of n and of k values
kq_status check_layer(int64_t m, int64_t n, int64_t k) {
    if (n < 1 || m < 0) return KQ_ERR_ARG;
    const kq_status st = check_matrix(n, k);
    if (st != KQ_OK) return st;
    if (m > KQ_GROUP_MAX_ROWS || m * n > KQ_GROUP_MAX_VALUES || m * k > KQ_GROUP_MAX_VALUES) return KQ_ERR_UNSUPPORTED;
    return KQ_OK;
}
kq_status check_ws(void* ws, size_t ws_bytes, size_t need) {
    if (need == 0) return KQ_OK;
    return ws == nullptr || !aligned(ws, 256) || ws_bytes < need ? KQ_ERR_WORKSPACE : KQ_OK;
}
size_t region(int64_t bytes) { return ((size_t)bytes + 255) & ~size_t(255); }

// the regions of a workspace in turn
struct Regions {
    char* at;
    template <class T = uint8_t>
    T* take(size_t bytes) {
        T* const p = (T*)at;
        at += bytes;
        return p;
    }
};

struct GradInputSizes {
    BlockGemmPlan plan;
    size_t dy, dy_exps, total;
    GradInputSizes(int32_t type, int64_t m, int64_t n, int64_t k) : plan(block_gemm_plan(type == KQ_T_F32, k, m, n)) {
        const int64_t np = block_pitch(n);
        dy = region(m * np);
        dy_exps = region(m * (np / kBlock));
        total = plan.part_bytes + dy + dy_exps;
    }
};
// The bias' gradient: the transposing pass leaves a sum for each 128 rows and the product adds them where it writes its first
// columns.  More of them than kBiasParts are added in kBiasGroups groups before, so that no workgroup waits for a long
// sum (32768 x 1024 x 1024: 168 us without the groups, 126 with them and 110 to 130 without a bias; one million rows of
// 128 x 128: 3.37 ms, 0.53 and 0.52).
constexpr int64_t kBiasParts = 64, kBiasGroups = 32;

struct GradWeightSizes {
    BlockGemmPlan plan;
    size_t dyt, dyt_exps, xt, xt_exps, sums, total;
    GradWeightSizes(int32_t dw_type, int64_t m, int64_t n, int64_t k) : plan(block_gemm_plan(dw_type == KQ_T_F32, k, n, m)) {
        const int64_t mp = block_pitch(m);
        dyt = region(n * mp);
        dyt_exps = region(n * (mp / kBlock));
        xt = region(k * mp);
        xt_exps = region(k * (mp / kBlock));
        sums = region((mp / kBlock + (mp / kBlock > kBiasParts ? kBiasGroups : 0)) * n * 4);
        total = plan.part_bytes + dyt + dyt_exps + xt + xt_exps + sums;
    }
};

}  // namespace

namespace kq {

// Few rows are multiplied row by row of W, others in large tiles: up to 16 the former is always the faster, beyond the two plans'
// modelled times decide (the quantizer's launch takes 2.8 us, of fp32 4.2).
BlockLinearPlan block_linear_plan(int x_type, int y_type, int64_t m, int64_t n, int64_t k) {
    BlockLinearPlan z = {};
    z.few = m <= kBlockMatvecRows;
    if (z.few) {
        z.few_plan = block_matvec_plan((int)m, n, k);
    } else {
        z.plan = block_gemm_plan(y_type == KQ_T_F32, n, m, k);
        if (m <= kBlockMatvecMost) {
            z.few_plan = block_matvec_plan(x_type, (int)m, n, k);
            z.few = z.few_plan.us < z.plan.us + (x_type == KQ_T_E4M3 ? 0.0f : x_type == KQ_T_F32 ? 4.2f : 2.8f);
        }
    }
    z.total = z.few_plan.ws_bytes;
    if (z.few) return z;
    z.x = x_type == KQ_T_E4M3 ? 0 : region(m * block_pitch(k));
    z.x_exps = x_type == KQ_T_E4M3 ? 0 : region(m * (block_pitch(k) / kBlock));
    z.total = z.plan.part_bytes + z.x + z.x_exps;
    return z;
}

}  // namespace kq

extern "C" {

kq_status kq_quantize_blocks(const void* X, int32_t type, int64_t ldx, int64_t m, int64_t k, int32_t rows, uint8_t* values,
                             uint8_t* exps, void* stream) {
    const kq_status st = check_matrix(m, k);
    if (st != KQ_OK) return st;
    if (!plain_type(type) || (rows != 1 && rows != kBlock)) return KQ_ERR_UNSUPPORTED;
    if (m == 0) return KQ_OK;
    if (!valid_tensor(X, type, ldx, k) || !valid_blocks(values, exps)) return KQ_ERR_ARG;
    const BlockQuantizeParams p = {X, ldx, type, m, k, block_pitch(k), values, exps};
    return hip_status(launch_quantize_blocks(p, rows, (hipStream_t)stream));
}

kq_status kq_reconstruct_blocks(const uint8_t* values, const uint8_t* exps, int64_t m, int64_t k, int32_t rows,
                                int32_t type, void* X_hat, int64_t ldx, void* stream) {
    const kq_status st = check_matrix(m, k);
    if (st != KQ_OK) return st;
    if (!plain_type(type) || (rows != 1 && rows != kBlock)) return KQ_ERR_UNSUPPORTED;
    if (m == 0) return KQ_OK;
    if (!valid_tensor(X_hat, type, ldx, k) || !valid_blocks(values, exps)) return KQ_ERR_ARG;
    const BlockReconstructParams p = {values, exps, m, k, block_pitch(k), rows, X_hat, ldx, type};
    return hip_status(launch_reconstruct_blocks(p, (hipStream_t)stream));
}

size_t kq_block_linear_workspace_bytes(int32_t x_type, int32_t y_type, int64_t m, int64_t n, int64_t k) {
    if (m < 1 || check_layer(m, n, k) != KQ_OK || !(plain_type(x_type) || x_type == KQ_T_E4M3) || !plain_type(y_type)) return 0;
    return block_linear_plan(x_type, y_type, m, n, k).total;
}

kq_status kq_block_linear(const void* X, int32_t x_type, int64_t ldx, const uint8_t* x_exps, int64_t m, int64_t n, int64_t k,
                          const uint8_t* values, const uint8_t* exps, const float* bias, void* Y, int32_t y_type,
                          int64_t ldy, void* ws, size_t ws_bytes, void* stream) {
    kq_status st = check_layer(m, n, k);
    if (st != KQ_OK) return st;
    const bool ready = x_type == KQ_T_E4M3;
    if (!(plain_type(x_type) || ready) || !plain_type(y_type)) return KQ_ERR_UNSUPPORTED;
    if (!valid_blocks(values, exps) || !aligned(bias, 4)) return KQ_ERR_ARG;
    if (m == 0) return KQ_OK;
    const int64_t kp = block_pitch(k);
    if (ready ? !valid_blocks((const uint8_t*)X, x_exps) || ldx != kp : x_exps != nullptr || !valid_tensor(X, x_type, ldx, k))
        return KQ_ERR_ARG;
    if (!valid_tensor(Y, y_type, ldy, n)) return KQ_ERR_ARG;
    const hipStream_t s = (hipStream_t)stream;
    const BlockLinearPlan z = block_linear_plan(x_type, y_type, m, n, k);
    if ((st = check_ws(ws, ws_bytes, z.total)) != KQ_OK) return st;
    if (z.few) {
        const BlockMatvecParams p = {values, exps, n, k, kp, X, x_type, ldx, x_exps, (int)m, bias, Y, y_type, ldy,
                                     (float*)ws, 1, 0};
        return hip_status(launch_block_matvec(z.few_plan, p, s));
    }
    Regions r = {(char*)ws};
    float* const part = r.take<float>(z.plan.part_bytes);
    const uint8_t* xv = (const uint8_t*)X;
    if (!ready) {
        const BlockQuantizeParams q = {X, ldx, x_type, m, k, kp, r.take(z.x), r.take(z.x_exps)};
        const hipError_t e = launch_quantize_blocks(q, 1, s);
        if (e != hipSuccess) return hip_status(e);
        xv = q.values;
        x_exps = q.exps;
    }
    BlockGemmParams p = {};
    p.A = {values, kp, exps, kp / kBlock, 1};
    p.B = {xv, kp, x_exps, kp / kBlock, 1};
    p.I = n;
    p.J = m;
    p.steps = (int)(kp / kBlock);
    p.bias = bias;
    p.out = Y;
    p.type = y_type;
    p.ldo = ldy;
    return hip_status(launch_block_gemm(y_type == KQ_T_F32, kFormBlocks, z.plan, p, part, s));
}

size_t kq_block_linear_grad_input_workspace_bytes(int32_t type, int64_t m, int64_t n, int64_t k) {
    if (m < 1 || check_layer(m, n, k) != KQ_OK || !plain_type(type)) return 0;
    return GradInputSizes(type, m, n, k).total;
}

kq_status kq_block_linear_grad_input(const void* dY, int32_t type, int64_t ldy, int64_t m, int64_t n, int64_t k,
                                     const uint8_t* values, const uint8_t* exps, void* dX, int64_t ldx, void* ws,
                                     size_t ws_bytes, void* stream) {
    kq_status st = check_layer(m, n, k);
    if (st != KQ_OK) return st;
    if (!plain_type(type)) return KQ_ERR_UNSUPPORTED;
    if (!valid_blocks(values, exps)) return KQ_ERR_ARG;
    if (m == 0) return KQ_OK;
    if (!valid_tensor(dY, type, ldy, n) || !valid_tensor(dX, type, ldx, k)) return KQ_ERR_ARG;
    const GradInputSizes z(type, m, n, k);
    if ((st = check_ws(ws, ws_bytes, z.total)) != KQ_OK) return st;
    const hipStream_t s = (hipStream_t)stream;
    Regions r = {(char*)ws};
    float* const part = r.take<float>(z.plan.part_bytes);
    const int64_t np = block_pitch(n), kp = block_pitch(k);
    const BlockQuantizeParams q = {dY, ldy, type, m, n, np, r.take(z.dy), r.take(z.dy_exps)};
    const hipError_t e = launch_quantize_blocks(q, 1, s);
    if (e != hipSuccess) return hip_status(e);
    BlockGemmParams p = {};
    p.A = {values, kp, exps, 1, kp / kBlock};  // row block of W^T = column block of W
    p.depth = n;
    p.a_cols = kp;
    p.B = {q.values, np, q.exps, np / kBlock, 1};
    p.I = k;
    p.J = m;
    p.steps = (int)(np / kBlock);
    p.out = dX;
    p.type = type;
    p.ldo = ldx;
    return hip_status(launch_block_gemm(type == KQ_T_F32, kFormColumns, z.plan, p, part, s));
}

size_t kq_block_linear_grad_weight_workspace_bytes(int32_t dw_type, int64_t m, int64_t n, int64_t k) {
    if (m < 1 || check_layer(m, n, k) != KQ_OK || !plain_type(dw_type)) return 0;
    return GradWeightSizes(dw_type, m, n, k).total;
}

kq_status kq_block_linear_grad_weight(const void* dY, int32_t type, int64_t ldy, int64_t m, int64_t n, int64_t k,
                                      const uint8_t* x_values, const uint8_t* x_exps, void* dW, int32_t dw_type,
                                      int64_t lddw, float* dbias, void* ws, size_t ws_bytes, void* stream) {
    kq_status st = check_layer(m, n, k);
    if (st != KQ_OK) return st;
    if (!plain_type(type) || !plain_type(dw_type)) return KQ_ERR_UNSUPPORTED;
    if (!valid_tensor(dW, dw_type, lddw, k) || !aligned(dbias, 4)) return KQ_ERR_ARG;
    // without rows there is nothing to read, and the gradients are zero
    if (m > 0 && (!valid_tensor(dY, type, ldy, n) || !valid_blocks(x_values, x_exps))) return KQ_ERR_ARG;
    const GradWeightSizes z(dw_type, m, n, k);
    if (m > 0 && (st = check_ws(ws, ws_bytes, z.total)) != KQ_OK) return st;
    const hipStream_t s = (hipStream_t)stream;
    const int64_t mp = block_pitch(m), kp = block_pitch(k);
    BlockGemmParams p = {};
    p.I = k;
    p.J = n;
    p.steps = (int)(mp / kBlock);
    p.out = dW;
    p.type = dw_type;
    p.ldo = lddw;
    float* part = nullptr;
    if (m > 0) {
        Regions r = {(char*)ws};
        part = r.take<float>(z.plan.part_bytes);
        const BlockTransposeParams g = {dY, ldy, type, nullptr, m, n, mp, r.take(z.dyt), r.take(z.dyt_exps),
                                        dbias ? r.take<float>(z.sums) : nullptr};
        const BlockTransposeParams x = {x_values, kp, KQ_T_E4M3, x_exps, m, k, mp, r.take(z.xt), r.take(z.xt_exps), nullptr};
        hipError_t e = launch_grad_weight_operands(x, g, s);
        if (e != hipSuccess) return hip_status(e);
        p.A = {x.values, mp, x.exps, mp / kBlock, 1};
        p.B = {g.values, mp, g.exps, mp / kBlock, 1};
        p.bias_part = g.sums;
        p.bias_parts = (int)(mp / kBlock);
        if (dbias && p.bias_parts > kBiasParts) {  // (the groups' sums follow the last of the parts; those that fill no group stay)
            const int each = p.bias_parts / (int)kBiasGroups, rest = p.bias_parts % (int)kBiasGroups;
            const JoinParams j = {g.sums, each, 1, kBiasGroups * n, nullptr, g.sums + p.bias_parts * n, kBiasGroups * n, KQ_T_F32};
            e = launch_join(j, s);
            if (e != hipSuccess) return hip_status(e);
            p.bias_part = g.sums + (int64_t)(p.bias_parts - rest) * n;
            p.bias_parts = rest + (int)kBiasGroups;
        }
    }
    p.dbias = dbias;
    return hip_status(launch_block_gemm(dw_type == KQ_T_F32, kFormRows, z.plan, p, part, s));
}

}  // extern "C"
