// The product with [N, K] weights and a feed-forward layer's epilogue (bias, activation, gate, residual) in one launch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "nmm_internal.h"
#include "nt_rows.h"
#include "nt_wide.h"

namespace nmm {
namespace {

using rows::RowsParams;

constexpr int64_t kLim = int64_t(1) << 31;
constexpr int kGridMost = 2048;            // workgroups: more items than that are taken in turns
constexpr int kCus = 256;
constexpr int kCols = 128;                 // rows of the weight a tile of wide_kernel

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Tiles of 16 rows of the weight.
int64_t rows16(int64_t N, bool gated) { return cdiv(gated ? 2 * N : N, 16); }

struct ActPlan {
    int rows = 0;                // of x a tile: 4, 8, 16, 32 (rows_kernel) or 64, 128 (wide_kernel)
    int ks = 1, slice_steps = 0; // slices of K, slots of each
    size_t ws_bytes = 0;
};

// Up to 32 rows of x, and more where the weight is small, go by rows_kernel: up to 256 workgroups of 32 rows of x and 16 of the weight
// while K is at most 4096, up to 1024 while it is at most 2048 (launch_nt then takes 32 of the weight).  64 rows x 512 x 512 5.0 us, in a tile of
// wide_kernel 9.2; 64 x 2048 x 2048 7.9 and 12.2, 256 x 2048 x 2048 13.0 and 15.4 to 20.6, 64 x 7168 x 2048 15.3 and 14.8, 64 x 4096 x
// 4096 (512 workgroups) 20.2 and 15.4.
// Else tiles of 64 or 128 rows of x and 128 of the weight: 64 where they number 64 at most, so that K still goes in four slices (256 rows
// x 7168 x 1024 17.7 us against 20.5 in 128s; 100 x 16384 x 7168, 112 of them, 75.7 against 54.3).  K is cut into slices, an XCD's each, while
// that leaves at most a workgroup per CU and four slots a slice: 256 rows x 7168 x 2 x 2048 75 us whole, 32 in four slices; 128 x
// 16384 x 7168 60 in four slices, 80 whole.
ActPlan plan_act(int64_t M, int64_t K, int64_t N, bool gated) {
    ActPlan q;
    const int64_t few = cdiv(M, 32) * rows16(N, gated);
    if (M <= 32 || (few <= kCus && K <= 4096) || (few <= 4 * kCus && K <= 2048)) {
        q.rows = M <= 4 ? 4 : M <= 8 ? 8 : M <= 16 ? 16 : 32;
        return q;
    }
    const int64_t steps = cdiv(K, rows::kWideK), blocks = cdiv(N, gated ? kCols / 2 : kCols);
    q.rows = M <= 64 || cdiv(M, 64) * blocks <= kCus / 4 ? 64 : 128;
    const int64_t tiles = cdiv(M, q.rows) * blocks;
    while (q.ks < 8 && tiles * q.ks * 2 <= kCus && steps >= q.ks * 8) q.ks *= 2;
    q.slice_steps = static_cast<int>(std::max<int64_t>(1, cdiv(steps, q.ks)));
    if (q.ks > 1) q.ws_bytes = size_t(kTicketBytes) + size_t(q.ks) * M * cdiv(N, 4) * 4 * (gated ? 2 : 1) * 4;
    return q;
}

template <int DT, int XR, int NT, int NW>
void launch_rows(RowsParams p, hipStream_t s) {
    p.n_blocks = static_cast<int>(cdiv(p.N, p.gated ? 8 * NT : 16 * NT));
    const int64_t items = cdiv(p.n_blocks, 8) * 8 * cdiv(p.M, 4 * XR);
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(items, kGridMost))), block(64 * NW);
    if (p.yf) hipLaunchKernelGGL((rows::rows_kernel<DT, rows::kDense, XR, NT, NW, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((rows::rows_kernel<DT, rows::kDense, XR, NT, NW>), grid, block, 0, s, p);
}

template <int DT, int XR>
void launch_nt(const RowsParams& p, hipStream_t s) {
    // 16 rows of the weight a workgroup, its four waves sharing K, while every one finds a CU of its own (gated, one row x 7168 x 2 x 2048
    // 11.5 us against 16.9 in 32s; 8 x 4096 x 4096 9.9 and 12.0); else 32 rows and two waves, of which three workgroups share a CU up to 16
    // rows of x (41 to 53 KB of LDS) and two at 32 (74 KB), where 16s have a CU each at 32 rows (32 x 16384 x 7168 45.1 us
    // against 58.5, 8 x 4096 x 5120 12.1 and 12.6, one row x 7168 x 8192 20.3 both)
    if (cdiv(p.M, 4 * XR) * rows16(p.N, p.gated != 0) <= kCus) launch_rows<DT, XR, 1, 4>(p, s);
    else launch_rows<DT, XR, 2, 2>(p, s);
}

template <int DT, int BM>
void launch_wide(RowsParams p, hipStream_t s) {
    p.n_blocks = static_cast<int>(cdiv(p.N, p.gated ? kCols / 2 : kCols));
    const int64_t items = cdiv(p.n_blocks, 8 / p.ks) * 8 * cdiv(p.M, BM);
    const dim3 grid(static_cast<uint32_t>(std::min<int64_t>(items, kGridMost))), block(rows::kWideThreads);
    if (p.yf) hipLaunchKernelGGL((rows::wide_kernel<DT, rows::kDense, BM, kCols, 3, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((rows::wide_kernel<DT, rows::kDense, BM, kCols, 3>), grid, block, 0, s, p);
    if (p.ks == 1) return;
    const dim3 all(static_cast<uint32_t>(cdiv(p.M * cdiv(p.N, 4), rows::kFinishThreads)));
    hipLaunchKernelGGL((rows::finish_kernel<DT>), all, dim3(rows::kFinishThreads), 0, s, p);
}

template <int DT>
void launch(const RowsParams& p, const ActPlan& q, hipStream_t s) {
    switch (q.rows) {
        case 4: return launch_nt<DT, 1>(p, s);
        case 8: return launch_nt<DT, 2>(p, s);
        case 16: return launch_nt<DT, 4>(p, s);
        case 32: return launch_nt<DT, 8>(p, s);
        case 64: return launch_wide<DT, 64>(p, s);
        default: return launch_wide<DT, 128>(p, s);
    }
}

}  // namespace

bool rows_overlap(const void* a, int64_t lda, int64_t wa, const void* b, int64_t ldb, int64_t wb, int64_t n) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    if (!a || !b || n <= 0 || wa <= 0 || wb <= 0) return false;
    if (pa + uintptr_t((n - 1) * lda + wa) <= pb || pb + uintptr_t((n - 1) * ldb + wb) <= pa) return false;
    if (lda != ldb || n == 1) return true;
    const uintptr_t d = (pb >= pa ? pb - pa : uintptr_t(lda) - (pa - pb) % uintptr_t(lda)) % uintptr_t(lda);
    return d < uintptr_t(wa) || d + uintptr_t(wb) > uintptr_t(lda);
}

}  // namespace nmm

using namespace nmm;

extern "C" {

size_t nmm_gemv_nt_act_workspace_size(const nmm_nt_act* product) {
    if (!product || product->M <= 0 || product->K <= 0 || product->N <= 0 || product->M >= kLim || product->K >= kLim ||
        product->N >= kLim)
        return 0;
    return plan_act(product->M, product->K, product->N, product->gated != 0).ws_bytes;
}

nmm_status nmm_gemv_nt_act(const nmm_nt_act* product, void* workspace, size_t workspace_bytes, void* stream) {
    if (!product) return NMM_ERR_NULL;
    const nmm_nt_act& a = *product;
    if (a.dt != NMM_F16 && a.dt != NMM_BF16) return NMM_ERR_DTYPE;
    if (a.M < 0 || a.K < 0 || a.N < 0 || a.M >= kLim || a.K >= kLim || a.N >= kLim) return NMM_ERR_SHAPE;
    if (a.act < NMM_ACT_NONE || a.act > NMM_ACT_GELU_TANH || a.gated < 0 || a.gated > 1) return NMM_ERR_ARG;
    if (a.M == 0 || a.N == 0) return NMM_OK;
    if (!a.y && !a.y_f32) return NMM_ERR_NULL;
    if (a.y && (a.ldy < a.N || a.ldy >= kLim)) return NMM_ERR_SHAPE;
    if (a.y_f32 && (a.ldyf < a.N || a.ldyf >= kLim)) return NMM_ERR_SHAPE;
    if (a.residual && (a.ldr < a.N || a.ldr >= kLim)) return NMM_ERR_SHAPE;
    if (!aligned(a.y, 2) || !aligned(a.y_f32, 4) || !aligned(a.bias, 2) || !aligned(a.residual, 2)) return NMM_ERR_ALIGN;
    const int64_t n_rows = a.gated ? 2 * a.N : a.N, k8 = cdiv(a.K, 8) * 8;
    if (n_rows >= kLim / 2) return NMM_ERR_SHAPE;
    if (a.K > 0) {
        if (!a.x || !a.Wt) return NMM_ERR_NULL;
        if (a.ldx < a.K || a.ldx >= kLim || a.ldwt < a.K || a.ldwt >= kLim) return NMM_ERR_SHAPE;
        if (!aligned(a.x, 16) || !aligned(a.Wt, 16) || a.ldx % 8 || a.ldwt % 8) return NMM_ERR_ALIGN;
        // buffer offsets are 32-bit: the weight, and the rows of x in a block
        if (((n_rows - 1) * a.ldwt + k8) * 2 >= kLim) return NMM_ERR_SHAPE;
        if (((std::min<int64_t>(a.M, 128) - 1) * a.ldx + k8) * 2 >= kLim) return NMM_ERR_SHAPE;
    }
    const bool in_place = a.residual && a.residual == a.y && a.ldr == a.ldy;
    if (!in_place && rows_overlap(a.residual, 2 * a.ldr, 2 * a.N, a.y, 2 * a.ldy, 2 * a.N, a.M)) return NMM_ERR_ARG;
    if (a.K > 0 && (rows_overlap(a.x, 2 * a.ldx, 2 * a.K, a.y, 2 * a.ldy, 2 * a.N, a.M) ||
                    rows_overlap(a.x, 2 * a.ldx, 2 * a.K, a.y_f32, 4 * a.ldyf, 4 * a.N, a.M)))
        return NMM_ERR_ARG;
    if (rows_overlap(a.residual, 2 * a.ldr, 2 * a.N, a.y_f32, 4 * a.ldyf, 4 * a.N, a.M) ||
        rows_overlap(a.y, 2 * a.ldy, 2 * a.N, a.y_f32, 4 * a.ldyf, 4 * a.N, a.M))
        return NMM_ERR_ARG;
    const ActPlan q = plan_act(a.M, a.K, a.N, a.gated != 0);
    const nmm_status st = validate_workspace(workspace, workspace_bytes, q.ws_bytes);
    if (st != NMM_OK) return st;
    RowsParams p{};
    p.ks = q.ks;
    p.slice_steps = q.slice_steps;
    if (q.ks > 1) {
        p.ld_part = cdiv(a.N, 4) * 4 * (a.gated ? 2 : 1);
        p.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kTicketBytes);
    }
    p.rot = rows::rotation(a.ldwt);
    p.x = static_cast<const uint16_t*>(a.x);
    if (a.K > 0) {             // (0: extents of nothing)
        p.ldx = a.ldx;
        p.w = static_cast<const uint8_t*>(a.Wt);
        p.row_bytes = static_cast<uint32_t>(a.ldwt * 2);
        p.w_extent = static_cast<uint32_t>(((n_rows - 1) * a.ldwt + k8) * 2);
    }
    p.K = static_cast<int>(a.K);
    p.N = static_cast<int>(a.N);
    p.M = static_cast<int>(a.M);
    p.gated = a.gated;
    p.act = a.act;
    p.bias = static_cast<const uint16_t*>(a.bias);
    p.res = static_cast<const uint16_t*>(a.residual);
    p.ldr = a.ldr;
    p.y = static_cast<uint16_t*>(a.y);
    p.ldy = a.ldy;
    p.yf = a.y_f32;
    p.ldyf = a.ldyf;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (a.dt == NMM_BF16) launch<NMM_BF16>(p, q, s);
    else launch<NMM_F16>(p, q, s);
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
