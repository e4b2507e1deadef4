// The gated feed-forward block for few rows (a token, a handful of them): bound by the weights, which are read once.
//
// 16-bit types: a CTA takes 8 rows of Wg and the same 8 of Wu, which are the 16 rows of one tensor-core fragment (mma.sync
// m16n8k16: the products are far from counting here, and fragments come straight from global memory without a tile in between);
// its warps share the summed axis.  The sum does not care for the order along that axis, so a lane takes 8 consecutive
// elements of its row (16 bytes) as its part of two products, and the same elements of x: whole 64-byte pieces of a row per load,
// no shuffles, no shared memory before the end.  All of a warp's loads of a turn are issued before the first is used.
//
// Binary32: a warp takes one row of Wg and of Wu, lanes along the summed axis, products on the CUDA cores.
#include <type_traits>

#include "bt_glu.cuh"

namespace bt {
namespace {

struct RowsArgs {
    const void *x, *w_gate, *w_up;
    void       *h, *g, *u;
    uint32_t    rows, d_in, d_ff;
    int32_t    *dev_status;
};

constexpr int kWarps   = 8;
constexpr int kColumns = 8;       // rows of each weight matrix per CTA
constexpr int kAhead   = 8;       // pieces of 32 summed elements that a warp loads ahead

__device__ __forceinline__ uint4 load_stream(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

template <int DT>
__device__ __forceinline__ void mma16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    if constexpr (DT == BT_BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int DT, int kAct>
__device__ __forceinline__ void write_outputs(const RowsArgs &p, const uint32_t row, const uint32_t f, const typename Num<DT>::Acc g, const typename Num<DT>::Acc u)
{
    using Elem           = typename Num<DT>::Elem;
    const uint64_t at    = static_cast<uint64_t>(row) * p.d_ff + f, bytes = static_cast<uint64_t>(p.rows) * p.d_ff * sizeof(Elem);
    const auto     store = [&](void *to, const typename Num<DT>::Acc v) {
        Elem *const o = static_cast<Elem *>(to) + at;
        if (extent_of(to, bytes).holds(o, sizeof(Elem))) *o = Num<DT>::narrow(v);
    };
    typename Num<DT>::Acc act;
    if constexpr (DT == BT_F32) act = act_of<kAct>(g);
    else act = act_short<kAct>(g);
    store(p.h, act * u);
    if (p.g) store(p.g, kAct == BT_ACT_RELU ? act : g);
    if (p.u) store(p.u, u);
}

// kTiles: groups of 8 rows of x
template <int DT, int kAct, int kTiles>
__global__ void __launch_bounds__(32 * kWarps)
glu_rows_kernel(const RowsArgs p)
{
    in_stream_order();
    __shared__ float sums[kWarps][kTiles][16][kColumns + 1];           // [warp][rows of x][weight row: g, u][row]
    if (p.dev_status && blockIdx.x == 0 && threadIdx.x == 0) *p.dev_status = BT_OK;
    const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, quad = lane / 4, part = lane % 4;
    const uint32_t f0 = blockIdx.x * kColumns, f = f0 + quad < p.d_ff ? f0 + quad : p.d_ff - 1;
    const uint32_t vecs = p.d_in / 8;                                  // of a row
    const uint4 *const wg = static_cast<const uint4 *>(p.w_gate) + static_cast<uint64_t>(f) * vecs;
    const uint4 *const wu = static_cast<const uint4 *>(p.w_up) + static_cast<uint64_t>(f) * vecs;
    const uint4       *x[kTiles];
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
        const uint32_t row = n * 8 + quad < p.rows ? n * 8 + quad : p.rows - 1;      // (a row beyond the last is computed and dropped)
        x[n] = static_cast<const uint4 *>(p.x) + static_cast<uint64_t>(row) * vecs;
    }
    float d[kTiles][4] = {};
    const uint32_t pieces = (vecs + 3) / 4;                            // of 32 elements
    for (uint32_t piece0 = warp; piece0 < pieces; piece0 += kWarps * kAhead) {
        uint4 a[kAhead], b[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint32_t v = (piece0 + k * kWarps) * 4 + part;
            const bool     in = v < vecs;
            a[k] = in ? load_stream(wg + v) : make_uint4(0, 0, 0, 0);
            b[k] = in ? load_stream(wu + v) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const uint32_t v = (piece0 + k * kWarps) * 4 + part;
#pragma unroll
            for (int n = 0; n < kTiles; ++n) {
                const uint4 c = v < vecs ? __ldg(x[n] + v) : make_uint4(0, 0, 0, 0);
                mma16<DT>(d[n], a[k].x, b[k].x, a[k].y, b[k].y, c.x, c.y);
                mma16<DT>(d[n], a[k].z, b[k].z, a[k].w, b[k].w, c.z, c.w);
            }
        }
    }
    // fragment: weight rows quad (of Wg) and quad + 8 (of Wu), rows of x 2 * part and 2 * part + 1
#pragma unroll
    for (int n = 0; n < kTiles; ++n) {
        sums[warp][n][quad][2 * part]         = d[n][0];
        sums[warp][n][quad][2 * part + 1]     = d[n][1];
        sums[warp][n][quad + 8][2 * part]     = d[n][2];
        sums[warp][n][quad + 8][2 * part + 1] = d[n][3];
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < kTiles * 8 * kColumns; e += 32 * kWarps) {
        const uint32_t n = e / 64, row = e / 8 % 8, c = e % 8;
        if (n * 8 + row >= p.rows || f0 + c >= p.d_ff) continue;
        float g = 0, u = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) g += sums[w][n][c][row], u += sums[w][n][c + 8][row];
        write_outputs<DT, kAct>(p, n * 8 + row, f0 + c, g, u);
    }
}

// binary32: kRows rows of x
template <int kAct, int kRows>
__global__ void __launch_bounds__(32 * kWarps)
glu_rows_f32_kernel(const RowsArgs p)
{
    in_stream_order();
    if (p.dev_status && blockIdx.x == 0 && threadIdx.x == 0) *p.dev_status = BT_OK;
    const uint32_t lane = threadIdx.x % 32, f = blockIdx.x * kWarps + threadIdx.x / 32, vecs = p.d_in / 4;
    if (f >= p.d_ff) return;
    const uint4 *const wg = static_cast<const uint4 *>(p.w_gate) + static_cast<uint64_t>(f) * vecs;
    const uint4 *const wu = static_cast<const uint4 *>(p.w_up) + static_cast<uint64_t>(f) * vecs;
    const uint4 *const x  = static_cast<const uint4 *>(p.x);
    Two<float> g[kRows], u[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) g[r] = u[r] = both(0.0f);
    constexpr int kUnroll = 4;
    for (uint32_t v0 = lane; v0 < vecs; v0 += 32 * kUnroll) {
        uint4 a[kUnroll], b[kUnroll];
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            const bool in = v0 + 32 * k < vecs;
            a[k] = in ? load_stream(wg + v0 + 32 * k) : make_uint4(0, 0, 0, 0);
            b[k] = in ? load_stream(wu + v0 + 32 * k) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int k = 0; k < kUnroll; ++k) {
            Two<float> ga[2], ua[2];
            widen_pairs<BT_F32>(a[k], ga), widen_pairs<BT_F32>(b[k], ua);
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const uint32_t row = r < static_cast<int>(p.rows) ? r : p.rows - 1;
                Two<float>     c[2];
                widen_pairs<BT_F32>(v0 + 32 * k < vecs ? __ldg(x + static_cast<uint64_t>(row) * vecs + v0 + 32 * k) : make_uint4(0, 0, 0, 0), c);
#pragma unroll
                for (int q = 0; q < 2; ++q) g[r] = fma2(ga[q], c[q], g[r]), u[r] = fma2(ua[q], c[q], u[r]);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
        const float gs = warp_sum(g[r].low() + g[r].high()), us = warp_sum(u[r].low() + u[r].high());
        if (lane == 0 && r < static_cast<int>(p.rows)) write_outputs<BT_F32, kAct>(p, r, f, gs, us);
    }
}

template <int DT, int kTiles>
cudaError_t start(const RowsArgs &p, int act, cudaStream_t stream)
{
    const unsigned grid = (p.d_ff + kColumns - 1) / kColumns;
    return with_act<DT>(act, [&](auto dt, auto a) {
        return launch(glu_rows_kernel<decltype(dt)::value, decltype(a)::value, kTiles>, grid, 32 * kWarps, 0, stream, p);
    });
}
template <int DT>
cudaError_t start_rows(const RowsArgs &p, int act, cudaStream_t stream)
{
    return p.rows <= 8 ? start<DT, 1>(p, act, stream) : p.rows <= 16 ? start<DT, 2>(p, act, stream) : start<DT, 4>(p, act, stream);
}
template <int kRows>
cudaError_t start_f32(const RowsArgs &p, int act, cudaStream_t stream)
{
    const unsigned grid = (p.d_ff + kWarps - 1) / kWarps;
    return with_act<BT_F32>(act, [&](auto, auto a) { return launch(glu_rows_f32_kernel<decltype(a)::value, kRows>, grid, 32 * kWarps, 0, stream, p); });
}

}  // namespace

bool glu_rows_takes(uint64_t rows, uint64_t d_in, int dtype)
{
    return dtype == BT_F32 ? rows <= 8 && d_in % 4 == 0 : (dtype == BT_F16 || dtype == BT_BF16) && rows <= 32 && d_in % 8 == 0;
}

cudaError_t launch_glu_rows(const GluCall &c, cudaStream_t stream)
{
    const RowsArgs p{c.x, c.w_gate, c.w_up, c.h, c.g, c.u, static_cast<uint32_t>(c.rows), static_cast<uint32_t>(c.d_in), static_cast<uint32_t>(c.d_ff), c.dev_status};
    if (c.dtype == BT_BF16) return start_rows<BT_BF16>(p, c.act, stream);
    if (c.dtype == BT_F16) return start_rows<BT_F16>(p, c.act, stream);
    return c.rows == 1 ? start_f32<1>(p, c.act, stream) : c.rows <= 2 ? start_f32<2>(p, c.act, stream) : c.rows <= 4 ? start_f32<4>(p, c.act, stream) : start_f32<8>(p, c.act, stream);
}

}  // namespace bt
