// The norms around a block of a residual network, with the block's gate and the scale of its residual sum:
//
//   p  = w_post ? rms(f) * w_post : f            rms(v) = v / sqrt(mean v^2 + eps)
//   x' = x + scale * gate * p                    (gate: one row for gate_rows consecutive rows)
//   n  = rms(x') * w_pre
//
// and their gradients.  Bound by HBM: the forward pass reads x and f and writes x' and n, the backward pass reads x', f, dn
// and dx' and writes dx and df; weights and gate stay in the caches.  A row is read once and kept in registers between its
// sums and its outputs; only rows longer than a CTA's registers are read again (from the caches).
//
// Backward: with r, rf the two norms' factors, q = scale * gate * w_post * f and wn = dn * w_pre,
//
//   t  = dx' + r wn - r^2 c x'   (= dx),   c  = r mean(wn x')
//   df = scale gate w_post rf t - rf^3 mean(t q) f,   mean(t q) = mean(dx' q) + r mean(wn q) - r^2 c mean(x' q)
//
// so that one reduction of six sums per row serves both norms.  The sums over rows (w_pre, w_post, gate) are held in
// binary32 by the threads that own the columns, one partial row per CTA (gate: per chunk of rows), and added up in a fixed
// order by a second kernel: no atomics, the same bits every time.
#include "bt_numeric.cuh"

namespace bt {
namespace {

struct NormArgs {
    const void *x, *f, *gate, *w_post, *w_pre;     // backward: x is x'
    const void *dn, *dy;                           // backward: gradients of n and of x' (either may be NULL)
    void       *x_out, *n_out;                     // forward; backward: dx, df
    void       *dgate, *dw_post, *dw_pre;          // backward
    float      *part_pre, *part_post, *part_gate;  // backward: partial rows (double where sums are)
    void       *stats;                             // backward, long rows: r, c, rf, mean(t q) of each row
    uint64_t    rows, d, gate_rows, chunk_rows;    // chunk_rows: consecutive rows of one team, at most
    uint32_t    chunks, group_chunks;              // group_chunks: chunks of one group of rows with a gate; 0: chunks go across groups
    double      scale, eps;
};

constexpr int      kMaxTeam   = 512;                                    // threads of a CTA that takes a row
constexpr int      kMaxWarps  = kMaxTeam / 32;
constexpr uint32_t kWarpTeams = 4;                                      // warps of a CTA whose teams are warps

// kVector: 16-byte accesses, else single elements (rows that do not all begin on a 16-byte boundary)
template <int DT, bool kVector>
struct Access {
    using Elem              = typename Num<DT>::Elem;
    using Acc               = typename Num<DT>::Acc;
    static constexpr int kW = kVector ? kLanes<DT> : 1;
    using Raw               = typename std::conditional<kVector, uint4, Elem>::type;
    __device__ static __forceinline__ Raw load(const void *row, const uint32_t i)
    {
        return static_cast<const Raw *>(row)[i];
    }
    __device__ static __forceinline__ void widen(const Raw &w, Acc (&v)[kW])
    {
        if constexpr (kVector) widen_vec<DT>(w, v);
        else v[0] = Num<DT>::widen(w);
    }
    __device__ static __forceinline__ void read(const void *row, const uint32_t i, Acc (&v)[kW]) { widen(load(row, i), v); }
    // weights and gates, which no output overlaps
    __device__ static __forceinline__ void read_shared(const void *row, const uint32_t i, Acc (&v)[kW])
    {
        widen(__ldg(static_cast<const Raw *>(row) + i), v);
    }
    __device__ static __forceinline__ void store(void *row, const uint32_t i, const Acc (&v)[kW], const Extent &e)
    {
        Raw *const p = static_cast<Raw *>(row) + i;
        if (!e.holds(p, sizeof(Raw))) return;
        if constexpr (kVector) *p = narrow_vec<DT>(v);
        else *p = Num<DT>::narrow(v[0]);
    }
};

template <typename Elem>
__device__ __forceinline__ const void *row_of(const void *base, const uint64_t row, const uint64_t d)
{
    return base ? static_cast<const void *>(static_cast<const Elem *>(base) + row * d) : nullptr;
}
template <typename Elem>
__device__ __forceinline__ void *row_of(void *base, const uint64_t row, const uint64_t d)
{
    return base ? static_cast<void *>(static_cast<Elem *>(base) + row * d) : nullptr;
}

__device__ __forceinline__ float  root_of(float v) { return rsqrtf(v); }
__device__ __forceinline__ double root_of(double v) { return rsqrt(v); }

// The sums of a team: a warp, or (kCta) the CTA.  `turn` alternates between two sets of words, so that one barrier serves a
// reduction: words are written again only behind the barrier of the reduction in between.
template <bool kCta, int kSums, typename A>
__device__ __forceinline__ void team_sums(A (&s)[kSums], A (*words)[kSums][kMaxWarps], uint32_t &turn)
{
#pragma unroll
    for (int k = 0; k < kSums; ++k) s[k] = warp_sum(s[k]);
    if constexpr (kCta) {
        const uint32_t warps = blockDim.x / 32;
        A (&w)[kSums][kMaxWarps] = words[turn & 1];
        ++turn;
        if (threadIdx.x % 32 == 0) {
#pragma unroll
            for (int k = 0; k < kSums; ++k) w[k][threadIdx.x / 32] = s[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kSums; ++k) {
            const A v = threadIdx.x % 32 < warps ? w[k][threadIdx.x % 32] : A(0);
            s[k]      = warp_sum(v);
        }
    }
}

// ---------------------------------------------------------------------------------------------- forward
// kHold accesses of each of x and f per thread; 0: rows of any length, read again for each use.
template <int DT, bool kVector, int kHold, bool kCta>
__global__ void __launch_bounds__(kCta ? kMaxTeam : 32 * kWarpTeams)
block_norm_fwd_kernel(const NormArgs a)
{
    in_stream_order();
    using X                = Access<DT, kVector>;
    using Elem             = typename X::Elem;
    using Acc              = typename X::Acc;
    constexpr int  kW      = X::kW;
    __shared__ Acc words[2][1][kMaxWarps];
    uint32_t       turn    = 0;
    const uint32_t team    = kCta ? blockDim.x : 32;
    const uint32_t t       = kCta ? threadIdx.x : threadIdx.x % 32;
    const uint32_t count   = static_cast<uint32_t>(a.d / kW);
    const Acc      scale = static_cast<Acc>(a.scale), eps = static_cast<Acc>(a.eps), of_d = Acc(1) / static_cast<Acc>(a.d);
    const uint64_t first   = kCta ? blockIdx.x : static_cast<uint64_t>(blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32;
    const uint64_t step    = kCta ? gridDim.x : static_cast<uint64_t>(gridDim.x) * (blockDim.x / 32);
    const Extent   all_x = extent_of(a.x_out, a.rows * a.d * sizeof(Elem)), all_n = extent_of(a.n_out, a.rows * a.d * sizeof(Elem));
    for (uint64_t row = first; row < a.rows; row += step) {
        const void *x = row_of<Elem>(a.x, row, a.d), *f = row_of<Elem>(a.f, row, a.d);
        const void *gate = a.gate ? row_of<Elem>(a.gate, row / a.gate_rows, a.d) : nullptr;
        void       *x_out = row_of<Elem>(a.x_out, row, a.d), *n_out = row_of<Elem>(a.n_out, row, a.d);
        if constexpr (kHold > 0) {
            Acc v[kHold][kW];
            if (f) {
                Acc fv[kHold][kW], s[1] = {0};
#pragma unroll
                for (int j = 0; j < kHold; ++j)
                    if (j * team + t < count) {
                        X::read(f, j * team + t, fv[j]);
                        X::read(x, j * team + t, v[j]);
                    }
                Acc rf = 1;
                if (a.w_post) {
#pragma unroll
                    for (int j = 0; j < kHold; ++j)
                        if (j * team + t < count) {
#pragma unroll
                            for (int k = 0; k < kW; ++k) s[0] += fv[j][k] * fv[j][k];
                        }
                    team_sums<kCta>(s, words, turn);
                    rf = root_of(s[0] * of_d + eps);
                }
                rf *= scale;
#pragma unroll
                for (int j = 0; j < kHold; ++j)
                    if (j * team + t < count) {
                        Acc w[kW];
#pragma unroll
                        for (int k = 0; k < kW; ++k) fv[j][k] *= rf;
                        if (a.w_post) {
                            X::read_shared(a.w_post, j * team + t, w);
#pragma unroll
                            for (int k = 0; k < kW; ++k) fv[j][k] *= w[k];
                        }
                        if (gate) {
                            X::read_shared(gate, j * team + t, w);
#pragma unroll
                            for (int k = 0; k < kW; ++k) fv[j][k] *= w[k];
                        }
#pragma unroll
                        for (int k = 0; k < kW; ++k) v[j][k] += fv[j][k];
                        X::store(x_out, j * team + t, v[j], all_x);
                    }
            } else {
#pragma unroll
                for (int j = 0; j < kHold; ++j)
                    if (j * team + t < count) X::read(x, j * team + t, v[j]);
            }
            if (!n_out) continue;
            Acc s[1] = {0};
#pragma unroll
            for (int j = 0; j < kHold; ++j)
                if (j * team + t < count) {
#pragma unroll
                    for (int k = 0; k < kW; ++k) s[0] += v[j][k] * v[j][k];
                }
            team_sums<kCta>(s, words, turn);
            const Acc r = root_of(s[0] * of_d + eps);
#pragma unroll
            for (int j = 0; j < kHold; ++j)
                if (j * team + t < count) {
                    Acc w[kW];
                    X::read_shared(a.w_pre, j * team + t, w);
#pragma unroll
                    for (int k = 0; k < kW; ++k) v[j][k] = v[j][k] * r * w[k];
                    X::store(n_out, j * team + t, v[j], all_n);
                }
        } else {
            Acc rf = 1;
            if (f && a.w_post) {
                Acc s[1] = {0};
                for (uint32_t i = t; i < count; i += team) {
                    Acc w[kW];
                    X::read(f, i, w);
#pragma unroll
                    for (int k = 0; k < kW; ++k) s[0] += w[k] * w[k];
                }
                team_sums<kCta>(s, words, turn);
                rf = root_of(s[0] * of_d + eps);
            }
            rf *= scale;
            const auto sum_at = [&](const uint32_t i, Acc (&v)[kW]) {
                X::read(x, i, v);
                if (!f) return;
                Acc p[kW], w[kW];
                X::read(f, i, p);
#pragma unroll
                for (int k = 0; k < kW; ++k) p[k] *= rf;
                if (a.w_post) {
                    X::read_shared(a.w_post, i, w);
#pragma unroll
                    for (int k = 0; k < kW; ++k) p[k] *= w[k];
                }
                if (gate) {
                    X::read_shared(gate, i, w);
#pragma unroll
                    for (int k = 0; k < kW; ++k) p[k] *= w[k];
                }
#pragma unroll
                for (int k = 0; k < kW; ++k) v[k] += p[k];
            };
            Acc r = 0;
            if (n_out) {
                Acc s[1] = {0};
                for (uint32_t i = t; i < count; i += team) {
                    Acc v[kW];
                    sum_at(i, v);
#pragma unroll
                    for (int k = 0; k < kW; ++k) s[0] += v[k] * v[k];
                }
                team_sums<kCta>(s, words, turn);
                r = root_of(s[0] * of_d + eps);
            }
            for (uint32_t i = t; i < count; i += team) {
                Acc v[kW], w[kW];
                sum_at(i, v);
                if (f) X::store(x_out, i, v, all_x);
                if (!n_out) continue;
                X::read_shared(a.w_pre, i, w);
#pragma unroll
                for (int k = 0; k < kW; ++k) v[k] = v[k] * r * w[k];
                X::store(n_out, i, v, all_n);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------- backward
// What a row's outputs need besides its elements.
template <typename Acc>
struct RowFactors {
    Acc r, rrc;      // dn's factor; r^2 c
    Acc rf, rf3m;    // df's factor; rf^3 mean(t q)
};
template <typename Acc>
__device__ __forceinline__ RowFactors<Acc> factors_of(const Acc (&s)[6], const Acc of_d, const Acc eps, const bool post)
{
    RowFactors<Acc> q;
    q.r            = root_of(s[0] * of_d + eps);
    q.rrc          = q.r * q.r * (q.r * (s[1] * of_d));
    q.rf           = post ? root_of(s[2] * of_d + eps) : Acc(1);
    const Acc mean = (s[3] + q.r * s[4] - q.rrc * s[5]) * of_d;
    q.rf3m         = post ? q.rf * q.rf * q.rf * mean : Acc(0);
    return q;
}

// one element's share of a row's six sums: x', f, dx', wn = dn w_pre and gw = scale gate w_post
template <typename Acc>
__device__ __forceinline__ void add_sums(Acc (&s)[6], const Acc x, const Acc f, const Acc dy, const Acc wn, const Acc gw)
{
    const Acc q = gw * f;
    s[0] += x * x;
    s[1] += wn * x;
    s[2] += f * f;
    s[3] += dy * q;
    s[4] += wn * q;
    s[5] += x * q;
}

// The chunk of rows of a team.  Where the groups of rows that share a gate row are few, no chunk goes across groups
// (group_chunks); a chunk may then be empty.  A group that lies inside one chunk has its gate's gradient written at once; of one of
// several chunks every chunk leaves a partial row -- where the group begins in the chunk in slot 2 * chunk + 1, where it came from
// the chunk before in slot 2 * chunk.
struct Chunk {
    uint64_t first, end;
};
__device__ __forceinline__ Chunk chunk_of(const NormArgs &a, const uint32_t chunk)
{
    Chunk    c;
    uint64_t end = a.rows;
    if (a.group_chunks) {
        const uint64_t group = chunk / a.group_chunks, begin = group * a.gate_rows;
        end     = begin + a.gate_rows < a.rows ? begin + a.gate_rows : a.rows;
        c.first = begin + (chunk % a.group_chunks) * a.chunk_rows;
        if (c.first > end) c.first = end;
    } else {
        c.first = chunk * a.chunk_rows;
    }
    c.end = c.first + a.chunk_rows < end ? c.first + a.chunk_rows : end;
    return c;
}
// the chunk that a row lies in
__device__ __forceinline__ uint64_t chunk_at(const NormArgs &a, const uint64_t row)
{
    return a.group_chunks ? row / a.gate_rows * a.group_chunks + row % a.gate_rows / a.chunk_rows : row / a.chunk_rows;
}
// where the sum over the rows [.., row] of a chunk's last group goes: true if it is whole
__device__ __forceinline__ bool whole_group(const NormArgs &a, const Chunk &c, const uint64_t group, const uint32_t chunk, uint64_t &slot)
{
    const uint64_t begin = group * a.gate_rows, end = begin + a.gate_rows < a.rows ? begin + a.gate_rows : a.rows;
    slot = 2ull * chunk + (begin >= c.first ? 1 : 0);
    return begin >= c.first && end <= c.end;
}

// ---------------------------------------------------------------------------------------------- rows through a ring
// A CTA per row, and a ring of rows in shared memory, filled by asynchronous copies several rows ahead (RowRing).  The work on
// consecutive rows overlaps, so that one barrier per row serves all its sums: while a row's sums meet, the next
// row's are taken and the outputs of the one before are written.
__device__ __forceinline__ void copy_ahead(void *to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copy_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

// Eight sums over a warp by exchanges of halves (9 shuffles in place of 40): the lane ends with sum number lane / 4.
template <typename A>
__device__ __forceinline__ A warp_sums8(A (&v)[8])
{
    const uint32_t lane = threadIdx.x % 32;
#pragma unroll
    for (int half = 4; half >= 1; half /= 2) {
        const bool up = lane & (4 * half);
#pragma unroll
        for (int k = 0; k < half; ++k) {
            const A give = up ? v[k] : v[k + half], keep = up ? v[k + half] : v[k];
            v[k] = keep + __shfl_xor_sync(0xFFFFFFFFu, give, 4 * half);
        }
    }
    A s = v[0] + __shfl_xor_sync(0xFFFFFFFFu, v[0], 2);
    return s + __shfl_xor_sync(0xFFFFFFFFu, s, 1);
}
// kSums of the eight sums over the CTA's warps (at most 16 of them), the same in every lane
template <int kSums, typename A>
__device__ __forceinline__ void cta_sums(const A (*part)[8], const uint32_t warps, A (&s)[kSums])
{
    const uint32_t lane = threadIdx.x % 32;
    A              v    = 0;
#pragma unroll
    for (uint32_t k = 0; k < kMaxWarps / 4; ++k) {
        const uint32_t w = k * 4 + lane / 8;
        if (w < warps) v += part[w][lane % 8];
    }
    v += __shfl_xor_sync(0xFFFFFFFFu, v, 8);
    v += __shfl_xor_sync(0xFFFFFFFFu, v, 16);
#pragma unroll
    for (int k = 0; k < kSums; ++k) s[k] = __shfl_sync(0xFFFFFFFFu, v, k);
}
// the sum over a warp's lanes and over the CTA's warps, in two steps
template <typename A>
__device__ __forceinline__ A cta_sum(const A *part, const uint32_t warps)
{
    const uint32_t lane = threadIdx.x % 32;
    return warp_sum(lane < warps ? part[lane] : A(0));
}

// rows of the ring (rows that are copied by all: one more, see RowRing)
template <int kHold, bool kVector>
constexpr uint32_t kRingStages = !kVector ? 4 : kHold == 1 ? 5 : 3;

// What a thread holds of a row, two columns at a time: kHold times kP pairs.  kVector: kHold vectors of 16 bytes, `team` vectors
// apart; else kHold times eight single columns, `team` columns apart (rows that do not all begin on a 16-byte boundary).
template <int DT, int kHold, bool kVector>
struct Columns {
    using Elem               = typename Num<DT>::Elem;
    using Acc                = typename Num<DT>::Acc;
    using Pair               = Two<Acc>;
    static constexpr int kP  = kVector ? kPairs<DT> : 4;
    static constexpr int kES = static_cast<int>(sizeof(Elem));
    uint32_t t, team, d;

    // the column of half `h` of pair k of hold j
    __device__ __forceinline__ uint32_t column(const int j, const int k, const int h) const
    {
        return kVector ? (j * team + t) * (2 * kP) + 2 * k + h : ((j * kP + k) * 2 + h) * team + t;
    }
    __device__ __forceinline__ bool has(const int j, const int k, const int h) const { return column(j, k, h) < d; }
    __device__ __forceinline__ void fill(Pair (&v)[kP], const Acc with) const
    {
#pragma unroll
        for (int k = 0; k < kP; ++k) v[k] = both(with);
    }
    // a row of global memory that no output of the call overlaps; columns beyond it keep what v holds
    __device__ __forceinline__ void read(const Elem *row, const int j, Pair (&v)[kP]) const
    {
        if constexpr (kVector) {
            if (has(j, 0, 0)) widen_pairs<DT>(__ldg(reinterpret_cast<const uint4 *>(row) + j * team + t), v);
        } else {
#pragma unroll
            for (int k = 0; k < kP; ++k)
                v[k] = Pair::of(has(j, k, 0) ? static_cast<Acc>(Num<DT>::widen(row[column(j, k, 0)])) : v[k].low(),
                                has(j, k, 1) ? static_cast<Acc>(Num<DT>::widen(row[column(j, k, 1)])) : v[k].high());
        }
    }
    __device__ __forceinline__ void write(Elem *row, const int j, const Pair (&v)[kP], const Extent &all) const
    {
        if constexpr (kVector) {
            uint4 *const o = reinterpret_cast<uint4 *>(row) + j * team + t;
            if (has(j, 0, 0) && all.holds(o, 16)) *o = narrow_pairs<DT>(v);
        } else {
#pragma unroll
            for (int k = 0; k < kP; ++k) {
                Elem *const lo = row + column(j, k, 0), *const hi = row + column(j, k, 1);
                if (has(j, k, 0) && all.holds(lo, kES)) *lo = Num<DT>::narrow(v[k].low());
                if (has(j, k, 1) && all.holds(hi, kES)) *hi = Num<DT>::narrow(v[k].high());
            }
        }
    }
    // partial sums, in the sums' type
    __device__ __forceinline__ void write_sums(Acc *row, const int j, const Pair (&v)[kP], const Extent &all) const
    {
#pragma unroll
        for (int k = 0; k < kP; ++k) {
            Acc *const lo = row + column(j, k, 0), *const hi = row + column(j, k, 1);
            if (has(j, k, 0) && all.holds(lo, sizeof(Acc))) *lo = v[k].low();
            if (has(j, k, 1) && all.holds(hi, sizeof(Acc))) *hi = v[k].high();
        }
    }
};

// The ring of rows in shared memory: `stages` rows of kOperands operands.
// kVector: every thread copies the very vectors that it reads, and needs no barrier for them.  Else a row's bytes are copied from the
// 16-byte boundary before it to the one behind it, by the CTA together: what a thread reads others have copied, so
// that a row is waited for in front of the barrier before its use.
template <int DT, int kHold, bool kVector, int kOperands>
struct RowRing {
    using C                          = Columns<DT, kHold, kVector>;
    using Elem                       = typename C::Elem;
    using Pair                       = typename C::Pair;
    static constexpr uint32_t stages = kRingStages<kHold, kVector>;
    // copies of later rows that may be under way when a turn begins (kVector), or when the barrier before it is reached
    static constexpr int kBehind = static_cast<int>(stages) - (kVector ? 2 : 3);
    const C        &c;
    unsigned char  *at;
    uint32_t        slot_bytes;

    __device__ __forceinline__ RowRing(const C &columns, void *shared, const uint32_t bytes) : c(columns), at(static_cast<unsigned char *>(shared)), slot_bytes(bytes) {}
    __device__ __forceinline__ uint4 &vector(const uint32_t stage, const int o, const int j) const
    {
        return reinterpret_cast<uint4 *>(at)[((stage * kOperands + o) * kHold + j) * c.team + c.t];
    }
    // columns beyond the row, and operands that the call leaves out, are zeros (kVector: in the ring, once)
    __device__ __forceinline__ void clear(const bool (&present)[kOperands]) const
    {
        if constexpr (kVector)
            for (uint32_t s = 0; s < stages; ++s)
#pragma unroll
                for (int j = 0; j < kHold; ++j)
#pragma unroll
                    for (int o = 0; o < kOperands; ++o)
                        if (!c.has(j, 0, 0) || !present[o]) vector(s, o, j) = make_uint4(0, 0, 0, 0);
    }
    // row `row` of a tensor that ends `total` elements behind its base
    __device__ __forceinline__ void copy(const uint32_t stage, const int o, const void *base, const uint64_t row, const uint64_t total) const
    {
        if constexpr (kVector) {
            const uint4 *const from = reinterpret_cast<const uint4 *>(static_cast<const unsigned char *>(base) + row * c.d * C::kES) + c.t;
#pragma unroll
            for (int j = 0; j < kHold; ++j)
                if (c.has(j, 0, 0)) copy_ahead(&vector(stage, o, j), from + j * c.team);
        } else {
            const uint64_t begin = row * c.d * C::kES, end = begin + c.d * C::kES, all = total * C::kES;
            unsigned char *const to = at + (stage * kOperands + o) * slot_bytes;
            for (uint64_t b = (begin & ~15ull) + 16 * c.t; b < end; b += 16 * c.team) {
                const uint32_t size = b + 16 <= all ? 16u : static_cast<uint32_t>(all - b);      // nothing is read behind the tensor
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_addr(to + (b - (begin & ~15ull)))),
                             "l"(static_cast<const unsigned char *>(base) + b), "r"(size)
                             : "memory");
            }
        }
    }
    // what this thread holds of an operand's row (`row`: its number in its tensor)
    __device__ __forceinline__ void read(const uint32_t stage, const int o, const int j, const uint64_t row, const bool present, Pair (&v)[C::kP]) const
    {
        if constexpr (kVector) {
            widen_pairs<DT>(vector(stage, o, j), v);
        } else {
            if (!present) {
                c.fill(v, 0);
                return;
            }
            const Elem *const from = reinterpret_cast<const Elem *>(at + (stage * kOperands + o) * slot_bytes + (row * c.d * C::kES & 15u));
#pragma unroll
            for (int k = 0; k < C::kP; ++k)
                v[k] = Pair::of(c.has(j, k, 0) ? static_cast<typename C::Acc>(Num<DT>::widen(from[c.column(j, k, 0)])) : typename C::Acc(0),
                                c.has(j, k, 1) ? static_cast<typename C::Acc>(Num<DT>::widen(from[c.column(j, k, 1)])) : typename C::Acc(0));
        }
    }
};

// scale * gate * w_post of a thread's columns (kRowGate: without the gate, which changes from row to row)
template <int DT, int kHold, bool kVector, bool kRowGate>
__device__ __forceinline__ void branch_factors(const NormArgs &a, const uint64_t group, const Columns<DT, kHold, kVector> &c,
                                               Two<typename Num<DT>::Acc> (&gw)[kHold][Columns<DT, kHold, kVector>::kP])
{
    using C    = Columns<DT, kHold, kVector>;
    using Elem = typename C::Elem;
#pragma unroll
    for (int j = 0; j < kHold; ++j) {
        typename C::Pair w[C::kP];
        c.fill(gw[j], static_cast<typename C::Acc>(a.scale));
        if (a.w_post) {
            c.fill(w, 1);
            c.read(static_cast<const Elem *>(a.w_post), j, w);
#pragma unroll
            for (int k = 0; k < C::kP; ++k) gw[j][k] = gw[j][k] * w[k];
        }
        if (!kRowGate && a.gate) {
            c.fill(w, 1);
            c.read(static_cast<const Elem *>(a.gate) + group * a.d, j, w);
#pragma unroll
            for (int k = 0; k < C::kP; ++k) gw[j][k] = gw[j][k] * w[k];
        }
    }
}

// Forward.  In one turn of the loop: the sum of f^2 of a row, x' and its sum of the row before, n of the row before that.
// kRowGate: the gate changes from row to row and comes through the ring like a third operand.
template <int DT, int kHold, bool kVector, bool kRowGate>
__global__ void __launch_bounds__(kMaxTeam, 1)
block_norm_fwd_ring_kernel(const NormArgs a, const uint32_t slot_bytes)
{
    in_stream_order();
    using C    = Columns<DT, kHold, kVector>;
    using Elem = typename C::Elem;
    using Acc  = typename C::Acc;
    using Pair = typename C::Pair;
    constexpr int kP = C::kP, kOperands = kRowGate ? 3 : 2;
    using Ring = RowRing<DT, kHold, kVector, kOperands>;
    extern __shared__ uint4 shared[];
    __shared__ Acc part[2][2][kMaxWarps];                              // [turn][of f, of x'][warp]
    const uint32_t t = threadIdx.x, warps = blockDim.x / 32;
    const C        c{t, blockDim.x, static_cast<uint32_t>(a.d)};
    const Ring     ring(c, shared, slot_bytes);
    const Acc      eps = static_cast<Acc>(a.eps), of_d = Acc(1) / static_cast<Acc>(a.d);
    const uint64_t total = a.rows * a.d;
    const Extent   all_x = extent_of(a.x_out, total * sizeof(Elem)), all_n = extent_of(a.n_out, total * sizeof(Elem));

    uint64_t next = blockIdx.x;                                        // the row to copy next
    // (a commit for every turn, also behind the last row: the waits count groups)
    const auto fill = [&](const uint32_t stage) {
        if (next < a.rows) {
            ring.copy(stage, 0, a.x, next, total);
            if (a.f) ring.copy(stage, 1, a.f, next, total);
            if constexpr (kRowGate) ring.copy(stage, 2, a.gate, next / a.gate_rows, round_up_div(a.rows, a.gate_rows) * a.d);
            next += gridDim.x;
        }
        copy_commit();
    };
    bool present[kOperands];
    present[0] = true, present[1] = a.f != nullptr;
    if constexpr (kRowGate) present[2] = true;
    ring.clear(present);
    for (uint32_t s = 0; s + 1 < Ring::stages; ++s) fill(s);

    Pair gw[kHold][kP], w_pre[kHold][kP], y[kHold][kP];
    branch_factors<DT, kHold, kVector, kRowGate>(a, 0, c, gw);
#pragma unroll
    for (int j = 0; j < kHold; ++j) {
        c.fill(w_pre[j], 1);
        if (a.w_pre) c.read(static_cast<const Elem *>(a.w_pre), j, w_pre[j]);
    }
    if constexpr (!kVector) {                                          // the first row, copied by all
        copy_wait<Ring::kBehind + 1>();
        __syncthreads();
    }
    const uint64_t mine = (a.rows - blockIdx.x + gridDim.x - 1) / gridDim.x;      // rows of this CTA (the grid is not wider than the rows)
    const uint64_t stride = static_cast<uint64_t>(gridDim.x) * a.d;
    uint64_t       row = blockIdx.x, at_y = row * a.d, at_n = at_y;    // of the turn; where the rows written next begin
    uint32_t       stage_a = 0, stage_b = 0, stage_c = Ring::stages - 1;
    for (uint64_t turn = 0; turn < mine + 2; ++turn, row += gridDim.x) {
        const Acc(*const before)[kMaxWarps] = part[(turn & 1) ^ 1];
        Acc(*const now)[kMaxWarps]          = part[turn & 1];
        if (turn < mine) {
            if constexpr (kVector) copy_wait<Ring::kBehind>();
            if (a.w_post) {
                Pair s = both(Acc(0));
#pragma unroll
                for (int j = 0; j < kHold; ++j) {
                    Pair f[kP];
                    ring.read(stage_a, 1, j, row, true, f);
#pragma unroll
                    for (int k = 0; k < kP; ++k) s = fma2(f[k], f[k], s);
                }
                const Acc v = warp_sum(s.low() + s.high());
                if (t % 32 == 0) now[0][t / 32] = v;
            }
        }
        if (turn >= 2 && a.n_out) {
            // ---- n of the row two before, whose x' waits in y
            const Pair r = both(root_of(cta_sum(before[1], warps) * of_d + eps));
#pragma unroll
            for (int j = 0; j < kHold; ++j) {
                Pair n[kP];
#pragma unroll
                for (int k = 0; k < kP; ++k) n[k] = y[j][k] * r * w_pre[j][k];
                c.write(static_cast<Elem *>(a.n_out) + at_n, j, n, all_n);
            }
            at_n += stride;
        }
        if (turn >= 1 && turn <= mine) {
            // ---- x' of the row before
            const uint64_t before_row = row - gridDim.x;
            const Pair     rf = both(a.w_post ? root_of(cta_sum(before[0], warps) * of_d + eps) : Acc(1));
            Pair           s  = both(Acc(0));
#pragma unroll
            for (int j = 0; j < kHold; ++j) {
                Pair f[kP];
                ring.read(stage_b, 0, j, before_row, true, y[j]);
                ring.read(stage_b, 1, j, before_row, a.f != nullptr, f);
                if constexpr (kRowGate) {
                    Pair g[kP];
                    ring.read(stage_b, 2, j, before_row / a.gate_rows, true, g);
#pragma unroll
                    for (int k = 0; k < kP; ++k) f[k] = f[k] * g[k];
                }
#pragma unroll
                for (int k = 0; k < kP; ++k) {
                    y[j][k] = fma2(f[k] * rf, gw[j][k], y[j][k]);
                    s       = fma2(y[j][k], y[j][k], s);
                }
                if (a.x_out) c.write(static_cast<Elem *>(a.x_out) + at_y, j, y[j], all_x);
            }
            at_y += stride;
            if (a.n_out) {
                const Acc v = warp_sum(s.low() + s.high());
                if (t % 32 == 0) now[1][t / 32] = v;
            }
            stage_b = stage_b + 1 == Ring::stages ? 0 : stage_b + 1;
        }
        if constexpr (!kVector) copy_wait<Ring::kBehind>();            // the next row's copies, those of all with the barrier
        __syncthreads();                                               // this turn's sums are there; those of the turn before are free
        fill(stage_c);
        stage_c = stage_c + 1 == Ring::stages ? 0 : stage_c + 1;
        stage_a = stage_a + 1 == Ring::stages ? 0 : stage_a + 1;
    }
}

// Backward, over the rows of a chunk.  In one turn of the loop: the six sums of a row, the outputs of the row before.
// kRowGate: the gate changes from row to row and comes through the ring like a fifth operand.
template <int DT, int kHold, bool kVector, bool kRowGate>
__global__ void __launch_bounds__(kMaxTeam, 1)
block_norm_bwd_ring_kernel(const NormArgs a, const uint32_t slot_bytes)
{
    in_stream_order();
    using C    = Columns<DT, kHold, kVector>;
    using Elem = typename C::Elem;
    using Acc  = typename C::Acc;
    using Pair = typename C::Pair;
    constexpr int kP = C::kP, kOperands = kRowGate ? 5 : 4;
    using Ring = RowRing<DT, kHold, kVector, kOperands>;
    extern __shared__ uint4 shared[];
    __shared__ Acc part[2][kMaxWarps][8];
    const uint32_t t = threadIdx.x, chunk = blockIdx.x, warps = blockDim.x / 32;
    const C        c{t, blockDim.x, static_cast<uint32_t>(a.d)};
    const Ring     ring(c, shared, slot_bytes);
    const Acc      scale = static_cast<Acc>(a.scale), eps = static_cast<Acc>(a.eps), of_d = Acc(1) / static_cast<Acc>(a.d);
    const uint64_t total = a.rows * a.d, gates = round_up_div(a.rows, a.gate_rows) * a.d;
    const Extent   all_x = extent_of(a.x_out, total * sizeof(Elem)), all_f = extent_of(a.n_out, total * sizeof(Elem));
    const Extent   all_g = extent_of(a.dgate, gates * sizeof(Elem)), part_g = extent_of(a.part_gate, 2ull * a.chunks * a.d * sizeof(Acc));
    const Extent   part_w = extent_of(a.part_pre, a.chunks * a.d * sizeof(Acc)), part_p = extent_of(a.part_post, a.chunks * a.d * sizeof(Acc));
    const Chunk    rows     = chunk_of(a, chunk);
    const uint64_t of_chunk = a.group_chunks ? chunk / a.group_chunks : 0;       // the group of all its rows, unless kRowGate

    uint64_t next = rows.first;                                        // the row to copy next
    // (a commit for every row of the ring, also behind the chunk's end: the waits count groups)
    const auto fill = [&](const uint32_t stage) {
        if (next < rows.end) {
            ring.copy(stage, 0, a.x, next, total);
            if (a.f) ring.copy(stage, 1, a.f, next, total);
            if (a.dn) ring.copy(stage, 2, a.dn, next, total);
            if (a.dy) ring.copy(stage, 3, a.dy, next, total);
            if constexpr (kRowGate) ring.copy(stage, 4, a.gate, next / a.gate_rows, gates);
            ++next;
        }
        copy_commit();
    };
    bool present[kOperands];
    present[0] = true, present[1] = a.f != nullptr, present[2] = a.dn != nullptr, present[3] = a.dy != nullptr;
    if constexpr (kRowGate) present[4] = true;
    ring.clear(present);
    for (uint32_t s = 0; s + 1 < Ring::stages; ++s) fill(s);

    Pair w_pre[kHold][kP], gw[kHold][kP];
    branch_factors<DT, kHold, kVector, kRowGate>(a, of_chunk, c, gw);
#pragma unroll
    for (int j = 0; j < kHold; ++j) {
        c.fill(w_pre[j], 1);
        if (a.w_pre) c.read(static_cast<const Elem *>(a.w_pre), j, w_pre[j]);
    }
    // a row's operands
    const auto operands = [&](const uint32_t stage, const uint64_t row, const int j, Pair (&x)[kP], Pair (&f)[kP], Pair (&dn)[kP], Pair (&dy)[kP], Pair (&g)[kP]) {
        ring.read(stage, 0, j, row, true, x);
        ring.read(stage, 1, j, row, a.f != nullptr, f);
        ring.read(stage, 2, j, row, a.dn != nullptr, dn);
        ring.read(stage, 3, j, row, a.dy != nullptr, dy);
        if constexpr (kRowGate) ring.read(stage, 4, j, row / a.gate_rows, true, g);
    };

    // sum_pre: of dn x' r.  sum_f: of t f rf, of the rows that share a gate; times scale w_post it is the gate's gradient, times
    // scale gate its share of w_post's (sum_post).
    Pair sum_pre[kHold][kP], sum_f[kHold][kP], sum_post[kRowGate ? kHold : 1][kP];
#pragma unroll
    for (int j = 0; j < kHold; ++j) c.fill(sum_pre[j], 0), c.fill(sum_f[j], 0), c.fill(sum_post[kRowGate ? j : 0], 0);
    if constexpr (!kVector) {                                          // the first row, copied by all
        copy_wait<Ring::kBehind + 1>();
        __syncthreads();
    }
    uint32_t stage_a = 0, stage_b = 0, stage_c = Ring::stages - 1;     // of the row whose sums are taken, of the one before, to fill
    uint64_t at_out = rows.first * a.d;
    for (uint64_t row = rows.first; row <= rows.end; ++row) {
        if (row < rows.end) {
            // ---- this row's sums
            if constexpr (kVector) copy_wait<Ring::kBehind>();
            Pair p[6];
#pragma unroll
            for (int k = 0; k < 6; ++k) p[k] = both(Acc(0));
#pragma unroll
            for (int j = 0; j < kHold; ++j) {
                Pair x[kP], f[kP], dn[kP], dy[kP], g[kP];
                operands(stage_a, row, j, x, f, dn, dy, g);
#pragma unroll
                for (int k = 0; k < kP; ++k) {
                    const Pair wn = dn[k] * w_pre[j][k];
                    Pair       q  = gw[j][k] * f[k];
                    if constexpr (kRowGate) q = q * g[k];
                    p[0] = fma2(x[k], x[k], p[0]);
                    p[1] = fma2(wn, x[k], p[1]);
                    p[2] = fma2(f[k], f[k], p[2]);
                    p[3] = fma2(dy[k], q, p[3]);
                    p[4] = fma2(wn, q, p[4]);
                    p[5] = fma2(x[k], q, p[5]);
                }
            }
            Acc s[8] = {};
#pragma unroll
            for (int k = 0; k < 6; ++k) s[k] = p[k].low() + p[k].high();
            const Acc v = warp_sums8(s);
            if (t % 4 == 0) part[row & 1][t / 32][t % 32 / 4] = v;
        }
        if (row > rows.first) {
            // ---- the row before: its outputs
            const uint64_t before = row - 1;
            Acc            s[6];
            cta_sums(part[before & 1], warps, s);
            const RowFactors<Acc> q = factors_of(s, of_d, eps, a.w_post != nullptr);
            const Pair r = both(q.r), rrc = both(-q.rrc), rf = both(q.rf), rf3m = both(-q.rf3m);
#pragma unroll
            for (int j = 0; j < kHold; ++j) {
                Pair x[kP], f[kP], dn[kP], dy[kP], g[kP];
                operands(stage_b, before, j, x, f, dn, dy, g);
#pragma unroll
                for (int k = 0; k < kP; ++k) {
                    const Pair tv = fma2(rrc, x[k], fma2(r, dn[k] * w_pre[j][k], dy[k]));
                    sum_pre[j][k] = fma2(dn[k], x[k] * r, sum_pre[j][k]);
                    sum_f[j][k]   = fma2(tv, f[k] * rf, sum_f[j][k]);
                    Pair tg       = tv * gw[j][k];
                    if constexpr (kRowGate) tg = tg * g[k];
                    f[k]  = fma2(tg, rf, rf3m * f[k]);
                    dy[k] = tv;
                }
                if (a.x_out) c.write(static_cast<Elem *>(a.x_out) + at_out, j, dy, all_x);
                if (a.n_out) c.write(static_cast<Elem *>(a.n_out) + at_out, j, f, all_f);
            }
            at_out += a.d;
            // the last of the group's rows in this chunk: its gate's gradient, or this chunk's share of it
            if (a.gate && (row == rows.end || (kRowGate && row % a.gate_rows == 0))) {
                const uint64_t group = before / a.gate_rows;
                uint64_t       to;
                const bool     whole = whole_group(a, rows, group, chunk, to);
#pragma unroll
                for (int j = 0; j < kHold; ++j) {
                    Pair w[kP], g[kP];
                    c.fill(w, 1);
                    if (a.w_post) c.read(static_cast<const Elem *>(a.w_post), j, w);
                    if constexpr (kRowGate) ring.read(stage_b, 4, j, group, true, g);
#pragma unroll
                    for (int k = 0; k < kP; ++k) {
                        w[k] = w[k] * both(scale) * sum_f[j][k];
                        if constexpr (kRowGate) sum_post[j][k] = fma2(both(scale) * g[k], sum_f[j][k], sum_post[j][k]), sum_f[j][k] = both(Acc(0));
                    }
                    if (a.dgate && whole) c.write(static_cast<Elem *>(a.dgate) + group * a.d, j, w, all_g);
                    if (a.dgate && !whole) c.write_sums(reinterpret_cast<Acc *>(a.part_gate) + to * a.d, j, w, part_g);
                }
            }
            stage_b = stage_b + 1 == Ring::stages ? 0 : stage_b + 1;
        }
        if constexpr (!kVector) copy_wait<Ring::kBehind>();            // the next row's copies, those of all with the barrier
        __syncthreads();                                               // the sums of this row are there; the words of the one before are free
        fill(stage_c);
        stage_c = stage_c + 1 == Ring::stages ? 0 : stage_c + 1;
        stage_a = stage_a + 1 == Ring::stages ? 0 : stage_a + 1;
    }
#pragma unroll
    for (int j = 0; j < kHold; ++j) {
        if (!kRowGate && a.dw_post) {
            Pair g[kP];
            c.fill(g, 1);
            if (a.gate) c.read(static_cast<const Elem *>(a.gate) + of_chunk * a.d, j, g);
#pragma unroll
            for (int k = 0; k < kP; ++k) sum_f[j][k] = sum_f[j][k] * both(scale) * g[k];
        }
        if (a.dw_pre) c.write_sums(reinterpret_cast<Acc *>(a.part_pre) + chunk * a.d, j, sum_pre[j], part_w);
        if (a.dw_post) c.write_sums(reinterpret_cast<Acc *>(a.part_post) + chunk * a.d, j, kRowGate ? sum_post[kRowGate ? j : 0] : sum_f[j], part_p);
    }
}

// kHold accesses of every operand per thread, held in registers with the column sums.
template <int DT, bool kVector, int kHold, bool kCta>
__global__ void __launch_bounds__(kCta ? kMaxTeam : 32 * kWarpTeams)
block_norm_bwd_kernel(const NormArgs a)
{
    in_stream_order();
    using X                = Access<DT, kVector>;
    using Elem             = typename X::Elem;
    using Acc              = typename X::Acc;
    constexpr int  kW      = X::kW;
    __shared__ Acc words[2][6][kMaxWarps];
    uint32_t       turn    = 0;
    const uint32_t team    = kCta ? blockDim.x : 32;
    const uint32_t t       = kCta ? threadIdx.x : threadIdx.x % 32;
    const uint32_t chunk   = kCta ? blockIdx.x : blockIdx.x * (blockDim.x / 32) + threadIdx.x / 32;
    const uint32_t count   = static_cast<uint32_t>(a.d / kW);
    const Acc      scale = static_cast<Acc>(a.scale), eps = static_cast<Acc>(a.eps), of_d = Acc(1) / static_cast<Acc>(a.d);
    const uint64_t bytes = a.rows * a.d * sizeof(Elem);
    const Extent   all_x = extent_of(a.x_out, bytes), all_f = extent_of(a.n_out, bytes);
    const Extent   all_g = extent_of(a.dgate, round_up_div(a.rows, a.gate_rows) * a.d * sizeof(Elem));
    const Extent   part_g = extent_of(a.part_gate, 2ull * a.chunks * a.d * sizeof(Acc));
    const Extent   part_w = extent_of(a.part_pre, a.chunks * a.d * sizeof(Acc)), part_p = extent_of(a.part_post, a.chunks * a.d * sizeof(Acc));
    if (chunk >= a.chunks) return;                                     // (a whole team; a CTA team is a CTA)
    const Chunk c = chunk_of(a, chunk);
    Acc         sum_pre[kHold][kW] = {}, sum_post[kHold][kW] = {}, sum_gate[kHold][kW] = {};
    for (uint64_t row = c.first; row < c.end; ++row) {
        const void *x = row_of<Elem>(a.x, row, a.d), *f = row_of<Elem>(a.f, row, a.d);
        const void *dn = row_of<Elem>(a.dn, row, a.d), *dy = row_of<Elem>(a.dy, row, a.d);
        const uint64_t group = row / a.gate_rows;
        const void    *gate  = a.gate ? row_of<Elem>(a.gate, group, a.d) : nullptr;
        // the operands wait in registers as they lie in memory; weights and gate are read again from the L1
        typename X::Raw xr[kHold], fr[kHold], nr[kHold], yr[kHold];
        Acc             s[6] = {};
#pragma unroll
        for (int j = 0; j < kHold; ++j) {
            const uint32_t i = j * team + t;
            if (i >= count) continue;
            xr[j] = X::load(x, i);
            if (f) fr[j] = X::load(f, i);
            if (dn) nr[j] = X::load(dn, i);
            if (dy) yr[j] = X::load(dy, i);
        }
        // element values of access j: x', f, dx', dn, w_pre, scale * gate, w_post
        const auto element = [&](const int j, Acc (&xv)[kW], Acc (&fv)[kW], Acc (&dyv)[kW], Acc (&dnv)[kW], Acc (&wpre)[kW], Acc (&gw)[kW], Acc (&pw)[kW]) {
            const uint32_t i = j * team + t;
#pragma unroll
            for (int k = 0; k < kW; ++k) fv[k] = dnv[k] = dyv[k] = 0, wpre[k] = pw[k] = gw[k] = 1;
            X::widen(xr[j], xv);
            if (f) X::widen(fr[j], fv);
            if (dn) X::widen(nr[j], dnv), X::read_shared(a.w_pre, i, wpre);
            if (dy) X::widen(yr[j], dyv);
            if (a.w_post) X::read_shared(a.w_post, i, pw);
            if (gate) X::read_shared(gate, i, gw);
#pragma unroll
            for (int k = 0; k < kW; ++k) gw[k] *= scale;
        };
#pragma unroll
        for (int j = 0; j < kHold; ++j) {
            if (j * team + t >= count) continue;
            Acc xv[kW], fv[kW], dyv[kW], dnv[kW], wpre[kW], gw[kW], pw[kW];
            element(j, xv, fv, dyv, dnv, wpre, gw, pw);
#pragma unroll
            for (int k = 0; k < kW; ++k) add_sums(s, xv[k], fv[k], dyv[k], dnv[k] * wpre[k], gw[k] * pw[k]);
        }
        team_sums<kCta>(s, words, turn);
        const RowFactors<Acc> q = factors_of(s, of_d, eps, a.w_post != nullptr);
        void *dx = row_of<Elem>(a.x_out, row, a.d), *df = row_of<Elem>(a.n_out, row, a.d);
#pragma unroll
        for (int j = 0; j < kHold; ++j) {
            const uint32_t i = j * team + t;
            if (i >= count) continue;
            Acc xv[kW], fv[kW], dyv[kW], dnv[kW], wpre[kW], gw[kW], pw[kW];
            element(j, xv, fv, dyv, dnv, wpre, gw, pw);
#pragma unroll
            for (int k = 0; k < kW; ++k) {
                const Acc tv = dyv[k] + q.r * (dnv[k] * wpre[k]) - q.rrc * xv[k];
                sum_pre[j][k] += dnv[k] * (xv[k] * q.r);
                const Acc fh = fv[k] * q.rf, dp = tv * gw[k];
                sum_gate[j][k] += scale * tv * (fh * pw[k]);
                sum_post[j][k] += dp * fh;
                fv[k]  = dp * pw[k] * q.rf - q.rf3m * fv[k];
                dyv[k] = tv;
            }
            if (dx) X::store(dx, i, dyv, all_x);
            if (df) X::store(df, i, fv, all_f);
        }
        // the last of the group's rows in this chunk: its gate's gradient, or this chunk's share of it
        if (a.dgate && (row + 1 == c.end || (row + 1) % a.gate_rows == 0)) {
            uint64_t   slot;
            const bool whole = whole_group(a, c, group, chunk, slot);
#pragma unroll
            for (int j = 0; j < kHold; ++j) {
                const uint32_t i = j * team + t;
                if (i < count) {
                    if (whole) X::store(row_of<Elem>(a.dgate, group, a.d), i, sum_gate[j], all_g);
                    else
#pragma unroll
                        for (int k = 0; k < kW; ++k) {
                            Acc *const o = reinterpret_cast<Acc *>(a.part_gate) + slot * a.d + i * kW + k;
                            if (part_g.holds(o, sizeof(Acc))) *o = sum_gate[j][k];
                        }
                }
#pragma unroll
                for (int k = 0; k < kW; ++k) sum_gate[j][k] = 0;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < kHold; ++j) {
        const uint32_t i = j * team + t;
        if (i >= count) continue;
#pragma unroll
        for (int k = 0; k < kW; ++k) {
            const uint64_t o = chunk * a.d + i * kW + k;
            if (a.dw_pre && part_w.holds(reinterpret_cast<Acc *>(a.part_pre) + o, sizeof(Acc))) reinterpret_cast<Acc *>(a.part_pre)[o] = sum_pre[j][k];
            if (a.dw_post && part_p.holds(reinterpret_cast<Acc *>(a.part_post) + o, sizeof(Acc))) reinterpret_cast<Acc *>(a.part_post)[o] = sum_post[j][k];
        }
    }
}

// Rows longer than a CTA's registers: dx and df by a kernel that reads a row twice and leaves its factors behind ...
template <int DT>
__global__ void __launch_bounds__(kMaxTeam)
block_norm_bwd_rows_kernel(const NormArgs a)
{
    in_stream_order();
    using X    = Access<DT, false>;
    using Elem = typename X::Elem;
    using Acc  = typename X::Acc;
    __shared__ Acc words[2][6][kMaxWarps];
    uint32_t       turn = 0;
    const Acc      scale = static_cast<Acc>(a.scale), eps = static_cast<Acc>(a.eps), of_d = Acc(1) / static_cast<Acc>(a.d);
    const uint64_t bytes = a.rows * a.d * sizeof(Elem);
    const Extent   all_x = extent_of(a.x_out, bytes), all_f = extent_of(a.n_out, bytes), all_s = extent_of(a.stats, a.rows * sizeof(RowFactors<Acc>));
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Elem *x = static_cast<const Elem *>(a.x) + row * a.d, *gate = static_cast<const Elem *>(row_of<Elem>(a.gate, row / a.gate_rows, a.d));
        const Elem *f = static_cast<const Elem *>(row_of<Elem>(a.f, row, a.d)), *dn = static_cast<const Elem *>(row_of<Elem>(a.dn, row, a.d));
        const Elem *dy = static_cast<const Elem *>(row_of<Elem>(a.dy, row, a.d));
        const Elem *w_pre = static_cast<const Elem *>(a.w_pre), *w_post = static_cast<const Elem *>(a.w_post);
        const auto  at = [](const Elem *p, const uint64_t i, const Acc none) { return p ? static_cast<Acc>(Num<DT>::widen(p[i])) : none; };
        Acc         s[6] = {};
        for (uint64_t i = threadIdx.x; i < a.d; i += blockDim.x)
            add_sums(s, at(x, i, 0), at(f, i, 0), at(dy, i, 0), dn ? at(dn, i, 0) * at(w_pre, i, 1) : Acc(0), scale * at(gate, i, 1) * at(w_post, i, 1));
        team_sums<true>(s, words, turn);
        const RowFactors<Acc> q = factors_of(s, of_d, eps, w_post != nullptr);
        if (threadIdx.x == 0 && all_s.holds(static_cast<RowFactors<Acc> *>(a.stats) + row, sizeof(q))) static_cast<RowFactors<Acc> *>(a.stats)[row] = q;
        void *dx = row_of<Elem>(a.x_out, row, a.d), *df = row_of<Elem>(a.n_out, row, a.d);
        for (uint64_t i = threadIdx.x; i < a.d; i += blockDim.x) {
            const Acc xv = at(x, i, 0), wn = dn ? at(dn, i, 0) * at(w_pre, i, 1) : Acc(0), gw = scale * at(gate, i, 1) * at(w_post, i, 1);
            Acc       t[1] = {at(dy, i, 0) + q.r * wn - q.rrc * xv};
            Acc       o[1] = {t[0] * gw * q.rf - q.rf3m * at(f, i, 0)};
            if (dx) X::store(dx, static_cast<uint32_t>(i), t, all_x);
            if (df) X::store(df, static_cast<uint32_t>(i), o, all_f);
        }
    }
}
// ... and the column sums by one that gives every thread a column of a chunk.
template <int DT>
__global__ void block_norm_bwd_columns_kernel(const NormArgs a)
{
    in_stream_order();
    using Elem = typename Num<DT>::Elem;
    using Acc  = typename Num<DT>::Acc;
    const uint64_t i     = static_cast<uint64_t>(blockIdx.x % static_cast<uint32_t>(round_up_div(a.d, blockDim.x))) * blockDim.x + threadIdx.x;
    const uint32_t chunk = blockIdx.x / static_cast<uint32_t>(round_up_div(a.d, blockDim.x));
    if (i >= a.d || chunk >= a.chunks) return;
    const Acc    scale  = static_cast<Acc>(a.scale);
    const Extent all_g  = extent_of(a.dgate, round_up_div(a.rows, a.gate_rows) * a.d * sizeof(Elem));
    const Extent part_g = extent_of(a.part_gate, 2ull * a.chunks * a.d * sizeof(Acc));
    const Extent part_w = extent_of(a.part_pre, a.chunks * a.d * sizeof(Acc)), part_p = extent_of(a.part_post, a.chunks * a.d * sizeof(Acc));
    const auto   at = [i](const void *p, const uint64_t row, const uint64_t d, const Acc none) {
        return p ? static_cast<Acc>(Num<DT>::widen(static_cast<const Elem *>(p)[row * d + i])) : none;
    };
    const Acc   w_pre = at(a.w_pre, 0, a.d, 1), w_post = at(a.w_post, 0, a.d, 1);
    const Chunk c = chunk_of(a, chunk);
    Acc         sum_pre = 0, sum_post = 0, sum_gate = 0;
    for (uint64_t row = c.first; row < c.end; ++row) {
        const RowFactors<Acc> q     = static_cast<const RowFactors<Acc> *>(a.stats)[row];
        const uint64_t        group = row / a.gate_rows;
        const Acc x = at(a.x, row, a.d, 0), dn = at(a.dn, row, a.d, 0), fh = at(a.f, row, a.d, 0) * q.rf;
        const Acc t = at(a.dy, row, a.d, 0) + q.r * (a.dn ? dn * w_pre : Acc(0)) - q.rrc * x;
        sum_pre += dn * (x * q.r);
        sum_gate += scale * t * (fh * w_post);
        sum_post += scale * t * at(a.gate, group, a.d, 1) * fh;
        if (a.dgate && (row + 1 == c.end || (row + 1) % a.gate_rows == 0)) {
            uint64_t   slot;
            const bool whole = whole_group(a, c, group, chunk, slot);
            if (whole) {
                Elem *const o = static_cast<Elem *>(a.dgate) + group * a.d + i;
                if (all_g.holds(o, sizeof(Elem))) *o = Num<DT>::narrow(sum_gate);
            } else {
                Acc *const o = reinterpret_cast<Acc *>(a.part_gate) + slot * a.d + i;
                if (part_g.holds(o, sizeof(Acc))) *o = sum_gate;
            }
            sum_gate = 0;
        }
    }
    const uint64_t o = chunk * a.d + i;
    if (a.dw_pre && part_w.holds(reinterpret_cast<Acc *>(a.part_pre) + o, sizeof(Acc))) reinterpret_cast<Acc *>(a.part_pre)[o] = sum_pre;
    if (a.dw_post && part_p.holds(reinterpret_cast<Acc *>(a.part_post) + o, sizeof(Acc))) reinterpret_cast<Acc *>(a.part_post)[o] = sum_post;
}

// The partial rows added up: 0 w_pre, 1 w_post, 2 + k the k-th group of rows with a gate or, where there are more groups
// than borders between chunks, the group that lies across the k-th border.  A thread takes every kSplit-th partial row of its
// column; the CTA adds the kSplit sums in order.
constexpr int kFinishColumns = 32, kSplit = 16;
template <int DT>
__global__ void __launch_bounds__(kFinishColumns *kSplit)
block_norm_finish_kernel(const NormArgs a)
{
    in_stream_order();
    using Elem = typename Num<DT>::Elem;
    using Acc  = typename Num<DT>::Acc;
    __shared__ Acc part[kSplit][kFinishColumns];
    const uint32_t columns = static_cast<uint32_t>(round_up_div(a.d, kFinishColumns));
    const uint32_t what    = blockIdx.x / columns;
    const uint32_t lane = threadIdx.x % kFinishColumns, share = threadIdx.x / kFinishColumns;
    const uint64_t i    = static_cast<uint64_t>(blockIdx.x % columns) * kFinishColumns + lane;
    const Acc     *from;
    Elem          *to;
    uint64_t       count;
    bool           across = false;                                     // from one chunk to the next, slots of a gate group
    if (what < 2) {
        from  = reinterpret_cast<const Acc *>(what == 0 ? a.part_pre : a.part_post);
        to    = static_cast<Elem *>(what == 0 ? a.dw_pre : a.dw_post);
        count = a.chunks;
        if (!to) return;
    } else {
        if (!a.dgate) return;
        uint64_t group = what - 2;
        if (round_up_div(a.rows, a.gate_rows) >= a.chunks && !a.group_chunks) {                  // by borders
            const uint64_t border = (what - 1) * a.chunk_rows;          // the next chunk's first row
            if (border >= a.rows || border % a.gate_rows == 0) return;
            group = border / a.gate_rows;
            if (group * a.gate_rows / a.chunk_rows != what - 2) return;  // (a group across several borders: at its first)
        }
        const uint64_t begin = group * a.gate_rows, end = begin + a.gate_rows < a.rows ? begin + a.gate_rows : a.rows;
        const uint64_t from_chunk = chunk_at(a, begin), to_chunk = chunk_at(a, end - 1);
        if (from_chunk == to_chunk) return;                             // written whole
        // slot 2 * chunk + 1 of the first chunk, then slot 2 * chunk of the others, one after the other every second row
        from   = reinterpret_cast<const Acc *>(a.part_gate) + (2 * from_chunk + 1) * a.d;
        to     = static_cast<Elem *>(a.dgate) + group * a.d;
        count  = to_chunk - from_chunk + 1;
        across = true;
    }
    Acc s = 0;
    if (i < a.d && share < count) {
        const Acc     *at   = from + i + (across ? (share == 0 ? 0 : 2 * share - 1) : share) * a.d;
        const uint64_t step = (across ? 2 : 1) * kSplit * a.d;
        s = *at;
        at += step - (across && share == 0 ? a.d : 0);                  // (slot 2 * chunk + 1 of the first chunk is one row nearer)
#pragma unroll 8
        for (uint64_t k = share + kSplit; k < count; k += kSplit, at += step) s += *at;
    }
    part[share][lane] = s;
    __syncthreads();
    if (share != 0 || i >= a.d) return;
#pragma unroll
    for (int k = 1; k < kSplit; ++k) s += part[k][lane];
    if (extent_of(to, a.d * sizeof(Elem)).holds(to + i, sizeof(Elem))) to[i] = Num<DT>::narrow(s);
}

// ---------------------------------------------------------------------------------------------- host side
constexpr uint32_t kMaxChunks  = 4096;      // chunks of rows of a backward pass
constexpr uint32_t kLongChunks = 64;        // the same for rows longer than a CTA's registers

// threads of a CTA that holds `count` accesses, `hold` per thread
uint32_t team_of(uint64_t count, uint32_t hold) { return static_cast<uint32_t>(round_up_div(round_up_div(count, hold), 32) * 32); }
// Vectors per thread of the ring kernels: two from 64 on, which halves what the sums over a row cost per element; CTAs of an SM:
// 512 threads' worth.  Rows of single elements: eight columns per thread, sixteen where that takes more than a CTA.
uint32_t hold_of(uint64_t count) { return count < 64 ? 1 : 2; }
constexpr size_t kMostShared = 220 * 1024;

// How a ring kernel takes rows of d elements: hold 0 if it cannot.
struct RingPlan {
    uint32_t hold, team, slot;     // slot: bytes of an operand's row, rows of single elements
    size_t   smem;
};
RingPlan ring_plan(uint64_t d, int es, uint32_t operands)
{
    const uint64_t lanes = 16 / static_cast<uint64_t>(es);
    RingPlan       p{};
    if (d % lanes == 0) {
        const uint64_t count = d / lanes;
        if (count > 2 * kMaxTeam) return p;
        p.hold = hold_of(count), p.team = team_of(count, p.hold);
        p.smem = static_cast<size_t>(p.hold == 1 ? kRingStages<1, true> : kRingStages<2, true>) * operands * p.hold * p.team * 16;
    } else {
        if (d > 16 * kMaxTeam) return p;
        p.hold = d <= 8 * kMaxTeam ? 1 : 2, p.team = team_of(d, 8 * p.hold);
        p.slot = static_cast<uint32_t>((d * static_cast<uint64_t>(es) + 15) / 16 * 16 + 16);
        p.smem = static_cast<size_t>(kRingStages<1, false>) * operands * p.slot;
    }
    if (p.smem > kMostShared) p.hold = 0;
    return p;
}

// Can a CTA's registers hold a row of the backward pass?
bool row_fits(uint64_t d, int es)
{
    const uint64_t lanes = 16 / static_cast<uint64_t>(es);
    return d % lanes == 0 ? d <= 2 * lanes * kMaxTeam : d <= 8 * kMaxTeam || ring_plan(d, es, 5).hold != 0;
}

template <typename K>
cudaError_t start_ring(K kernel, const NormArgs &a, unsigned grid, const RingPlan &p, cudaStream_t stream)
{
    const cudaError_t e = reported(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(p.smem)));
    return e != cudaSuccess ? e : launch(kernel, grid, p.team, p.smem, stream, a, p.slot);
}

// go(hold, whether rows are whole vectors)
template <typename F>
cudaError_t with_ring(const RingPlan &p, bool vector, const F &go)
{
    using std::bool_constant;
    using std::integral_constant;
    if (p.hold == 1) return vector ? go(integral_constant<int, 1>(), bool_constant<true>()) : go(integral_constant<int, 1>(), bool_constant<false>());
    return vector ? go(integral_constant<int, 2>(), bool_constant<true>()) : go(integral_constant<int, 2>(), bool_constant<false>());
}

template <int DT, bool kVector, int kHold, bool kCta>
cudaError_t start_fwd(const NormArgs &a, uint32_t threads, int sms, cudaStream_t stream)
{
    const uint64_t teams = kCta ? 1 : kWarpTeams, want = round_up_div(a.rows, teams);
    const uint64_t most  = static_cast<uint64_t>(sms) * (2048 / threads);
    return launch(block_norm_fwd_kernel<DT, kVector, kHold, kCta>, static_cast<unsigned>(want < most ? want : most), threads, 0, stream, a);
}

template <int DT>
cudaError_t forward(const NormArgs &a, cudaStream_t stream)
{
    const int sms = sm_count();
    if (sms == 0) return cudaErrorInvalidDevice;
    const uint64_t count    = a.d / kLanes<DT>;
    const bool     vector   = a.d % kLanes<DT> == 0, row_gate = a.gate && a.gate_rows < a.rows;
    const RingPlan p        = ring_plan(a.d, static_cast<int>(sizeof(typename Num<DT>::Elem)), row_gate ? 3 : 2);
    if (p.hold != 0) {
        // 512 threads an SM (three CTAs of 256 where the registers allow them: bf16 16384 x 4096 97 us against 86)
        const uint32_t resident = kMaxTeam / p.team;
        const uint64_t most     = static_cast<uint64_t>(sms) * (resident < 1 ? 1 : resident);
        const unsigned grid     = static_cast<unsigned>(a.rows < most ? a.rows : most);
        const auto     go   = [&](auto hold, auto vec) {
            return row_gate ? start_ring(block_norm_fwd_ring_kernel<DT, decltype(hold)::value, decltype(vec)::value, true>, a, grid, p, stream)
                            : start_ring(block_norm_fwd_ring_kernel<DT, decltype(hold)::value, decltype(vec)::value, false>, a, grid, p, stream);
        };
        return with_ring(p, vector, go);
    }
    if (vector) {
        if (count <= 4 * kMaxTeam) return start_fwd<DT, true, 4, true>(a, team_of(count, 4), sms, stream);
        return start_fwd<DT, true, 0, true>(a, kMaxTeam, sms, stream);
    }
    // (single elements whose ring does not fit shared memory)
    if (a.d <= 4 * kMaxTeam) return start_fwd<DT, false, 4, true>(a, team_of(a.d, 4), sms, stream);
    return start_fwd<DT, false, 0, true>(a, kMaxTeam, sms, stream);
}

template <int DT, bool kVector, int kHold, bool kCta>
cudaError_t start_bwd(const NormArgs &a, uint32_t threads, cudaStream_t stream)
{
    const uint32_t teams = kCta ? 1 : kWarpTeams;
    return launch(block_norm_bwd_kernel<DT, kVector, kHold, kCta>, static_cast<unsigned>(round_up_div(a.chunks, teams)), threads, 0, stream, a);
}

// rows that a CTA's registers hold (row_fits)
template <int DT>
cudaError_t bwd_of(const NormArgs &a, cudaStream_t stream)
{
    const bool     vector = a.d % kLanes<DT> == 0, row_gate = a.gate && !a.group_chunks;
    const RingPlan p      = ring_plan(a.d, static_cast<int>(sizeof(typename Num<DT>::Elem)), row_gate ? 5 : 4);
    if (p.hold != 0) {
        const auto go = [&](auto hold, auto vec) {
            return row_gate ? start_ring(block_norm_bwd_ring_kernel<DT, decltype(hold)::value, decltype(vec)::value, true>, a, a.chunks, p, stream)
                            : start_ring(block_norm_bwd_ring_kernel<DT, decltype(hold)::value, decltype(vec)::value, false>, a, a.chunks, p, stream);
        };
        return with_ring(p, vector, go);
    }
    // (the operands of such rows do not fit shared memory several times)
    return vector ? start_bwd<DT, true, 2, true>(a, team_of(a.d / kLanes<DT>, 2), stream) : start_bwd<DT, false, 8, true>(a, team_of(a.d, 8), stream);
}

// The most chunks of a backward pass: as many teams as the SMs hold at a time.
uint32_t chunks_of(uint64_t rows, uint64_t d, int es, int sms)
{
    const uint64_t lanes = 16 / static_cast<uint64_t>(es), count = d / lanes;
    uint64_t       most;
    if (!row_fits(d, es)) most = kLongChunks;
    else most = static_cast<uint64_t>(sms) * (kMaxTeam / (d % lanes == 0 ? team_of(count, hold_of(count)) : team_of(d, d <= 8 * kMaxTeam ? 8 : 16)));
    if (most > kMaxChunks) most = kMaxChunks;
    if (most > rows / 4) most = rows / 4 > static_cast<uint64_t>(sms) ? rows / 4 : static_cast<uint64_t>(sms);   // partial rows cost, too
    return static_cast<uint32_t>(most < rows ? most : rows);
}
// how the rows are dealt: inside the groups of rows with a gate while every group can have a chunk
void set_chunks(NormArgs &a, uint32_t most)
{
    const uint64_t groups = a.gate ? round_up_div(a.rows, a.gate_rows) : 1, group_rows = a.gate && a.gate_rows < a.rows ? a.gate_rows : a.rows;
    if (groups <= most) {
        const uint64_t each = most / groups < group_rows ? most / groups : group_rows;
        a.chunk_rows        = round_up_div(group_rows, each);
        a.group_chunks      = static_cast<uint32_t>(round_up_div(group_rows, a.chunk_rows));
        a.chunks            = static_cast<uint32_t>(groups) * a.group_chunks;
        a.gate_rows         = group_rows;
    } else {
        a.chunk_rows   = round_up_div(a.rows, most);
        a.group_chunks = 0;
        a.chunks       = static_cast<uint32_t>(round_up_div(a.rows, a.chunk_rows));
    }
}

template <int DT>
cudaError_t backward(const NormArgs &a, cudaStream_t stream)
{
    constexpr int es = static_cast<int>(sizeof(typename Num<DT>::Elem));
    cudaError_t   e;
    if (!row_fits(a.d, es)) {
        const int sms = sm_count();
        if (sms == 0) return cudaErrorInvalidDevice;
        const uint64_t most = static_cast<uint64_t>(sms) * 4;
        e = launch(block_norm_bwd_rows_kernel<DT>, static_cast<unsigned>(a.rows < most ? a.rows : most), kMaxTeam, 0, stream, a);
        if (e != cudaSuccess) return e;
        if (!a.dgate && !a.dw_pre && !a.dw_post) return cudaSuccess;
        e = launch(block_norm_bwd_columns_kernel<DT>, static_cast<unsigned>(round_up_div(a.d, 128) * a.chunks), 128, 0, stream, a);
    } else {
        e = bwd_of<DT>(a, stream);
    }
    if (e != cudaSuccess || (!a.dgate && !a.dw_pre && !a.dw_post)) return e;
    const uint64_t groups = round_up_div(a.rows, a.gate_rows), borders = a.chunks - 1;
    const uint64_t shared = a.dgate ? (a.group_chunks || groups < borders ? groups : borders) : 0;
    return launch(block_norm_finish_kernel<DT>, static_cast<unsigned>(round_up_div(a.d, kFinishColumns) * (2 + shared)), kFinishColumns * kSplit, 0,
                  stream, a);
}

size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

struct Parts {
    uint32_t chunks;                             // at most
    size_t   pre, post, gate, stats, bytes;      // offsets
};
// the workspace of a backward pass; sms: 0 for the most that any GPU could ask for
Parts parts_of(uint64_t rows, uint64_t d, int es, int sms)
{
    const size_t acc = es == 8 ? 8 : 4;
    Parts        p{};
    p.chunks     = chunks_of(rows, d, es, sms);
    const size_t row = d * acc;
    p.pre   = 0;
    p.post  = round_up(p.chunks * row);
    p.gate  = p.post + round_up(p.chunks * row);
    p.stats = p.gate + round_up(2ull * p.chunks * row);
    p.bytes = p.stats + (row_fits(d, es) ? 0 : round_up(rows * 4 * acc));
    return p;
}

int check_common(const void *x, const void *f, const void *gate, const void *w_post, const void *w_pre, uint64_t rows, uint64_t d, uint64_t gate_rows,
                 int dtype, float scale, float eps)
{
    if (element_size(dtype) == 0) return BT_ERR_DTYPE;
    if (d == 0 || gate_rows == 0) return BT_ERR_SHAPE;
    if (!(eps >= 0.0f) || scale != scale) return BT_ERR_SHAPE;
    if (d > (1ull << 24) || rows > (1ull << 40) / d) return BT_ERR_TOO_LARGE;
    if (rows == 0) return BT_OK;
    if (!x || (!f && (gate || w_post))) return BT_ERR_NULL;
    for (const void *p : {x, f, gate, w_post, w_pre})
        if (!on_boundary(p, 16)) return BT_ERR_ALIGN;
    return BT_OK;
}

template <typename F>
int dispatch(int dtype, const F &go)
{
    cudaError_t e;
    switch (dtype) {
    case BT_F32: e = go(std::integral_constant<int, BT_F32>()); break;
    case BT_F16: e = go(std::integral_constant<int, BT_F16>()); break;
    case BT_BF16: e = go(std::integral_constant<int, BT_BF16>()); break;
    default: e = go(std::integral_constant<int, BT_F64>()); break;
    }
    return e == cudaSuccess ? BT_OK : BT_ERR_CUDA;
}

}  // namespace
}  // namespace bt

extern "C" {

size_t bt_block_norm_workspace_bytes(uint64_t rows, uint64_t d, int dtype)
{
    const int es = bt::element_size(dtype);
    if (es == 0 || rows == 0 || d == 0) return 0;
    if (d > (1ull << 24) || rows > (1ull << 40) / d) return 0;
    const int sms = bt::sm_count();
    return bt::parts_of(rows, d, es, sms ? sms : 148).bytes;
}

int bt_block_norm_fwd(const void *x, uint64_t rows, uint64_t d, uint64_t gate_rows, int dtype, float scale, float eps, const void *f,
                      const void *gate, const void *w_post, const void *w_pre, void *x_out, void *n_out, void *stream)
{
    const int st = bt::check_common(x, f, gate, w_post, w_pre, rows, d, gate_rows, dtype, scale, eps);
    if (st != BT_OK || rows == 0) return st;
    if ((f != nullptr) != (x_out != nullptr) || (n_out != nullptr) != (w_pre != nullptr) || (!x_out && !n_out)) return BT_ERR_NULL;
    if (!bt::on_boundary(x_out, 16) || !bt::on_boundary(n_out, 16)) return BT_ERR_ALIGN;
    bt::NormArgs a{};
    a.x = x, a.f = f, a.gate = gate, a.w_post = w_post, a.w_pre = w_pre;
    a.x_out = x_out, a.n_out = n_out;
    a.rows = rows, a.d = d, a.gate_rows = gate_rows;
    a.scale = scale, a.eps = eps;
    return bt::dispatch(dtype, [&](auto dt) { return bt::forward<decltype(dt)::value>(a, static_cast<cudaStream_t>(stream)); });
}

int bt_block_norm_bwd(const void *x_out, uint64_t rows, uint64_t d, uint64_t gate_rows, int dtype, float scale, float eps, const void *f,
                      const void *gate, const void *w_post, const void *w_pre, const void *grad_n, const void *grad_x_out, void *grad_x,
                      void *grad_f, void *grad_gate, void *grad_w_post, void *grad_w_pre, void *workspace, size_t workspace_bytes, void *stream)
{
    int st = bt::check_common(x_out, f, gate, w_post, w_pre, rows, d, gate_rows, dtype, scale, eps);
    if (st != BT_OK) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if ((grad_gate && !gate && rows) || (grad_w_post && !w_post && rows) || (grad_f && !f && rows)) return BT_ERR_NULL;
    for (const void *p : {static_cast<const void *>(grad_x), static_cast<const void *>(grad_f), static_cast<const void *>(grad_gate),
                          static_cast<const void *>(grad_w_post), static_cast<const void *>(grad_w_pre), grad_n, grad_x_out,
                          static_cast<const void *>(workspace)})
        if (!bt::on_boundary(p, 16)) return BT_ERR_ALIGN;
    const int es = bt::element_size(dtype);
    if (rows == 0) {                                                    // sums over no rows
        for (void *p : {grad_w_post, grad_w_pre})
            if (p && bt::reported(cudaMemsetAsync(p, 0, d * es, s)) != cudaSuccess) return BT_ERR_CUDA;
        return BT_OK;
    }
    if ((grad_n != nullptr) != (w_pre != nullptr) || (grad_w_pre && !w_pre) || (!grad_n && !grad_x_out)) return BT_ERR_NULL;
    const int sms = bt::sm_count();
    if (sms == 0) return BT_ERR_CUDA;
    const bt::Parts p = bt::parts_of(rows, d, es, sms);
    const bool needs  = grad_gate || grad_w_post || grad_w_pre || !bt::row_fits(d, es);
    if (needs && !workspace) return BT_ERR_NULL;
    if (needs && workspace_bytes < p.bytes) return BT_ERR_WORKSPACE;
    unsigned char *w = static_cast<unsigned char *>(workspace);
    bt::NormArgs   a{};
    a.x = x_out, a.f = f, a.gate = gate, a.w_post = w_post, a.w_pre = w_pre, a.dn = grad_n, a.dy = grad_x_out;
    a.x_out = grad_x, a.n_out = grad_f, a.dgate = grad_gate, a.dw_post = grad_w_post, a.dw_pre = grad_w_pre;
    if (needs) {
        a.part_pre = reinterpret_cast<float *>(w + p.pre), a.part_post = reinterpret_cast<float *>(w + p.post);
        a.part_gate = reinterpret_cast<float *>(w + p.gate), a.stats = w + p.stats;
    }
    a.rows = rows, a.d = d, a.gate_rows = gate_rows;
    bt::set_chunks(a, p.chunks);
    a.scale = scale, a.eps = eps;
    return bt::dispatch(dtype, [&](auto dt) { return bt::backward<decltype(dt)::value>(a, s); });
}

}  // extern "C"
