// vms_lowrank and vms_lowrank_backward (include/vms_ops.h): out = y + scale (x a^T) b^T, an adapter for each request.
//
// With ranks of some tens every product here does 2 rank operations per element of x, y or dout that it moves, a tenth of
// what the matrix units could do in that time: all kernels are bound by memory, and the tiles are laid out so that each of
// the wide tensors is read once, 16 bytes a lane, straight into the operand registers of the matrix instructions:
//   down    hidden = scale x a^T     rows of x and of a are both consecutive in the summed dimension
//   up      out = y + hidden b^T     hidden in registers for all columns, the products transposed so that a lane ends up
//                                    with 16 bytes of consecutive columns of one row
//   outer   da = dhidden^T x, db = dout^T hidden, summed over rows: a lane reads some columns of eight rows and swaps
//                                    them in its own registers
// The forward pass is down and up; the backward pass is down on dout with b transposed, up with a transposed, and outer
// twice.  An order of the summed elements is the same for both operands of a product, so any order will do; the lanes'
// loads decide it.
#include "ops_common.hpp"

namespace {

// The 16 x 16 matrix instructions.  Operands: lane = 16 group + m has, of row (or column) m, the EPL elements that start
// at EPL * group; 4 EPL elements are a step.  Result: column m, rows 4 group to 4 group + 3.
template <class T>
struct Mma {
    static const int EPL = 8, STEP = 32;
    typedef T Frag __attribute__((ext_vector_type(8)));
};
template <>
struct Mma<float> {
    static const int EPL = 4, STEP = 16;
    typedef f32x4 Frag;
};
DI f32x4 mma(Mma<float>::Frag a, Mma<float>::Frag b, f32x4 c)
{
#pragma unroll
    for (int i = 0; i < 4; i++) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
    return c;
}
DI f32x4 mma(Mma<f16>::Frag a, Mma<f16>::Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
DI f32x4 mma(Mma<bf16>::Frag a, Mma<bf16>::Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// N consecutive elements at any element's address
template <class T, int N>
struct Some {
    typedef T type __attribute__((ext_vector_type(N)));
    typedef type loose __attribute__((aligned(sizeof(T))));
};
template <int N, class T>
DI typename Some<T, N>::type load_some(const T *p) { return *reinterpret_cast<const typename Some<T, N>::loose *>(p); }
// the same, 0 beyond the first n (n may be negative, p is then not followed)
template <int N, class T>
DI typename Some<T, N>::type load_first(const T *p, int n)
{
    if (LIKELY(n >= N)) return load_some<N>(p);
    typename Some<T, N>::type v;
#pragma unroll
    for (int i = 0; i < N; i++) v[i] = i < n ? p[i] : (T)0.f;
    return v;
}

struct Requests {
    const int32_t *starts, *which;
    u32 n, adapters, rows;
};

struct Tile {
    int adapter;            // -1: none
    u32 row, rows;
};

// rows of request i, kept inside the tensors whatever the numbers say
DI void request_rows(const Requests &q, u32 i, u32 *lo, u32 *hi)
{
    const int a = q.starts[i], b = q.starts[i + 1];
    *lo = min((u32)max(a, 0), q.rows);
    *hi = max(min((u32)max(b, 0), q.rows), *lo);
}

// Tile `tile` of the batch, at most SIZE rows of one request: the wavefront counts the tiles of 64 requests at a time.
// In front of the requests and behind them are the rows that belong to none.
template <int SIZE>
DI bool find_tile(const Requests &q, u32 tile, Tile *out)
{
    if (!q.starts) {
        out->adapter = 0;
        out->row = tile * SIZE;
        out->rows = min((u32)SIZE, q.rows - min(out->row, q.rows));
        return out->row < q.rows;
    }
    u32 before = 0;
    for (u32 base = 0; base < q.n + 2; base += 64) {
        const u32 i = base + lane_id();         // 0: in front, 1 .. n: request i - 1, n + 1: behind
        u32 lo = 0, hi = 0;
        int adapter = -1;
        if (i < q.n + 2) {
            lo = i == 0 ? 0 : min((u32)max(q.starts[i - 1], 0), q.rows);
            hi = i == q.n + 1 ? q.rows : max(min((u32)max(q.starts[i], 0), q.rows), lo);
            if (i > 0 && i <= q.n) adapter = q.which[i - 1];
        }
        u32 total;
        const u32 count = (hi - lo + SIZE - 1) / SIZE, upto = wave_scan_add(count, &total);
        if (tile < before + total) {
            const u32 at = first_lane(ballot(tile < before + upto));
            const u32 nth = tile - before - (from_lane(upto, at) - from_lane(count, at));
            const u32 row = from_lane(lo, at) + nth * SIZE;
            out->row = row;
            out->rows = min((u32)SIZE, from_lane(hi, at) - row);
            out->adapter = (int)from_lane((u32)adapter, at);
            if (out->adapter < 0 || out->adapter >= (int)q.adapters) out->adapter = -1;
            return true;
        }
        before += total;
    }
    return false;
}

// ---- down: hidden[row][j] = scale sum_k x[row][k] w[j][k] ------------------------------------------------------------

struct DownParams {
    const void *x, *w;          // w [adapters][rank][in]
    float *hidden;              // [splits][rows][NR * 16], zeros behind the rank
    const float *scales;
    Requests q;
    u64 ldx;
    float scale;
    u32 in, rank, splits;
};

// STEPS steps of the summed dimension, all loads in front
template <class T, int MR, int NR, int STEPS>
DI void down_steps(const T *const x[MR], const T *const w[NR], u32 s, f32x4 acc[MR][NR])
{
    typedef typename Mma<T>::Frag Frag;
    const int EPL = Mma<T>::EPL, STEP = Mma<T>::STEP;
    Frag a[STEPS][MR], b[STEPS][NR];
#pragma unroll
    for (int k = 0; k < STEPS; k++) {
#pragma unroll
        for (int i = 0; i < MR; i++) a[k][i] = load_some<EPL>(x[i] + (u64)(s + k) * STEP);
#pragma unroll
        for (int j = 0; j < NR; j++) b[k][j] = load_some<EPL>(w[j] + (u64)(s + k) * STEP);
    }
#pragma unroll
    for (int k = 0; k < STEPS; k++)
#pragma unroll
        for (int i = 0; i < MR; i++)
#pragma unroll
            for (int j = 0; j < NR; j++) acc[i][j] = mma(b[k][j], a[k][i], acc[i][j]);
}

// MR x 16 rows and the whole rank in a workgroup; its four wavefronts, and `splits` workgroups, share the summed dimension.
template <class T, int MR, int NR>
__global__ __launch_bounds__(256) void lowrank_down_kernel(const DownParams p)
{
    typedef typename Mma<T>::Frag Frag;
    const int EPL = Mma<T>::EPL, STEP = Mma<T>::STEP, AT_ONCE = 2;
    __shared__ f32x4 part[4][NR][64];
    Tile t;
    if (!find_tile<MR * 16>(p.q, blockIdx.x, &t) || t.adapter < 0) return;
    const u32 lane = lane_id(), m = lane & 15, group = lane >> 4, wave = wave_of_group();
    const T *x[MR], *w[NR];     // rows beyond the tile and the rank are the last one again: their results go nowhere
#pragma unroll
    for (int i = 0; i < MR; i++) x[i] = (const T *)p.x + (t.row + min(i * 16 + m, t.rows - 1)) * p.ldx + group * EPL;
#pragma unroll
    for (int j = 0; j < NR; j++) w[j] = (const T *)p.w + ((u64)t.adapter * p.rank + min(j * 16 + m, p.rank - 1)) * p.in + group * EPL;
    f32x4 acc[MR][NR];
#pragma unroll
    for (int i = 0; i < MR; i++)
#pragma unroll
        for (int j = 0; j < NR; j++) acc[i][j] = f32x4{ 0.f, 0.f, 0.f, 0.f };

    const u32 steps = p.in / STEP, shares = p.splits * 4, share = blockIdx.y * 4 + wave;
    const u32 first = (u32)((u64)steps * share / shares), last = (u32)((u64)steps * (share + 1) / shares);
    u32 s = first;
    for (; s + AT_ONCE <= last; s += AT_ONCE) down_steps<T, MR, NR, AT_ONCE>(x, w, s, acc);
    for (; s < last; s++) down_steps<T, MR, NR, 1>(x, w, s, acc);
    if (share == shares - 1 && steps * STEP < p.in) {
        const int n = (int)(p.in - steps * STEP) - (int)group * EPL;
        Frag b[NR];
#pragma unroll
        for (int j = 0; j < NR; j++) b[j] = load_first<EPL>(w[j] + (u64)steps * STEP, n);
#pragma unroll
        for (int i = 0; i < MR; i++) {
            const Frag a = load_first<EPL>(x[i] + (u64)steps * STEP, n);
#pragma unroll
            for (int j = 0; j < NR; j++) acc[i][j] = mma(b[j], a, acc[i][j]);
        }
    }

    const float scale = p.scales ? p.scales[t.adapter] : p.scale;
#pragma unroll
    for (int i = 0; i < MR; i++) {
        if (i) __syncthreads();
#pragma unroll
        for (int j = 0; j < NR; j++) part[wave][j][lane] = acc[i][j];
        __syncthreads();
        for (u32 at = threadIdx.x; at < NR * 64; at += 256) {
            const u32 j = at >> 6, l = at & 63, row = i * 16 + (l & 15), col = j * 16 + (l >> 4) * 4;
            f32x4 v = part[0][j][l];
#pragma unroll
            for (int u = 1; u < 4; u++)
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] += part[u][j][l][e];
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = col + e < p.rank ? v[e] * scale : 0.f;
            if (row < t.rows) *(f32x4 *)(p.hidden + (((u64)blockIdx.y * p.q.rows + t.row + row) * NR * 16 + col)) = v;
        }
    }
}

// ---- up: out[row][c] = base[row][c] + sum_j hidden[row][j] w[c][j] ---------------------------------------------------

struct UpParams {
    const float *hidden;        // [splits][rows][padded]
    const void *w, *base;       // w [adapters][out][rank]; base nullable
    void *out;
    Requests q;
    u64 ldb, ldo;
    u32 cols, rank, padded, splits, trips;
};

// MR x 16 rows; a wavefront makes 128 bytes of each row at a time, the four of them neighbours, `trips` times.
template <class T, int MR, int JS>
__global__ __launch_bounds__(256) void lowrank_up_kernel(const UpParams p)
{
    typedef typename Mma<T>::Frag Frag;
    const int EPL = Mma<T>::EPL, STEP = Mma<T>::STEP, WIDE = 128 / sizeof(T), QN = EPL / 4;
    Tile t;
    if (!find_tile<MR * 16>(p.q, blockIdx.x, &t)) return;
    const u32 lane = lane_id(), m = lane & 15, group = lane >> 4;
    u32 col = (blockIdx.y * p.trips * 4 + wave_of_group()) * WIDE;
    T *const out = (T *)p.out + (u64)t.row * p.ldo;
    const T *const base = p.base ? (const T *)p.base + (u64)t.row * p.ldb : nullptr;
    if (t.adapter < 0) {
        if (p.base == p.out) return;
        for (u32 trip = 0; trip < p.trips; trip++, col += 4 * WIDE)
            for (u32 r = 0; r < t.rows; r++)
                for (u32 c = col + lane; c < min(col + WIDE, p.cols); c += 64)
                    out[r * p.ldo + c] = base ? base[r * p.ldb + c] : (T)0.f;
        return;
    }
    // hidden, rounded to the type of the tensors: half a step of the type for each term of the sum over the rank
    Frag h[MR][JS];
#pragma unroll
    for (int i = 0; i < MR; i++)
#pragma unroll
        for (int s = 0; s < JS; s++) {
            const u32 j = s * STEP + group * EPL;
            float v[EPL] = {};
            if (j < p.padded) {
                const float *from = p.hidden + (u64)(t.row + min(i * 16 + m, t.rows - 1)) * p.padded + j;
                for (u32 u = 0; u < p.splits; u++, from += (u64)p.q.rows * p.padded)
#pragma unroll
                    for (int e = 0; e < EPL; e += 4) {
                        const f32x4 f = *(const f32x4 *)(from + e);
#pragma unroll
                        for (int k = 0; k < 4; k++) v[e + k] += f[k];
                    }
            }
#pragma unroll
            for (int e = 0; e < EPL; e++) h[i][s][e] = (T)v[e];
        }
    const T *const w = (const T *)p.w + (u64)t.adapter * p.cols * p.rank;
    for (u32 trip = 0; trip < p.trips; trip++, col += 4 * WIDE) {
#pragma unroll
        for (int half = 0; half < 2; half++) {
            const u32 c0 = col + half * (WIDE / 2);
            if (c0 >= p.cols) return;
            // product q has the columns whose place in a lane's EPL is 4 q to 4 q + 3
            Frag b[QN][JS];
#pragma unroll
            for (int q = 0; q < QN; q++) {
                const u32 c = min(c0 + (m >> 2) * EPL + q * 4 + (m & 3), p.cols - 1);
#pragma unroll
                for (int s = 0; s < JS; s++) {
                    const u32 j = s * STEP + group * EPL;
                    b[q][s] = load_first<EPL>(w + (u64)c * p.rank + j, (int)p.rank - (int)j);
                }
            }
            const u32 c = c0 + group * EPL;
            const int n = (int)p.cols - (int)c;
#pragma unroll
            for (int i = 0; i < MR; i++) {
                const u32 row = i * 16 + m;
                f32x4 acc[QN];
#pragma unroll
                for (int q = 0; q < QN; q++) {
                    acc[q] = f32x4{ 0.f, 0.f, 0.f, 0.f };
#pragma unroll
                    for (int s = 0; s < JS; s++) acc[q] = mma(b[q][s], h[i][s], acc[q]);
                }
                if (row < t.rows && n > 0) {
                    Frag y;
#pragma unroll
                    for (int e = 0; e < EPL; e++) y[e] = (T)0.f;
                    if (base) y = load_first<EPL>(base + row * p.ldb + c, n);
#pragma unroll
                    for (int e = 0; e < EPL; e++) y[e] = (T)((float)y[e] + acc[e >> 2][e & 3]);
                    T *const to = out + row * p.ldo + c;
                    if (LIKELY(n >= EPL)) {
                        *reinterpret_cast<typename Some<T, EPL>::loose *>(to) = y;
                    } else {
#pragma unroll
                        for (int e = 0; e < EPL; e++)
                            if (e < n) to[e] = y[e];
                    }
                }
            }
        }
    }
}

// ---- outer: sums[chunk][adapter][j][c] = sum over the chunk's rows of hidden[row][j] v[row][c] ----------------------

// The 16-bit kernels read hidden as operands of their type, eight rows a lane: [padded][stride].  The 32-bit one reads
// [rows][padded].
struct FoldParams {
    const float *from[2];
    void *to[2];
    u32 splits[2];
    u32 rows, padded, stride;
};

template <class T>
__global__ __launch_bounds__(256) void lowrank_fold_kernel(const FoldParams p)
{
    const u32 job = blockIdx.z, j = blockIdx.y * 16 + (threadIdx.x & 15), row = (blockIdx.x * 16 + (threadIdx.x >> 4)) * 8;
    if (!p.to[job]) return;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = 0.f;
    for (u32 u = 0; u < p.splits[job]; u++)
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (row + e < p.rows) v[e] += p.from[job][((u64)u * p.rows + row + e) * p.padded + j];
    if (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (row + e < p.rows) ((float *)p.to[job])[(u64)(row + e) * p.padded + j] = v[e];
    } else if (row < p.stride) {
        store8((T *)p.to[job] + (u64)j * p.stride + row, 8, v);
    }
}

struct OuterJob {
    const void *v, *hidden;
    float *sums;
    u64 ldv;
    u32 cols, panels, chunks, chunk_rows;
};
struct OuterParams {
    OuterJob job[2];
    Requests q;
    u32 stride;
};

// two 16-bit elements of each of two registers, swapped: (a0 b0) and (a1 b1) of (a0 a1), (b0 b1)
DI u32 low_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
DI u32 high_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// rows t .. t + 31 (n of them) of CQ columns a lane: acc[q][j] += v^T hidden
template <class T, int CQ, int NR>
DI void outer_step(const OuterJob &o, u32 stride, u32 t, u32 n, u32 col, int cols, f32x4 acc[CQ][NR])
{
    typedef typename Mma<T>::Frag Frag;
    const u32 lane = lane_id(), m = lane & 15, group = lane >> 4;
    u32 v[8][CQ / 2];
    const T *const from = (const T *)o.v + col;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const u32 r = group * 8 + e;
        typename Some<T, CQ>::type x;
        if (LIKELY(r < n)) {
            x = load_first<CQ>(from + (t + r) * o.ldv, cols);
        } else {
#pragma unroll
            for (int q = 0; q < CQ; q++) x[q] = (T)0.f;
        }
        __builtin_memcpy(v[e], &x, sizeof x);
    }
    Frag h[NR];
#pragma unroll
    for (int j = 0; j < NR; j++)
        h[j] = load_first<8>((const T *)o.hidden + (u64)(j * 16 + m) * stride + t + group * 8, (int)n - (int)group * 8);
#pragma unroll
    for (int q = 0; q < CQ; q += 2) {
        u32 lo[4], hi[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            lo[e] = low_halves(v[2 * e][q / 2], v[2 * e + 1][q / 2]);
            hi[e] = high_halves(v[2 * e][q / 2], v[2 * e + 1][q / 2]);
        }
        Frag a, b;
        __builtin_memcpy(&a, lo, sizeof a);
        __builtin_memcpy(&b, hi, sizeof b);
#pragma unroll
        for (int j = 0; j < NR; j++) {
            acc[q][j] = mma(a, h[j], acc[q][j]);
            acc[q + 1][j] = mma(b, h[j], acc[q + 1][j]);
        }
    }
}

// the same in 32 bits, four rows an instruction
template <int CQ, int NR>
DI void outer_step32(const OuterJob &o, u32 t, u32 n, u32 col, int cols, f32x4 acc[CQ][NR])
{
    const u32 lane = lane_id(), m = lane & 15, group = lane >> 4;
    typename Some<float, CQ>::type v[4];
    float h[4][NR];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const u32 r = e * 4 + group;
        if (LIKELY(r < n)) {
            v[e] = load_first<CQ>((const float *)o.v + (t + r) * o.ldv + col, cols);
        } else {
#pragma unroll
            for (int q = 0; q < CQ; q++) v[e][q] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < NR; j++) h[e][j] = r < n ? ((const float *)o.hidden)[(u64)(t + r) * (NR * 16) + j * 16 + m] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < 4; e++)
#pragma unroll
        for (int q = 0; q < CQ; q++)
#pragma unroll
            for (int j = 0; j < NR; j++) acc[q][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][q], h[e][j], acc[q][j], 0, 0, 0);
}

// A panel of 16 CQ columns, one chunk of rows, one adapter: the four wavefronts take the steps of its rows in turn and join
// their sums.
template <class T, int CQ, int NR>
__global__ __launch_bounds__(256) void lowrank_outer_kernel(const OuterParams p)
{
    const u32 STEP = sizeof(T) == 4 ? 16 : 32;
    __shared__ float part[4][CQ][64 * 4];
    const u32 blocks = p.job[0].panels * p.job[0].chunks, second = blockIdx.x >= blocks;
    const OuterJob &o = p.job[second];
    const u32 block = blockIdx.x - (second ? blocks : 0), panel = block % o.panels, chunk = block / o.panels, adapter = blockIdx.y;
    const u32 lane = lane_id(), wave = wave_of_group();
    const u32 col = (panel * 16 + (lane & 15)) * CQ;
    const int cols = (int)o.cols - (int)col;
    const u32 from = chunk * o.chunk_rows, upto = min(from + o.chunk_rows, p.q.rows);
    f32x4 acc[CQ][NR];
#pragma unroll
    for (int q = 0; q < CQ; q++)
#pragma unroll
        for (int j = 0; j < NR; j++) acc[q][j] = f32x4{ 0.f, 0.f, 0.f, 0.f };
    const u32 requests = p.q.starts ? p.q.n : 1;
    for (u32 base = 0; base < requests; base += 64) {
        u32 lo = 0, hi = 0;
        const u32 i = base + lane;
        if (!p.q.starts) {
            lo = from;
            hi = lane ? from : upto;
        } else if (i < requests && p.q.which[i] == (int)adapter) {
            request_rows(p.q, i, &lo, &hi);
            lo = max(lo, from);
            hi = min(hi, upto);
        }
        u64 left = ballot(lo < hi);
        while (left) {
            const u32 at = first_lane(left);
            left &= left - 1;
            const u32 end = from_lane(hi, at);
            for (u32 t = from_lane(lo, at) + wave * STEP; t < end; t += 4 * STEP) {
                if constexpr (sizeof(T) == 4)
                    outer_step32<CQ, NR>(o, t, end - t, col, cols, acc);
                else
                    outer_step<T, CQ, NR>(o, p.stride, t, end - t, col, cols, acc);
            }
        }
    }
    // lane 16 group + m has column m of hidden and, for q, the columns (4 group + i) CQ + q of the panel
    float *const sums = o.sums + ((u64)chunk * gridDim.y + adapter) * (NR * 16) * o.cols;
    const u32 place = threadIdx.x & 15, hidden = threadIdx.x >> 4, at = ((place >> 2) * 16 + hidden) * 4 + (place & 3);
    const u32 c = (panel * 16 + place) * CQ;
#pragma unroll
    for (int j = 0; j < NR; j++) {
        if (j) __syncthreads();
#pragma unroll
        for (int q = 0; q < CQ; q++) *(f32x4 *)&part[wave][q][lane * 4] = acc[q][j];
        __syncthreads();
        float *const to = sums + (u64)(j * 16 + hidden) * o.cols + c;
#pragma unroll
        for (int q = 0; q < CQ; q++) {
            const float v = part[0][q][at] + part[1][q][at] + part[2][q][at] + part[3][q][at];
            if (c + q < o.cols) to[q] = v;
        }
    }
}

// da [adapters][rank][cols] or, transposed, db [adapters][cols][rank] from the chunks' sums; eight j a lane
struct JoinJob {
    const float *sums;
    void *to;
    u32 cols, chunks, transposed;
};
struct JoinParams {
    JoinJob job[2];
    u32 rank, padded, first_blocks;
};

template <class T>
__global__ __launch_bounds__(256) void lowrank_join_kernel(const JoinParams p)
{
    const u32 second = blockIdx.x >= p.first_blocks;
    const JoinJob &o = p.job[second];
    const u32 c = (blockIdx.x - (second ? p.first_blocks : 0)) * 256 + threadIdx.x, j = blockIdx.y * 8, adapter = blockIdx.z;
    if (c >= o.cols) return;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = 0.f;
    const u64 apart = (u64)gridDim.z * p.padded * o.cols;
    const float *from = o.sums + ((u64)adapter * p.padded + j) * o.cols + c;
    for (u32 u = 0; u < o.chunks; u++, from += apart)
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += from[(u64)e * o.cols];
    if (o.transposed) {
        store8((T *)o.to + ((u64)adapter * o.cols + c) * p.rank + j, p.rank - j, v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (j + e < p.rank) ((T *)o.to)[((u64)adapter * p.rank + j + e) * o.cols + c] = (T)v[e];
    }
}

// to[i][c][r] = from[i][r][c], a tile of 32 x 32 at a time
struct SwapJob {
    const void *from;
    void *to;
    u32 rows, cols, blocks;
};
struct SwapParams {
    SwapJob job[2];
};

template <class T>
__global__ __launch_bounds__(256) void lowrank_swap_kernel(const SwapParams p)
{
    __shared__ T tile[32][34];
    const u32 second = blockIdx.x >= p.job[0].blocks;
    const SwapJob &o = p.job[second];
    const u32 block = blockIdx.x - (second ? p.job[0].blocks : 0), wide = (o.cols + 31) / 32;
    const u32 c0 = block % wide * 32, r0 = block / wide * 32, x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const u64 start = (u64)blockIdx.y * o.rows * o.cols;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const u32 i = y + k * 8;
        if (r0 + i < o.rows && c0 + x < o.cols) tile[i][x] = ((const T *)o.from)[start + (u64)(r0 + i) * o.cols + c0 + x];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const u32 i = y + k * 8;
        if (c0 + i < o.cols && r0 + x < o.rows) ((T *)o.to)[start + (u64)(c0 + i) * o.rows + r0 + x] = tile[x][i];
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------

u32 padded_rank(u32 rank) { return rank <= 16 ? 16 : rank <= 32 ? 32 : rank <= 64 ? 64 : 128; }

// How a batch is cut.  A tile has as many rows as a request has on average, at most 64 (32 where the rank needs the
// registers): larger tiles read the weights less often, smaller ones keep single tokens from paying for rows that are
// not there.
struct Cut {
    u32 tile16, tiles;      // 16 rows each; tiles there can be
};

Cut cut_of(const vms_lowrank_args *a)
{
    Cut c;
    const u64 requests = a->d_starts ? a->n_requests : 1, each = requests ? a->rows / requests : a->rows;
    c.tile16 = each >= 48 ? 4 : each >= 24 ? 2 : 1;
    if (c.tile16 == 4 && padded_rank(a->rank) == 128) c.tile16 = 2;
    const u64 size = c.tile16 * 16, tiles = a->d_starts ? a->rows / size + requests + 2 : (a->rows + size - 1) / size;
    c.tiles = (u32)(tiles < a->rows ? tiles : a->rows);
    if (!c.tiles) c.tiles = 1;
    return c;
}

// workgroups that share the summed dimension: two on every compute unit, but two steps at least for a wavefront
u32 splits_of(const vms_lowrank_args *a, const Cut &c, u64 in)
{
    const u64 steps = in / (a->dtype == VMS_F32 ? 16 : 32), most = steps / 8;
    u64 s = (2 * OPS_CUS + c.tiles - 1) / c.tiles;
    if (s > most) s = most;
    if (s > 16) s = 16;
    return s ? (u32)s : 1;
}

int check(const vms_lowrank_args *a)
{
    if (!a) return VMS_EINVAL;
    if (a->struct_size != sizeof *a) return VMS_ESTRUCT;
    if (a->dtype > VMS_BF16 || a->rows >> 28 || !a->in || a->in >> 22 || !a->out || a->out >> 22) return VMS_EINVAL;
    if (!a->rank || a->rank > VMS_LOWRANK_MAX_RANK || !a->n_adapters || a->n_adapters > 65535) return VMS_EINVAL;
    if (a->d_starts && a->n_requests >> 22) return VMS_EINVAL;
    return VMS_OK;
}

int check_inputs(const vms_lowrank_args *a)
{
    if (!input_ok(a->d_a, a->dtype) || !input_ok(a->d_b, a->dtype)) return VMS_EINVAL;
    if (a->rows && (!input_ok(a->d_x, a->dtype) || !stride_ok(a->ldx))) return VMS_EINVAL;
    if ((uintptr_t)a->d_scales % 4 || (uintptr_t)a->d_starts % 4 || (uintptr_t)a->d_which % 4) return VMS_EINVAL;
    if (a->d_starts && a->n_requests && !a->d_which) return VMS_EINVAL;
    if (a->rows && (!a->d_hidden || (uintptr_t)a->d_hidden % 16 || a->hidden_bytes < vms_lowrank_hidden_bytes(a))) return VMS_EWORKSPACE;
    return VMS_OK;
}

Requests requests_of(const vms_lowrank_args *a)
{
    return Requests{ a->d_starts, a->d_which, a->d_starts ? a->n_requests : 0, a->n_adapters, (u32)a->rows };
}

template <class T, int MR>
int launch_down(const DownParams &p, u32 tiles, void *stream)
{
    const dim3 grid(tiles, p.splits), block(256);
    switch (padded_rank(p.rank)) {
    case 16: return ops_launch(lowrank_down_kernel<T, MR, 1>, grid, block, 0, p, stream);
    case 32: return ops_launch(lowrank_down_kernel<T, MR, 2>, grid, block, 0, p, stream);
    case 64: return ops_launch(lowrank_down_kernel<T, MR, 4>, grid, block, 0, p, stream);
    }
    return ops_launch(lowrank_down_kernel<T, MR == 4 ? 2 : MR, 8>, grid, block, 0, p, stream);
}

template <class T>
int down(const vms_lowrank_args *a, const Cut &c, const void *x, u64 ldx, const void *w, u64 in, float *hidden, void *stream)
{
    const DownParams p = { x, w, hidden, a->d_scales, requests_of(a), ldx, a->scale, (u32)in, a->rank, splits_of(a, c, in) };
    switch (c.tile16) {
    case 1: return launch_down<T, 1>(p, c.tiles, stream);
    case 2: return launch_down<T, 2>(p, c.tiles, stream);
    }
    return launch_down<T, 4>(p, c.tiles, stream);
}

template <class T, int MR>
int launch_up(const UpParams &p, dim3 grid, void *stream)
{
    const dim3 block(256);
    const int per = Mma<T>::STEP;
    switch (p.padded) {
    case 16: return ops_launch(lowrank_up_kernel<T, MR, 1>, grid, block, 0, p, stream);
    case 32: return ops_launch(lowrank_up_kernel<T, MR, 32 / per>, grid, block, 0, p, stream);
    case 64: return ops_launch(lowrank_up_kernel<T, MR, 64 / per>, grid, block, 0, p, stream);
    }
    return ops_launch(lowrank_up_kernel<T, MR == 4 ? 2 : MR, 128 / per>, grid, block, 0, p, stream);
}

template <class T>
int up(const vms_lowrank_args *a, const Cut &c, const float *hidden, u32 splits, const void *w, const void *base, u64 ldb, void *out,
       u64 ldo, u64 cols, void *stream)
{
    const u64 trip = 4 * 128 / sizeof(T), all = (cols + trip - 1) / trip;
    // workgroups enough for eight on every compute unit before one takes a second trip
    u64 trips = all * c.tiles / (OPS_CUS * 8);
    trips = trips < 1 ? 1 : trips > 8 ? 8 : trips;
    const UpParams p = { hidden, w, base, out, requests_of(a), ldb, ldo, (u32)cols, a->rank, padded_rank(a->rank), splits, (u32)trips };
    const dim3 grid(c.tiles, (u32)((all + trips - 1) / trips));
    switch (c.tile16) {
    case 1: return launch_up<T, 1>(p, grid, stream);
    case 2: return launch_up<T, 2>(p, grid, stream);
    }
    return launch_up<T, 4>(p, grid, stream);
}

// columns that a lane takes in the outer products: as many as the registers hold beside the rank
u32 outer_columns(u32 dtype, u32 padded) { return dtype != VMS_F32 && padded <= 32 ? 8 : 4; }

void outer_cut(const vms_lowrank_args *a, u64 cols, OuterJob *o)
{
    const u32 wide = 16 * outer_columns(a->dtype, padded_rank(a->rank));
    o->cols = (u32)cols;
    o->panels = (u32)((cols + wide - 1) / wide);
    // four workgroups on every compute unit, 128 rows at least for each
    u64 chunks = (OPS_CUS * 4 + (u64)o->panels * a->n_adapters - 1) / ((u64)o->panels * a->n_adapters), most = (a->rows + 127) / 128;
    if (chunks > most) chunks = most;
    if (!chunks) chunks = 1;
    o->chunk_rows = (u32)(((a->rows + chunks - 1) / chunks + 31) / 32 * 32);
    o->chunks = o->chunk_rows ? (u32)((a->rows + o->chunk_rows - 1) / o->chunk_rows) : 1;
}

template <class T>
int launch_outer(const OuterParams &p, u32 padded, dim3 grid, void *stream)
{
    const dim3 block(256);
    const int few = sizeof(T) == 4 ? 4 : 8;
    switch (padded) {
    case 16: return ops_launch(lowrank_outer_kernel<T, few, 1>, grid, block, 0, p, stream);
    case 32: return ops_launch(lowrank_outer_kernel<T, few, 2>, grid, block, 0, p, stream);
    case 64: return ops_launch(lowrank_outer_kernel<T, 4, 4>, grid, block, 0, p, stream);
    }
    return ops_launch(lowrank_outer_kernel<T, 4, 8>, grid, block, 0, p, stream);
}

// where the parts of the backward pass's workspace begin; 0 bytes for what the wanted gradients do not need
struct Layout {
    size_t at, bt, dhidden, hfold, dfold, dasums, dbsums, total;
    OuterJob da, db;
    u32 stride;
};

bool wants_hidden_gradient(const vms_lowrank_backward_args *a) { return a->d_dx || a->d_da; }

Layout layout_of(const vms_lowrank_backward_args *a)
{
    const vms_lowrank_args &f = a->f;
    const size_t e = type_bytes(f.dtype), padded = padded_rank(f.rank);
    const Cut c = cut_of(&f);
    Layout l = {};
    size_t end = 0;
    const auto place = [&end](size_t *at, size_t bytes) {
        *at = end;
        end += (bytes + 255) & ~(size_t)255;
    };
    l.stride = (u32)((f.rows + 7) / 8 * 8);
    const size_t folded = padded * l.stride * e;
    place(&l.at, a->d_dx ? (size_t)f.n_adapters * f.rank * f.in * e : 0);
    place(&l.bt, wants_hidden_gradient(a) ? (size_t)f.n_adapters * f.rank * f.out * e : 0);
    place(&l.dhidden, wants_hidden_gradient(a) ? (size_t)splits_of(&f, c, f.out) * f.rows * padded * 4 : 0);
    place(&l.hfold, a->d_db ? folded : 0);
    place(&l.dfold, a->d_da ? folded : 0);
    outer_cut(&f, f.in, &l.da);
    outer_cut(&f, f.out, &l.db);
    place(&l.dasums, a->d_da ? (size_t)l.da.chunks * f.n_adapters * padded * f.in * 4 : 0);
    place(&l.dbsums, a->d_db ? (size_t)l.db.chunks * f.n_adapters * padded * f.out * 4 : 0);
    l.total = end;
    return l;
}

template <class T>
int backward(const vms_lowrank_backward_args *a, void *stream)
{
    const vms_lowrank_args &f = a->f;
    const u32 padded = padded_rank(f.rank);
    const Cut c = cut_of(&f);
    Layout l = layout_of(a);
    char *const ws = (char *)a->d_workspace;
    float *const dhidden = (float *)(ws + l.dhidden);
    int rc = VMS_OK;
    if (wants_hidden_gradient(a)) {
        const auto blocks = [](u64 r, u64 k) { return (u32)((r + 31) / 32 * ((k + 31) / 32)); };
        SwapParams s = { { { f.d_b, ws + l.bt, (u32)f.out, f.rank, blocks(f.out, f.rank) }, { f.d_a, ws + l.at, f.rank, (u32)f.in, 0 } } };
        if (a->d_dx) s.job[1].blocks = blocks(f.rank, f.in);
        rc = ops_launch(lowrank_swap_kernel<T>, dim3(s.job[0].blocks + s.job[1].blocks, f.n_adapters), dim3(256), 0, s, stream);
        if (!rc) rc = down<T>(&f, c, a->d_dout, a->lddout, ws + l.bt, f.out, dhidden, stream);
    }
    if (!rc && a->d_dx) rc = up<T>(&f, c, dhidden, splits_of(&f, c, f.out), ws + l.at, nullptr, 0, a->d_dx, a->lddx, f.in, stream);
    if (rc || !(a->d_da || a->d_db)) return rc;
    const FoldParams fold = { { f.d_hidden, dhidden },
                              { a->d_db ? ws + l.hfold : nullptr, a->d_da ? ws + l.dfold : nullptr },
                              { splits_of(&f, c, f.in), splits_of(&f, c, f.out) },
                              (u32)f.rows, padded, l.stride };
    rc = ops_launch(lowrank_fold_kernel<T>, dim3((u32)((f.rows + 127) / 128), padded / 16, 2), dim3(256), 0, fold, stream);
    if (rc) return rc;
    OuterParams o = { { l.da, l.db }, requests_of(&f), l.stride };
    o.job[0].v = f.d_x;
    o.job[0].ldv = f.ldx;
    o.job[0].hidden = ws + l.dfold;
    o.job[0].sums = (float *)(ws + l.dasums);
    o.job[1].v = a->d_dout;
    o.job[1].ldv = a->lddout;
    o.job[1].hidden = ws + l.hfold;
    o.job[1].sums = (float *)(ws + l.dbsums);
    JoinParams j = { { { o.job[0].sums, a->d_da, (u32)f.in, l.da.chunks, 0 }, { o.job[1].sums, a->d_db, (u32)f.out, l.db.chunks, 1 } },
                     f.rank, padded, (u32)((f.in + 255) / 256) };
    u32 blocks = (u32)((f.out + 255) / 256);
    if (!a->d_da) o.job[0].chunks = j.first_blocks = 0;
    if (!a->d_db) o.job[1].chunks = blocks = 0;
    const u32 grid = o.job[0].panels * o.job[0].chunks + o.job[1].panels * o.job[1].chunks;
    rc = launch_outer<T>(o, padded, dim3(grid, f.n_adapters), stream);
    if (rc) return rc;
    return ops_launch(lowrank_join_kernel<T>, dim3(j.first_blocks + blocks, (f.rank + 7) / 8, f.n_adapters), dim3(256), 0, j, stream);
}

struct ClearParams {
    void *to[2];
    u64 n[2];
};
__global__ __launch_bounds__(256) void lowrank_clear_kernel(const ClearParams p)
{
    for (int k = 0; k < 2; k++)
        if (p.to[k])
            for (u64 i = blockIdx.x * 256u + threadIdx.x; i < p.n[k]; i += gridDim.x * 256u) ((unsigned short *)p.to[k])[i] = 0;
}

}  // namespace

extern "C" size_t vms_lowrank_hidden_bytes(const vms_lowrank_args *a)
{
    if (check(a)) return 0;
    return (size_t)splits_of(a, cut_of(a), a->in) * a->rows * padded_rank(a->rank) * sizeof(float);
}

extern "C" int vms_lowrank(const vms_lowrank_args *a, void *stream)
{
    int rc = check(a);
    if (rc) return rc;
    if (!a->rows) return VMS_OK;
    rc = check_inputs(a);
    if (rc) return rc;
    if (!input_ok(a->d_y, a->dtype) || !stride_ok(a->ldy) || !output_ok(a->d_out, a->dtype, a->ldo, a->out) || !stride_ok(a->ldo)) return VMS_EINVAL;
    if (a->d_y == a->d_out && a->ldy != a->ldo) return VMS_EINVAL;
    const Cut c = cut_of(a);
    return with_type(a->dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        const int r = down<T>(a, c, a->d_x, a->ldx, a->d_a, a->in, a->d_hidden, stream);
        return r ? r : up<T>(a, c, a->d_hidden, splits_of(a, c, a->in), a->d_b, a->d_y, a->ldy, a->d_out, a->ldo, a->out, stream);
    });
}

extern "C" size_t vms_lowrank_backward_workspace_bytes(const vms_lowrank_backward_args *a)
{
    if (!a || a->struct_size != sizeof *a || check(&a->f) || !a->f.rows) return 0;
    return layout_of(a).total;
}

extern "C" int vms_lowrank_backward(const vms_lowrank_backward_args *a, void *stream)
{
    if (!a) return VMS_EINVAL;
    if (a->struct_size != sizeof *a) return VMS_ESTRUCT;
    int rc = check(&a->f);
    if (rc) return rc;
    const vms_lowrank_args &f = a->f;
    for (const void *d : { a->d_da, a->d_db })
        if (d && !input_ok(d, f.dtype)) return VMS_EINVAL;
    if (!f.rows) {
        if (!a->d_da && !a->d_db) return VMS_OK;
        const u64 halves = type_bytes(f.dtype) / 2 * f.n_adapters * (u64)f.rank;
        const ClearParams p = { { a->d_da, a->d_db }, { halves * f.in, halves * f.out } };
        return ops_launch(lowrank_clear_kernel, dim3(OPS_CUS), dim3(256), 0, p, stream);
    }
    rc = check_inputs(&f);
    if (rc) return rc;
    if (!input_ok(a->d_dout, f.dtype) || !stride_ok(a->lddout)) return VMS_EINVAL;
    if (a->d_dx && (!output_ok(a->d_dx, f.dtype, a->lddx, f.in) || !stride_ok(a->lddx))) return VMS_EINVAL;
    if (!a->d_dx && !a->d_da && !a->d_db) return VMS_OK;
    if (!a->d_workspace || (uintptr_t)a->d_workspace % 16 || a->workspace_bytes < layout_of(a).total) return VMS_EWORKSPACE;
    return with_type(f.dtype, [&](auto *t) { return backward<std::remove_pointer_t<decltype(t)>>(a, stream); });
}
