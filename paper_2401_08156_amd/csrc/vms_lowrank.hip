// vms_lowrank and vms_lowrank_backward (include/vms_ops.h): out = y + scale (x a^T) b^T, an adapter for each request.
//
// With ranks of some tens every product here does 2 rank operations per element of x, y or dout that it moves, a tenth of
// what the matrix units could do in that time: all kernels are bound by memory, and each of the wide tensors is read once,
// straight into the operand registers of the matrix instructions:
//   down    hidden = scale x a^T     summed along the rows of x and of a
//   up      out = y + hidden b^T     a panel of b in the LDS for all rows of a tile
//   outer   da = dhidden^T x, db = dout^T hidden, summed over rows: a lane reads some columns of eight rows and swaps
//                                    them in its own registers
// The forward pass is down and up; the backward pass is down on dout with b transposed, up with a transposed, and outer
// twice.  Single tokens of small adapters have a forward pass of one launch (`one`).  The order of the summed elements is the same for both operands of a product, so any order will do.
//
// The operands want a row in each of 16 neighbouring lanes, the memory path 64 consecutive bytes in each four: taken as the
// operands want them, loads of 16 bytes a lane go through the address unit one lane at a time (64 accesses an instruction by
// its counter; the unit was busy for three quarters of the time, at 2 TB/s).  So four loads take four rows of 256 bytes
// each, and four neighbouring lanes swap their four registers (quad_swap).
#include "ops_common.hpp"

namespace {

// The 16 x 16 matrix instructions.  Operands: lane = 16 group + m has, of row (or column) m, the EPL elements that start
// at EPL * group; 4 EPL elements are a step.  Result: column m, rows 4 group to 4 group + 3.
template <class T>
struct Mma {
    static const int EPL = 8, STEP = 32, PLANES = 2;
    typedef T Frag __attribute__((ext_vector_type(8)));
};
template <>
struct Mma<float> {
    static const int EPL = 4, STEP = 16, PLANES = 1;
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
template <int N, bool ONCE = false, class T>
DI typename Some<T, N>::type load_some(const T *p)
{
    const auto *const from = reinterpret_cast<const typename Some<T, N>::loose *>(p);
    return ONCE ? __builtin_nontemporal_load(from) : *from;
}
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

// the same without a branch, for a row of N elements or more that ends n elements behind p: where those are fewer than N, the
// row's last N, 0 in the place of those that p lies behind.  Which elements a sum takes in which place is all the same, as
// long as both of its factors agree.
template <int N, class T>
DI typename Some<T, N>::type load_last(const T *p, int n)
{
    const int back = max(N - n, 0);
    typename Some<T, N>::type v = load_some<N>(p - back);
    const int PER = 4 / sizeof(T);          // elements of a register
    u32 words[N / PER];
    __builtin_memcpy(words, &v, sizeof v);
#pragma unroll
    for (int i = 0; i < N / PER; i++) words[i] &= back <= i * PER ? ~0u : back < (i + 1) * PER ? 0xFFFF0000u : 0u;
    __builtin_memcpy(&v, words, sizeof v);
    return v;
}

// the same for a shorter row
template <int N, class T>
DI typename Some<T, N>::type load_short(const T *p, int n)
{
    typename Some<T, N>::type v;
#pragma unroll
    for (int i = 0; i < N; i++) {
        const T x = p[min(i, n - 1)];
        v[i] = i < n ? x : (T)0.f;
    }
    return v;
}

// The lanes of a quad swap their registers: lane c's r[i] becomes lane i's r[c]
template <class V>
DI void quad_swap(V r[4])
{
    u32 v[4][4];
    __builtin_memcpy(v, r, sizeof v);
    const bool odd = threadIdx.x & 1, upper = threadIdx.x & 2;
#pragma unroll
    for (int k = 0; k < 4; k++) {
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
            const u32 a = dpp_perm<DPP_QUAD_XOR1>(v[i][k]), b = dpp_perm<DPP_QUAD_XOR1>(v[i + 1][k]);
            v[i][k] = odd ? b : v[i][k];
            v[i + 1][k] = odd ? v[i + 1][k] : a;
        }
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const u32 a = dpp_perm<DPP_QUAD_XOR2>(v[i][k]), b = dpp_perm<DPP_QUAD_XOR2>(v[i + 2][k]);
            v[i][k] = upper ? b : v[i][k];
            v[i + 2][k] = upper ? v[i + 2][k] : a;
        }
    }
    __builtin_memcpy(r, v, sizeof v);
}

// The same four rows of 256 bytes in a lane's terms: before a swap, register u of lane 16 group + 4 quad + c is bytes
// 64 group + 16 c of row 4 quad + u; after it, of row 4 quad + c it has bytes 64 group + 16 u.
const int SLAB_BYTES = 256;
DI u32 slab_row(u32 lane, int u) { return (lane >> 2 & 3) * 4 + u; }
DI u32 slab_byte(u32 lane) { return (lane >> 4) * 64 + (lane & 3) * 16; }

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

// What a batch's hidden values are kept as.  They are sums, and the products that read them take the type of the tensors: in
// 16 bits a value goes through as two of the type, itself rounded and what that left, in two planes.  An output is
// rounded once then, whatever the batch: the two hold a value to 2^-16 of it in bfloat16, to 2^-22 in float16 (to 2^-25 where
// it is small; one beyond 65504 is an infinity).  A single rounded value would save `outer` 16 us of 93 (8192 rows, 4096 -> 16384,
// rank 64) and `up` nothing, and make the outputs' error 1.4 times as large.
// The values are laid out twice, in the order in which the lanes of `up` and of `outer` read them, padded to 16 rows.
// Where there are not tiles enough for the compute units, workgroups share the summed dimension and leave parts of the sums,
// in 32 bits: [splits][rows][padded].
struct Hidden {
    void *up;                   // [planes][rows / 16][padded / EPL][16][EPL]
    void *outer;                // 16 bits: [planes][rows / 8][padded][8]; 32 bits: [rows][padded]
    float *parts;               // not null: what `down` leaves
    u32 splits, padded;
    bool folded;                // the parts are put together in `up` and `outer` before they are read
};

template <class T>
DI u64 up_place(u64 row, u32 j, u32 padded)
{
    const u32 EPL = Mma<T>::EPL;
    return (row >> 4) * 16 * padded + j / EPL * (16 * EPL) + (row & 15) * EPL + j % EPL;
}
template <class T>
DI u64 outer_place(u64 row, u32 j, u32 padded)
{
    return sizeof(T) == 4 ? row * padded + j : ((row >> 3) * padded + j) * 8 + (row & 7);
}

// elements of a plane
DI u64 plane(u64 rows, u32 padded) { return (rows + 15) / 16 * 16 * padded; }

// v as the sum of PLANES values of the type (where the first is an infinity the second adds nothing)
template <class T>
DI void in_planes(float v, T o[2])
{
    o[0] = (T)v;
    const float left = v - (float)o[0];
    o[1] = (T)(fabsf((float)o[0]) < INFINITY ? left : 0.f);
}

// four values of a row, from column `col` of the rank on
template <class T>
DI void store_hidden(const Hidden &h, const f32x4 &v, u64 row, u32 col, u32 split, u64 rows)
{
    if (h.parts) {
        *(f32x4 *)(h.parts + (split * rows + row) * h.padded + col) = v;
        return;
    }
    typename Some<T, 4>::type o[2];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        T both[2];
        in_planes<T>(v[e], both);
        o[0][e] = both[0];
        o[1][e] = both[1];
    }
#pragma unroll
    for (int k = 0; k < Mma<T>::PLANES; k++) {
        const u64 from = k * plane(rows, h.padded);
        *(typename Some<T, 4>::type *)((T *)h.up + from + up_place<T>(row, col, h.padded)) = o[k];
#pragma unroll
        for (int e = 0; e < 4; e++) ((T *)h.outer)[from + outer_place<T>(row, col + e, h.padded)] = o[k][e];
    }
}

struct DownParams {
    const void *x, *w;          // w [adapters][rank][in]
    Hidden h;
    const float *scales;
    Requests q;
    u64 ldx;
    float scale;
    u32 in, rank;
};

// One slab of the summed dimension: 256 bytes of each row, of which `n` elements exist (SLAB_WHOLE: all; SLAB_LAST: the end of
// a row that is a load long or longer; SLAB_SHORT: a shorter row)
enum Slab { SLAB_WHOLE, SLAB_LAST, SLAB_SHORT };
template <class T, int MR, int NR, Slab KIND>
DI void down_slab(const char *x, const char *w, const u32 (&xat)[MR][4], const u32 (&wat)[NR][4], int n, f32x4 (&acc)[MR][NR])
{
    typedef typename Mma<T>::Frag Frag;
    const int EPL = Mma<T>::EPL;
    const int SOME = NR < 4 ? NR : 4;       // of the rank's parts at a time; the registers do not hold more
    Frag a[MR][4], b[SOME][4];
    n -= (int)(slab_byte(lane_id()) / sizeof(T));
    const auto load = [n](const char *p, u32 at) {
        const T *const from = (const T *)(p + at);
        return KIND == SLAB_WHOLE ? load_some<EPL>(from) : KIND == SLAB_LAST ? load_last<EPL>(from, n) : load_short<EPL>(from, n);
    };
#pragma unroll
    for (int i = 0; i < MR; i++)
#pragma unroll
        for (int u = 0; u < 4; u++) a[i][u] = load(x, xat[i][u]);
#pragma unroll
    for (int from = 0; from < NR; from += SOME) {
#pragma unroll
        for (int j = 0; j < SOME; j++)
#pragma unroll
            for (int u = 0; u < 4; u++) b[j][u] = load(w, wat[from + j][u]);
        // (loads in front of the swaps, and those one after the other: mixed freely they take more registers than there are)
        __builtin_amdgcn_sched_barrier(0);
        if (from == 0) {
#pragma unroll
            for (int i = 0; i < MR; i++) {
                quad_swap(a[i]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int j = 0; j < SOME; j++) {
            quad_swap(b[j]);
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int i = 0; i < MR; i++) acc[i][from + j] = mma(b[j][u], a[i][u], acc[i][from + j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// A wavefront's share of the sums for a tile's MR x 16 rows and the whole rank: a run of slabs (16384 x 4096 in 32 bits at rank
// 16: 62 us, 69 with a slab in `shares`), and for the last one what is left of a row.  Tiles begin at different places (`turn`): rows are often a power of two apart, so that what all tiles read
// at one place is in one channel of the caches.
template <class T, int MR, int NR>
DI void down_sums(const DownParams &p, const Tile &t, u32 share, u32 shares, u32 turn, f32x4 (&acc)[MR][NR])
{
    const u32 SLAB = SLAB_BYTES / sizeof(T), lane = lane_id();
    const char *const x = (const char *)((const T *)p.x + t.row * p.ldx);
    const char *const w = (const char *)((const T *)p.w + (u64)t.adapter * p.rank * p.in);
    u32 xat[MR][4], wat[NR][4];     // rows beyond the tile and the rank are the last one again: their results go nowhere
#pragma unroll
    for (int u = 0; u < 4; u++) {
#pragma unroll
        for (int i = 0; i < MR; i++) xat[i][u] = min(i * 16 + slab_row(lane, u), t.rows - 1) * (u32)p.ldx * (u32)sizeof(T) + slab_byte(lane);
#pragma unroll
        for (int j = 0; j < NR; j++) wat[j][u] = min(j * 16 + slab_row(lane, u), p.rank - 1) * p.in * (u32)sizeof(T) + slab_byte(lane);
    }
#pragma unroll
    for (int i = 0; i < MR; i++)
#pragma unroll
        for (int j = 0; j < NR; j++) acc[i][j] = f32x4{ 0.f, 0.f, 0.f, 0.f };
    const u32 slabs = p.in / SLAB;
    turn = slabs ? turn % slabs : 0;
    const u32 run = (slabs + shares - 1) / shares, from = min(share * run, slabs), upto = min(from + run, slabs);
    for (u32 s = from; s < upto; s++) {
        const u64 at = (u64)(s + turn < slabs ? s + turn : s + turn - slabs) * SLAB_BYTES;
        down_slab<T, MR, NR, SLAB_WHOLE>(x + at, w + at, xat, wat, 0, acc);
    }
    if (share == shares - 1 && slabs * SLAB < p.in) {
        const u64 at = (u64)slabs * SLAB_BYTES;
        if (LIKELY(p.in >= (u32)Mma<T>::EPL))
            down_slab<T, MR, NR, SLAB_LAST>(x + at, w + at, xat, wat, (int)(p.in - slabs * SLAB), acc);
        else
            down_slab<T, MR, NR, SLAB_SHORT>(x + at, w + at, xat, wat, (int)p.in, acc);
    }
}

// MR x 16 rows and the whole rank in a workgroup; its WAVES wavefronts, and `splits` workgroups, share the summed dimension.
template <class T, int MR, int NR, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void lowrank_down_kernel(const DownParams p)
{
    __shared__ f32x4 part[WAVES][NR][64];
    Tile t;
    if (!find_tile<MR * 16>(p.q, blockIdx.x, &t) || t.adapter < 0) return;
    const u32 lane = lane_id(), wave = wave_of_group();
    f32x4 acc[MR][NR];
    down_sums<T, MR, NR>(p, t, blockIdx.y * WAVES + wave, p.h.splits * WAVES, blockIdx.x * WAVES, acc);
    const float scale = p.scales ? p.scales[t.adapter] : p.scale;
#pragma unroll
    for (int i = 0; i < MR; i++) {
        if (i) __syncthreads();
#pragma unroll
        for (int j = 0; j < NR; j++) part[wave][j][lane] = acc[i][j];
        __syncthreads();
        for (u32 at = threadIdx.x; at < NR * 64; at += WAVES * 64) {
            const u32 j = at >> 6, l = at & 63, row = i * 16 + (l & 15), col = j * 16 + (l >> 4) * 4;
            f32x4 v = part[0][j][l];
#pragma unroll
            for (int u = 1; u < WAVES; u++)
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] += part[u][j][l][e];
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = col + e < p.rank ? v[e] * scale : 0.f;
            if (row < t.rows) store_hidden<T>(p.h, v, t.row + row, col, blockIdx.y, p.q.rows);
        }
    }
}

// The same for long requests, long sums and ranks above 32.  There the weights, read once for 32 rows, are two thirds of what
// goes through the vector cache.  Here four wavefronts with 32 rows each share them in the LDS, a slab for each half of the
// workgroup at a time, and the next slabs are on their way meanwhile.
template <class T, int NR>
__global__ __launch_bounds__(512) void lowrank_down_shared_kernel(const DownParams p)
{
    typedef typename Mma<T>::Frag Frag;
    const int EPL = Mma<T>::EPL, MR = 2, CHUNKS = NR * 16 * 16, FILL = CHUNKS / 256;
    const u32 SLAB = SLAB_BYTES / sizeof(T);
    __shared__ Frag panel[2][2][CHUNKS];        // 16 chunks of 16 bytes for each of NR * 16 rows of w
    Tile t;
    if (!find_tile<128>(p.q, blockIdx.x, &t) || t.adapter < 0) return;
    const u32 lane = lane_id(), m = lane & 15, group = lane >> 4, wave = wave_of_group(), mine = wave >> 2, local = threadIdx.x & 255;
    const u32 first = (wave & 3) * 32, rows = t.rows > first ? t.rows - first : 0, last = rows ? rows - 1 : 0;
    const char *const x = (const char *)((const T *)p.x + (t.row + (rows ? first : 0)) * p.ldx);
    const char *const w = (const char *)((const T *)p.w + (u64)t.adapter * p.rank * p.in);
    u32 xat[MR][4];
#pragma unroll
    for (int u = 0; u < 4; u++)
#pragma unroll
        for (int i = 0; i < MR; i++) xat[i][u] = min(i * 16 + slab_row(lane, u), last) * (u32)p.ldx * (u32)sizeof(T) + slab_byte(lane);
    f32x4 acc[MR][NR];
#pragma unroll
    for (int i = 0; i < MR; i++)
#pragma unroll
        for (int j = 0; j < NR; j++) acc[i][j] = f32x4{ 0.f, 0.f, 0.f, 0.f };

    // the sums over a slab: its weights in the LDS, x in registers
    const auto multiply = [&](const Frag (&to)[CHUNKS], Frag (&a)[MR][4]) {
        const int AHEAD = NR == 4;              // (the registers of the highest ranks do not hold a second one)
        Frag b[AHEAD + 1][4];
        const auto read = [&](int j) {
#pragma unroll
            for (int u = 0; u < 4; u++) b[j & AHEAD][u] = to[(j * 16 + m) * 16 + ((group * 4 + u) ^ m)];
        };
        if (AHEAD) read(0);
#pragma unroll
        for (int i = 0; i < MR; i++) quad_swap(a[i]);
#pragma unroll
        for (int j = 0; j < NR; j++) {
            if (j + AHEAD < NR) read(j + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < 4; u++)
#pragma unroll
                for (int i = 0; i < MR; i++) acc[i][j] = mma(b[j & AHEAD][u], a[i][u], acc[i][j]);
        }
    };
    // (chunk numbers mixed with the row's: 16 rows of one chunk lie in 16 places)
    const auto place = [&](u32 k) { return (k * 16 + local / 16) * 16 + (local % 16 ^ local / 16); };
    const u32 slabs = p.in / SLAB, shares = p.h.splits * 2, share = blockIdx.y * 2 + mine, trips = (slabs + shares - 1) / shares;
    // Each half takes a run of slabs (55 us for 8192 x 16384 in 16 bits and rank 64, against 64 with slabs taken in turn), and
    // tiles begin at different places.
    const u32 turn = slabs ? blockIdx.x * 5 % slabs : 0;
    u32 wat[FILL];
#pragma unroll
    for (int k = 0; k < FILL; k++) wat[k] = min(k * 16 + local / 16, p.rank - 1) * p.in * (u32)sizeof(T) + local % 16 * 16;
    const auto fetch = [&](u32 trip, Frag (&fill)[FILL], Frag (&a)[MR][4]) {    // slab `trip` of this half's
        const u32 s = share * trips + trip;
        if (s < slabs) {
            const u64 at = (u64)(s + turn < slabs ? s + turn : s + turn - slabs) * SLAB_BYTES;
#pragma unroll
            for (int k = 0; k < FILL; k++) fill[k] = load_some<EPL>((const T *)(w + at + wat[k]));
#pragma unroll
            for (int i = 0; i < MR; i++)
#pragma unroll
                for (int u = 0; u < 4; u++) a[i][u] = load_some<EPL>((const T *)(x + at + xat[i][u]));
        } else {
#pragma unroll
            for (int k = 0; k < FILL; k++) fill[k] = Frag{};
#pragma unroll
            for (int i = 0; i < MR; i++)
#pragma unroll
                for (int u = 0; u < 4; u++) a[i][u] = Frag{};
        }
    };
    // One trip: what was fetched goes to the LDS, the next is fetched, the sums are made.  A panel is written again in the
    // trip after next, when all are past it.
    const auto trip = [&](u32 k, Frag (&fill)[FILL], Frag (&a)[MR][4], Frag (&fill2)[FILL], Frag (&a2)[MR][4]) {
        Frag(&to)[CHUNKS] = panel[k & 1][mine];
#pragma unroll
        for (int i = 0; i < FILL; i++) to[place(i)] = fill[i];
        __syncthreads();
        if (k + 1 < trips) fetch(k + 1, fill2, a2);
        __builtin_amdgcn_sched_barrier(0);
        multiply(to, a);
    };
    Frag fill[2][FILL], a[2][MR][4];
    if (trips) fetch(0, fill[0], a[0]);
    u32 k = 0;
    for (; k + 2 <= trips; k += 2) {
        trip(k, fill[0], a[0], fill[1], a[1]);
        trip(k + 1, fill[1], a[1], fill[0], a[0]);
    }
    if (k < trips) trip(k, fill[0], a[0], fill[1], a[1]);
    if (slabs * SLAB < p.in && blockIdx.y == p.h.splits - 1) {      // what is left of a row, by the last one's first half
        const u64 at = (u64)slabs * SLAB_BYTES;
        const int n = mine ? 0 : (int)(p.in - slabs * SLAB), nx = n - (int)(slab_byte(lane) / sizeof(T));
#pragma unroll
        for (int i = 0; i < FILL; i++) fill[0][i] = load_last<EPL>((const T *)(w + at + wat[i]), n - (int)(local % 16 * EPL));
#pragma unroll
        for (int i = 0; i < MR; i++)
#pragma unroll
            for (int u = 0; u < 4; u++) a[0][i][u] = load_last<EPL>((const T *)(x + at + xat[i][u]), nx);
        Frag(&to)[CHUNKS] = panel[trips & 1][mine];
#pragma unroll
        for (int i = 0; i < FILL; i++) to[place(i)] = fill[0][i];
        __syncthreads();
        multiply(to, a[0]);
    }

    // the second half's sums to the first, through the LDS
    const float scale = p.scales ? p.scales[t.adapter] : p.scale;
    f32x4 *const part = (f32x4 *)panel;
    __syncthreads();
    if (mine == 1) {
#pragma unroll
        for (int i = 0; i < MR; i++)
#pragma unroll
            for (int j = 0; j < NR; j++) part[((wave & 3) * MR * NR + i * NR + j) * 64 + lane] = acc[i][j];
    }
    __syncthreads();
    if (mine == 1) return;
#pragma unroll
    for (int i = 0; i < MR; i++)
#pragma unroll
        for (int j = 0; j < NR; j++) {
            const f32x4 other = part[(wave * MR * NR + i * NR + j) * 64 + lane];
            const u32 row = i * 16 + m, col = j * 16 + group * 4;
            f32x4 v;
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = col + e < p.rank ? (acc[i][j][e] + other[e]) * scale : 0.f;
            if (row < rows) store_hidden<T>(p.h, v, t.row + first + row, col, blockIdx.y, p.q.rows);
        }
}

// ---- up: out[row][c] = base[row][c] + sum_j hidden[row][j] w[c][j] ---------------------------------------------------

struct UpParams {
    Hidden h;
    const void *w, *base;       // w [adapters][out][rank]; base nullable
    void *out;
    Requests q;
    u64 ldb, ldo;
    u32 cols, rank, trips, panels;
};

// Place of chunk `ch` (16 bytes along the rank) of column n of a panel, CPR chunks a column.  What 16 lanes read together
// are columns of four quarters of the panel, four neighbours of each: those bits of n are mixed into the chunk's number so
// that they lie in 16 places of 16 bytes that the LDS has at once.
template <int CPR, int QUARTER>
DI u32 panel_place(u32 n, u32 ch)
{
    const u32 q = n / QUARTER & 3;
    const u32 f = CPR == 4 ? q : CPR == 8 ? (n >> 1 & 1) | q << 1 : (n & 3) | q << 2;
    return n * CPR + (ch ^ f);
}

// Tiles of WR x MR x 16 rows.  A wavefront makes 256 bytes of each of its MR x 16 rows at a time, `trips` times.  WR = 4:
// the four of them have rows of their own and the same columns, whose part of w they share; WR = 1: the same rows, and
// columns and panels of their own.
template <class T, int MR, int JS, int WR, bool ONCE>
__global__ __launch_bounds__(256) void lowrank_up_kernel(const UpParams p)
{
    typedef typename Mma<T>::Frag Frag;
    const int EPL = Mma<T>::EPL, STEP = Mma<T>::STEP, PLANES = Mma<T>::PLANES, QN = EPL / 4, SLAB = SLAB_BYTES / sizeof(T), CPR = JS * STEP / EPL;
    const int PANELS = 4 / WR, FILL = SLAB * CPR / (64 * WR);       // chunks of a panel that a lane fetches
    __shared__ Frag panel[WR == 4 ? 2 : 1][PANELS][SLAB * CPR];
    Tile t;
    const u32 block = die_order(blockIdx.x, gridDim.x);
    if (!find_tile<WR * MR * 16>(p.q, block / p.panels, &t)) return;
    const u32 lane = lane_id(), m = lane & 15, group = lane >> 4, wave = wave_of_group();
    const u32 first = WR == 4 ? wave * MR * 16 : 0, rows = t.rows > first ? t.rows - first : 0, mine = WR == 4 ? 0 : wave;
    u32 col = (block % p.panels * p.trips * PANELS + mine) * SLAB;
    const bool none = t.adapter < 0;
    if (none && p.base == p.out) return;
    const u32 last = rows ? rows - 1 : 0;
    const u64 row0 = t.row + (rows ? first : 0);    // rows beyond the tile are its last one again, and not stored
    Frag h[PLANES][MR][JS];
#pragma unroll
    for (int i = 0; i < MR; i++) {
        const u64 row = row0 + min(i * 16 + m, last);
        if (none) break;
#pragma unroll
        for (int s = 0; s < JS; s++) {
            const u32 j = s * STEP + group * EPL;
            if (j >= p.h.padded) {
#pragma unroll
                for (int k = 0; k < PLANES; k++) h[k][i][s] = Frag{};
            } else if (!p.h.parts) {
#pragma unroll
                for (int k = 0; k < PLANES; k++)
                    h[k][i][s] = *(const Frag *)((const T *)p.h.up + k * plane(p.q.rows, p.h.padded) + up_place<T>(row, j, p.h.padded));
            } else {
                float v[EPL] = {};
                const float *from = p.h.parts + row * p.h.padded + j;
                for (u32 u = 0; u < p.h.splits; u++, from += (u64)p.q.rows * p.h.padded)
#pragma unroll
                    for (int e = 0; e < EPL; e += 4) {
                        const f32x4 f = *(const f32x4 *)(from + e);
#pragma unroll
                        for (int k = 0; k < 4; k++) v[e + k] += f[k];
                    }
#pragma unroll
                for (int e = 0; e < EPL; e++) {
                    T both[2];
                    in_planes<T>(v[e], both);
#pragma unroll
                    for (int k = 0; k < PLANES; k++) h[k][i][s][e] = both[k];
                }
            }
        }
    }
    const T *const w = (const T *)p.w + (u64)(none ? 0 : t.adapter) * p.cols * p.rank;
    const char *const base = p.base ? (const char *)((const T *)p.base + row0 * p.ldb) : nullptr;
    char *const out = (char *)((T *)p.out + row0 * p.ldo);
    u32 yat[MR][4];
#pragma unroll
    for (int i = 0; i < MR; i++)
#pragma unroll
        for (int u = 0; u < 4; u++) yat[i][u] = min(i * 16 + slab_row(lane, u), last) * (u32)p.ldb * (u32)sizeof(T);
    for (u32 trip = 0; trip < p.trips; trip++, col += PANELS * SLAB) {
        Frag(&to)[SLAB * CPR] = panel[WR == 4 ? trip & 1 : 0][mine];
        const u32 c = col + slab_byte(lane) / sizeof(T);
        Frag y[MR][4], fill[FILL];
        const bool whole = p.rank % EPL == 0 && col + SLAB <= p.cols;
        if (LIKELY(whole)) {        // no chunk is cut: one that is beyond the rank is another one, cleared
#pragma unroll
            for (int k = 0; k < FILL; k++) {
                const u32 at = k * 64 * WR + (WR == 4 ? threadIdx.x : lane), j = at % CPR * EPL;
                fill[k] = load_some<EPL>(w + (u64)(col + at / CPR) * p.rank + min(j, p.rank - EPL));
                if (j >= p.rank) fill[k] = Frag{};
            }
            if (base) {
#pragma unroll
                for (int i = 0; i < MR; i++)
#pragma unroll
                    for (int u = 0; u < 4; u++) y[i][u] = load_some<EPL, ONCE>((const T *)(base + yat[i][u]) + c);
            }
        } else {
#pragma unroll
            for (int k = 0; k < FILL; k++) {
                const u32 at = k * 64 * WR + (WR == 4 ? threadIdx.x : lane), n = min(col + at / CPR, p.cols - 1), j = at % CPR * EPL;
                fill[k] = load_first<EPL>(w + (u64)n * p.rank + j, (int)p.rank - (int)j);
            }
            if (base) {
#pragma unroll
                for (int i = 0; i < MR; i++)
#pragma unroll
                    for (int u = 0; u < 4; u++) y[i][u] = load_first<EPL>((const T *)(base + yat[i][u]) + c, (int)p.cols - (int)c);
            }
        }
#pragma unroll
        for (int k = 0; k < FILL; k++) {
            const u32 at = k * 64 * WR + (WR == 4 ? threadIdx.x : lane);
            to[panel_place<CPR, SLAB / 4>(at / CPR, at % CPR)] = fill[k];
        }
        // shared: this panel is written again in the trip after next, when all are past it; a wavefront's own: the LDS
        // answers it in order
        if (WR == 4)
            __syncthreads();
        else
            wave_sync();
        if (!rows || col >= p.cols) continue;
        if (base && !none) {
#pragma unroll
            for (int i = 0; i < MR; i++) quad_swap(y[i]);
        }
        // Product (u, q) has the columns whose place in the slab is SLAB / 4 group + EPL u + 4 q + 0 to 3: a lane ends up
        // with EPL consecutive columns of one row in its register u, as it has them of y.
#pragma unroll
        for (int u = 0; u < 4; u++) {
            if (none) break;
            f32x4 acc[MR][QN];
#pragma unroll
            for (int q = 0; q < QN; q++) {
                const u32 n = (m >> 2) * (SLAB / 4) + u * EPL + q * 4 + (m & 3);
#pragma unroll
                for (int i = 0; i < MR; i++) acc[i][q] = f32x4{ 0.f, 0.f, 0.f, 0.f };
#pragma unroll
                for (int s = 0; s < JS; s++) {
                    const Frag b = to[panel_place<CPR, SLAB / 4>(n, s * (STEP / EPL) + group)];
#pragma unroll
                    for (int k = 0; k < PLANES; k++)
#pragma unroll
                        for (int i = 0; i < MR; i++) acc[i][q] = mma(b, h[k][i][s], acc[i][q]);
                }
            }
#pragma unroll
            for (int i = 0; i < MR; i++)
#pragma unroll
                for (int e = 0; e < EPL; e++) y[i][u][e] = (T)((base ? (float)y[i][u][e] : 0.f) + acc[i][e >> 2][e & 3]);
        }
        const int n = (int)p.cols - (int)c;
#pragma unroll
        for (int i = 0; i < MR; i++) {
            if (!none) quad_swap(y[i]);
#pragma unroll
            for (int u = 0; u < 4; u++) {
                if (none && !base) y[i][u] = Frag{};
                const u32 row = i * 16 + slab_row(lane, u);
                if (row >= rows) continue;
                T *const dst = (T *)(out + row * (u32)p.ldo * (u32)sizeof(T)) + c;
                if (LIKELY(n >= EPL)) {
                    auto *const to16 = reinterpret_cast<typename Some<T, EPL>::loose *>(dst);
                    if (ONCE)
                        __builtin_nontemporal_store(y[i][u], to16);
                    else
                        *to16 = y[i][u];
                } else {
#pragma unroll
                    for (int e = 0; e < EPL; e++)
                        if (e < n) dst[e] = y[i][u][e];
                }
            }
        }
    }
}

// The same for requests of one token or two (96 of them, 4096 -> 16384 at rank 16: 12 us, 18 with the matrix units, which have
// one row in 16 to work on), where the forward pass is not the one launch below, and for their dx.  All there is to read is w:
// a lane has 16 bytes of it, the CPR lanes of a column put their sums together, and a wavefront makes 64 columns at a time.  A
// chunk of the rank belongs to the same lane in all of them, so its part of the (up to FEW_ROWS) rows' hidden values stays in
// registers, in 32 bits.
const int FEW_ROWS = 4;

// What 64 columns need: w, and the column of base that a lane keeps
template <class T, int CPR>
struct Few {
    typename Mma<T>::Frag w[CPR];
    T y[FEW_ROWS];
};

template <int CPR>
DI u32 few_column(u32 c0) { return c0 + lane_id() % CPR * (64 / CPR) + lane_id() / CPR; }

template <class T, int CPR>
DI void few_load(const UpParams &p, const Tile &t, u32 c0, Few<T, CPR> &f)
{
    const int EPL = Mma<T>::EPL;
    const u32 lane = lane_id(), col = few_column<CPR>(c0);
    const T *const w = (const T *)p.w + (u64)max(t.adapter, 0) * p.cols * p.rank;
#pragma unroll
    for (int i = 0; i < CPR; i++) f.w[i] = load_some<EPL>(w + (u64)min(c0 + (i * 64 + lane) / CPR, p.cols - 1) * p.rank + lane % CPR * EPL);
#pragma unroll
    for (int r = 0; r < FEW_ROWS; r++) {
        f.y[r] = (T)0.f;
        if (p.base && (u32)r < t.rows && col < p.cols) f.y[r] = ((const T *)p.base)[(t.row + r) * p.ldb + col];
    }
}

template <class T, int CPR>
DI void few_store(const UpParams &p, const Tile &t, u32 c0, const Few<T, CPR> &f, const float (&h)[FEW_ROWS][Mma<T>::EPL])
{
    const u32 chunk = lane_id() % CPR, col = few_column<CPR>(c0);
#pragma unroll
    for (int r = 0; r < FEW_ROWS; r++) {
        if ((u32)r >= t.rows) break;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < CPR; i++) {
            float v = 0.f;
#pragma unroll
            for (int e = 0; e < Mma<T>::EPL; e++) v += h[r][e] * (float)f.w[i][e];
            if (CPR > 1) v = dpp_add<DPP_QUAD_XOR1, 0xF>(v);
            if (CPR > 2) v = dpp_add<DPP_QUAD_XOR2, 0xF>(v);
            if (CPR > 4) v = dpp_add<DPP_ROW_HALF_MIRROR, 0xF>(v);
            if (CPR > 8) v = dpp_add<DPP_ROW_MIRROR, 0xF>(v);
            sum = chunk == i ? v : sum;
        }
        const float y = (float)f.y[r];
        if (col < p.cols) ((T *)p.out)[(t.row + r) * p.ldo + col] = (T)(t.adapter < 0 ? y : y + sum);
    }
}

template <class T, int CPR>
__global__ __launch_bounds__(256) void lowrank_up_few_kernel(const UpParams p)
{
    typedef typename Mma<T>::Frag Frag;
    const int EPL = Mma<T>::EPL;
    Tile t;
    const u32 block = die_order(blockIdx.x, gridDim.x);
    if (!find_tile<FEW_ROWS>(p.q, block / p.panels, &t)) return;
    const bool none = t.adapter < 0;
    if (none && p.base == p.out) return;
    const u32 lane = lane_id(), chunk = lane % CPR;
    float h[FEW_ROWS][EPL];
#pragma unroll
    for (int r = 0; r < FEW_ROWS; r++) {
        const u64 row = t.row + min((u32)r, t.rows - 1);
#pragma unroll
        for (int e = 0; e < EPL; e++) h[r][e] = 0.f;
        if (none) continue;
        if (p.h.parts) {
            for (u32 u = 0; u < p.h.splits; u++) {
                const float *from = p.h.parts + (u * (u64)p.q.rows + row) * p.h.padded + chunk * EPL;
#pragma unroll
                for (int e = 0; e < EPL; e++) h[r][e] += from[e];
            }
        } else {
#pragma unroll
            for (int k = 0; k < Mma<T>::PLANES; k++) {
                const Frag f = *(const Frag *)((const T *)p.h.up + k * plane(p.q.rows, p.h.padded) + up_place<T>(row, chunk * EPL, p.h.padded));
#pragma unroll
                for (int e = 0; e < EPL; e++) h[r][e] += (float)f[e];
            }
        }
    }
    u32 c0 = (block % p.panels * p.trips * 4 + wave_of_group()) * 64;
    for (u32 trip = 0; trip < p.trips && c0 < p.cols; trip++, c0 += 256) {
        Few<T, CPR> f;
        few_load(p, t, c0, f);
        few_store(p, t, c0, f, h);
    }
}

// Both products in one launch, for few tokens of small adapters: every workgroup makes the hidden values of its tile itself,
// which costs it the read of a and saves the wait for another kernel.  The weights of the first columns, and then always those
// of the next, are on their way meanwhile.
const int ONE_WAVES = 8;

struct OneParams {
    DownParams d;
    UpParams u;
};

template <class T, int CPR>
__global__ __launch_bounds__(ONE_WAVES * 64) void lowrank_one_kernel(const OneParams p)
{
    const int EPL = Mma<T>::EPL, NR = CPR * EPL > 16 ? CPR * EPL / 16 : 1;
    const bool NEXT = CPR <= 4;     // (the registers of the others do not hold two)
    __shared__ f32x4 part[ONE_WAVES][NR][64];
    __shared__ float hidden[FEW_ROWS][NR * 16];
    Tile t;
    const u32 block = die_order(blockIdx.x, gridDim.x), panel = block % p.u.panels, rank = p.d.rank;
    if (!find_tile<FEW_ROWS>(p.d.q, block / p.u.panels, &t)) return;
    const bool none = t.adapter < 0;
    if (none && p.u.base == p.u.out) return;
    const u32 lane = lane_id(), wave = wave_of_group(), step = ONE_WAVES * 64;
    u32 c0 = (panel * p.u.trips * ONE_WAVES + wave) * 64;
    const u32 upto = min((panel + 1) * p.u.trips * step, p.u.cols);
    Few<T, CPR> f[NEXT ? 2 : 1];
    if (NEXT && c0 < upto) few_load(p.u, t, c0, f[0]);
    float h[FEW_ROWS][EPL] = {};
    if (!none) {
        f32x4 acc[1][NR];
        down_sums<T, 1, NR>(p.d, t, wave, ONE_WAVES, block * ONE_WAVES, acc);
#pragma unroll
        for (int j = 0; j < NR; j++) part[wave][j][lane] = acc[0][j];
        __syncthreads();
        const float scale = p.d.scales ? p.d.scales[t.adapter] : p.d.scale;
        for (u32 at = threadIdx.x; at < NR * 64; at += step) {
            const u32 j = at >> 6, l = at & 63, row = l & 15, col = j * 16 + (l >> 4) * 4;
            f32x4 v = part[0][j][l];
#pragma unroll
            for (int u = 1; u < ONE_WAVES; u++)
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] += part[u][j][l][e];
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = col + e < rank ? v[e] * scale : 0.f;
            if (row >= t.rows) continue;
            *(f32x4 *)&hidden[row][col] = v;
            if (panel == 0) store_hidden<T>(p.d.h, v, t.row + row, col, 0, p.d.q.rows);      // for the backward pass
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < FEW_ROWS; r++)
#pragma unroll
            for (int e = 0; e < EPL; e++) h[r][e] = (u32)r < t.rows ? hidden[r][lane % CPR * EPL + e] : 0.f;
    }
    for (; c0 < upto; c0 += step) {
        if (!NEXT) few_load(p.u, t, c0, f[0]);
        if (NEXT && c0 + step < upto) few_load(p.u, t, c0 + step, f[1 % (NEXT + 1)]);
        few_store(p.u, t, c0, f[0], h);
        if (NEXT) f[0] = f[1 % (NEXT + 1)];
    }
}

// ---- outer: sums[chunk][adapter][j][c] = sum over the chunk's rows of hidden[row][j] v[row][c] ----------------------

// whole hidden values from parts
struct FoldParams {
    Hidden h[2];
    bool up[2], outer[2];       // which of the layouts are wanted
    u32 rows;
};

template <class T>
__global__ __launch_bounds__(64) void lowrank_fold_kernel(const FoldParams p)
{
    const Hidden &h = p.h[blockIdx.z];
    const bool up = p.up[blockIdx.z], outer = p.outer[blockIdx.z];
    const u32 quads = h.padded / 4;             // four values of four rows a lane
    const u32 at = blockIdx.x * 64 + threadIdx.x, col = at % quads * 4, row = at / quads * 4;
    if (row >= p.rows || !(up || outer)) return;
    f32x4 v[4];
#pragma unroll
    for (int r = 0; r < 4; r++) v[r] = f32x4{ 0.f, 0.f, 0.f, 0.f };
    for (u32 u = 0; u < h.splits; u += 4) {         // four parts' loads under way at a time
        f32x4 f[4][4];
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int r = 0; r < 4; r++)
                f[k][r] = u + k < h.splits && row + r < p.rows ? *(const f32x4 *)(h.parts + ((u64)(u + k) * p.rows + row + r) * h.padded + col) : f32x4{};
#pragma unroll
        for (int r = 0; r < 4; r++)
#pragma unroll
            for (int e = 0; e < 4; e++) v[r][e] += (f[0][r][e] + f[1][r][e]) + (f[2][r][e] + f[3][r][e]);
    }
    typedef typename Some<T, 4>::type Four;
#pragma unroll
    for (int r = 0; r < 4; r++) {
        Four o[2], c[2];            // row + r, and in 16 bits the four rows of column col + r
#pragma unroll
        for (int e = 0; e < 4; e++) {
            T both[2];
            in_planes<T>(v[r][e], both);
            o[0][e] = both[0];
            o[1][e] = both[1];
            in_planes<T>(sizeof(T) == 4 ? v[r][e] : v[e][r], both);
            c[0][e] = both[0];
            c[1][e] = both[1];
        }
#pragma unroll
        for (int k = 0; k < Mma<T>::PLANES; k++) {
            const u64 from = k * plane(p.rows, h.padded);
            if (up) *(Four *)((T *)h.up + from + up_place<T>(row + r, col, h.padded)) = o[k];
            if (outer) *(Four *)((T *)h.outer + from + (sizeof(T) == 4 ? outer_place<T>(row + r, col, h.padded) : outer_place<T>(row, col + r, h.padded))) = c[k];
        }
    }
}

// (The last rows' chunks come first: the kernel before has read dout from front to back, and its end may still be in the last
// cache.)
struct OuterJob {
    const void *v, *hidden;
    float *sums;
    u64 ldv;
    u32 cols, panels, chunks, chunk_rows;
};
struct OuterParams {
    OuterJob job[2];
    Requests q;
};

// two 16-bit elements of each of two registers, swapped: (a0 b0) and (a1 b1) of (a0 a1), (b0 b1)
DI u32 low_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
DI u32 high_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Rows t to t + 31 of CQ columns a lane, and what belongs to them of hidden; 0 in the place of rows that are not from lo to
// hi - 1, whatever lies there.  t is a multiple of 8.  WHOLE: all of these rows, and whole panels.
template <class T, int CQ, int NR, bool WHOLE>
DI void outer_load(const OuterJob &o, u32 t, u32 lo, u32 hi, u32 rows, u32 col, int cols, u32 (&v)[8][CQ / 2], typename Mma<T>::Frag (&h)[2][NR])
{
    typedef typename Mma<T>::Frag Frag;
    const u32 lane = lane_id(), m = lane & 15, r0 = t + (lane >> 4) * 8;
    const T *const from = (const T *)o.v + r0 * o.ldv + col;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        typename Some<T, CQ>::type x = {};
        if (WHOLE)
            x = load_some<CQ>(from + e * o.ldv);
        else if (r0 + e >= lo && r0 + e < hi)
            x = load_first<CQ>(from + e * o.ldv, cols);
        __builtin_memcpy(v[e], &x, sizeof x);
    }
#pragma unroll
    for (int k = 0; k < 2; k++) {
#pragma unroll
        for (int j = 0; j < NR; j++) {
            h[k][j] = Frag{};
            if (WHOLE || (r0 + 8 > lo && r0 < hi))
                h[k][j] = *(const Frag *)((const T *)o.hidden + k * plane(rows, NR * 16) + outer_place<T>(r0, j * 16 + m, NR * 16));
            if (!WHOLE) {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (r0 + e < lo || r0 + e >= hi) h[k][j][e] = (T)0.f;
            }
        }
    }
}

// acc[q][j] += v^T hidden for column q of a lane and the j-th 16 of the rank
template <class T, int CQ, int NR>
DI void outer_add(const u32 (&v)[8][CQ / 2], const typename Mma<T>::Frag (&h)[2][NR], f32x4 (&acc)[CQ][NR])
{
    typedef typename Mma<T>::Frag Frag;
#pragma unroll
    for (int q = 0; q < CQ; q += 2) {
        u32 low[4], high[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            low[e] = low_halves(v[2 * e][q / 2], v[2 * e + 1][q / 2]);
            high[e] = high_halves(v[2 * e][q / 2], v[2 * e + 1][q / 2]);
        }
        Frag a, b;
        __builtin_memcpy(&a, low, sizeof a);
        __builtin_memcpy(&b, high, sizeof b);
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int j = 0; j < NR; j++) {
                acc[q][j] = mma(a, h[k][j], acc[q][j]);
                acc[q + 1][j] = mma(b, h[k][j], acc[q + 1][j]);
            }
    }
}

// the same in 32 bits, 16 rows, four an instruction
template <int CQ, int NR, bool WHOLE>
DI void outer_load32(const OuterJob &o, u32 t, u32 lo, u32 hi, u32 col, int cols, typename Some<float, CQ>::type (&v)[4], float (&h)[4][NR])
{
    const u32 lane = lane_id(), m = lane & 15, group = lane >> 4;
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const u32 r = t + e * 4 + group;
        const bool in = WHOLE || (r >= lo && r < hi);
        v[e] = typename Some<float, CQ>::type{};
        if (WHOLE)
            v[e] = load_some<CQ>((const float *)o.v + r * o.ldv + col);
        else if (in)
            v[e] = load_first<CQ>((const float *)o.v + r * o.ldv + col, cols);
#pragma unroll
        for (int j = 0; j < NR; j++) h[e][j] = in ? ((const float *)o.hidden)[outer_place<float>(r, j * 16 + m, NR * 16)] : 0.f;
    }
}

template <int CQ, int NR>
DI void outer_add32(const typename Some<float, CQ>::type (&v)[4], const float (&h)[4][NR], f32x4 (&acc)[CQ][NR])
{
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
    const u32 block = blockIdx.x - (second ? blocks : 0), panel = block % o.panels, chunk = o.chunks - 1 - block / o.panels, adapter = blockIdx.y;
    const u32 lane = lane_id(), wave = wave_of_group();
    const u32 col = (panel * 16 + (lane & 15)) * CQ;
    const int cols = (int)o.cols - (int)col;
    const bool panel_whole = (panel + 1) * 16 * CQ <= o.cols;
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
        if (!p.q.starts) {          // one request, of adapter 0
            lo = from;
            hi = lane || adapter ? from : upto;
        } else if (i < requests && p.q.which[i] == (int)adapter) {
            request_rows(p.q, i, &lo, &hi);
            lo = max(lo, from);
            hi = min(hi, upto);
        }
        u64 left = ballot(lo < hi);
        while (left) {
            const u32 at = first_lane(left);
            left &= left - 1;
            const u32 begin = from_lane(lo, at), end = from_lane(hi, at);
            for (u32 t = begin / 8 * 8 + wave * STEP; t < end; t += 4 * STEP) {
                const bool whole = panel_whole && t >= begin && t + STEP <= end;
                if constexpr (sizeof(T) == 4) {
                    typename Some<float, CQ>::type v[4];
                    float h[4][NR];
                    if (LIKELY(whole))
                        outer_load32<CQ, NR, true>(o, t, begin, end, col, cols, v, h);
                    else
                        outer_load32<CQ, NR, false>(o, t, begin, end, col, cols, v, h);
                    outer_add32<CQ, NR>(v, h, acc);
                } else {
                    u32 v[8][CQ / 2];
                    typename Mma<T>::Frag h[2][NR];
                    if (LIKELY(whole))
                        outer_load<T, CQ, NR, true>(o, t, begin, end, p.q.rows, col, cols, v, h);
                    else
                        outer_load<T, CQ, NR, false>(o, t, begin, end, p.q.rows, col, cols, v, h);
                    outer_add<T, CQ, NR>(v, h, acc);
                }
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
    u32 u = 0;
    for (; u + 4 <= o.chunks; u += 4, from += 4 * apart) {      // four chunks' loads under way at a time
        float f[4][8];
#pragma unroll
        for (int k = 0; k < 4; k++)
#pragma unroll
            for (int e = 0; e < 8; e++) f[k][e] = from[k * apart + (u64)e * o.cols];
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] += (f[0][e] + f[1][e]) + (f[2][e] + f[3][e]);
    }
    for (; u < o.chunks; u++, from += apart)
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

// Tiles of 16 * tile16 rows that a batch can have.
u64 tiles_of(const vms_lowrank_args *a, u32 tile16)
{
    const u64 size = tile16 * 16, requests = a->n_requests;
    const u64 tiles = a->d_starts ? a->rows / size + requests + 2 : (a->rows + size - 1) / size;
    return tiles < a->rows ? tiles : a->rows;
}

const u32 DOWN_WAVES = 8;       // of a workgroup; twice that where the rank leaves the registers

// Rows of a tile of `down`, in sixteens: no more than a request has on average, so that single tokens do not pay for rows that
// are not there; at most four, two or one as the rank leaves registers; and half as many as long as there are then still no more
// tiles than compute units: larger tiles read the weights less often, but compute units without a tile read nothing, and a few
// tiles more than one for each take as long as two (24 requests of 6007 rows in all, 4096 -> 4096: rank 64 46 us forward with
// tiles of 32 rows, 54 with 16; rank 32 40 and 42).
u32 tile_of(const vms_lowrank_args *a)
{
    const u64 requests = a->d_starts ? a->n_requests : 1, each = requests ? a->rows / requests : a->rows;
    u32 t = each >= 48 ? 4 : each >= 24 ? 2 : 1;
    t = a->rank > 64 ? 1 : a->rank > 32 && t > 2 ? 2 : t;
    while (t > 1 && tiles_of(a, t / 2) <= OPS_CUS) t /= 2;
    return t;
}

struct Cut {
    u32 tile16, tiles, splits;  // tile16 8: the kernel with shared weights
    bool folded;                // the parts are put together before they are read
};

Cut cut_of(const vms_lowrank_args *a, u64 in)
{
    Cut c;
    const u64 requests = a->d_starts ? a->n_requests : 1, each = requests ? a->rows / requests : a->rows;
    // Shared weights save reads from the caches, as many as there are steps and ranks, and cost a launch: 8192 rows at rank 64
    // take 71 us with them and 82 without over 16384 columns, 26 and 23 over 4096; at rank 128 and 4096 columns the whole
    // step of 8192 rows 225 and 230 us.
    const bool shared = a->rank > 32 && in * padded_rank(a->rank) >= 1u << 19 && each >= 128 && a->rows >= 2048;
    c.tile16 = shared ? 8 : tile_of(a);
    const u64 tiles = tiles_of(a, c.tile16), slabs = in * type_bytes(a->dtype) / SLAB_BYTES;
    c.tiles = tiles ? (u32)tiles : 1;
    // A workgroup for each compute unit, but a slab at least for a wavefront.  Parts that `up` reads, again for each of its
    // panels, pay only with few tiles.  The kernel with shared weights, of few large tiles, always puts its parts together;
    // for the others that does not pay (2560 rows of 8192 in 32 bits, 160 tiles: 29 us whole, 31 and 5 in two parts).
    const u64 most = slabs / (shared ? 2 : DOWN_WAVES);
    u64 s = shared || c.tiles < OPS_CUS / 4 ? (OPS_CUS + c.tiles - 1) / c.tiles : 1;
    if (s > most) s = most;
    if (s > (shared ? 8 : 16)) s = shared ? 8 : 16;
    c.folded = s > 1 && shared;
    c.splits = s ? (u32)s : 1;
    return c;
}

// Requests of one token or two, of ranks that fill whole chunks, a power of two of them: the kernels without matrix units
bool few_of(const vms_lowrank_args *a)
{
    const u64 requests = a->d_starts ? a->n_requests : 1, each = requests ? a->rows / requests : a->rows;
    const u32 epl = 16 / type_bytes(a->dtype), chunks = a->rank / epl;
    return each <= 2 && a->rank % epl == 0 && chunks <= 16 && (chunks & (chunks - 1)) == 0;
}

// tiles of FEW_ROWS rows that a batch can have
u64 few_tiles(const vms_lowrank_args *a)
{
    const u64 tiles = a->d_starts ? a->rows / FEW_ROWS + a->n_requests + 2 : (a->rows + FEW_ROWS - 1) / FEW_ROWS;
    return tiles < a->rows ? tiles : a->rows;
}

// Both products in one launch?  Where a workgroup has not too much of `in` to sum, again for each of a request's panels, and
// every workgroup a place at once.  In 16 bits, 4096 -> 16384 at rank 16: 6.3 us for a token, 8.6 in two launches; 15.6 and 18.4
// for 96 tokens, 38 and 64 for 500; 2048 -> 4096 at rank 64 8.0 and 8.0 for a token.  In 32 bits the matrix instructions of a
// tile of one row take four times as long: 512 -> 2048 at rank 16 5.9 and 8.1 us, but 4096 -> 4096 12 and 9.6.
bool one_launch(const vms_lowrank_args *a)
{
    return few_of(a) && few_tiles(a) <= OPS_CUS * 2 && padded_rank(a->rank) * a->in * type_bytes(a->dtype) <= (a->dtype == VMS_F32 ? 1u << 16 : 1u << 18);
}

// how the hidden values of the forward pass are made
Cut forward_cut(const vms_lowrank_args *a)
{
    Cut c = cut_of(a, a->in);
    if (one_launch(a)) {
        c.splits = 1;
        c.folded = false;
    }
    return c;
}

// bytes of one layout with its planes
size_t laid_out(const vms_lowrank_args *a) { return (a->rows + 15) / 16 * 16 * padded_rank(a->rank) * (a->dtype == VMS_F32 ? 4 : 2 * 2); }

size_t parts_bytes(const vms_lowrank_args *a, const Cut &c) { return c.splits > 1 ? (size_t)c.splits * a->rows * padded_rank(a->rank) * 4 : 0; }

size_t hidden_bytes(const vms_lowrank_args *a, const Cut &c) { return (c.splits == 1 || c.folded ? 2 * laid_out(a) : 0) + parts_bytes(a, c); }

Hidden hidden_at(const vms_lowrank_args *a, const Cut &c, void *at)
{
    const u32 padded = padded_rank(a->rank);
    char *const p = (char *)at;
    if (c.splits == 1) return Hidden{ p, p + laid_out(a), nullptr, 1, padded, false };
    if (c.folded) return Hidden{ p, p + laid_out(a), (float *)(p + 2 * laid_out(a)), c.splits, padded, true };
    return Hidden{ nullptr, nullptr, (float *)p, c.splits, padded, false };
}

int check(const vms_lowrank_args *a)
{
    if (!a) return VMS_EINVAL;
    if (a->struct_size != sizeof *a) return VMS_ESTRUCT;
    if (a->dtype > VMS_BF16 || a->rows >> 28 || !a->in || a->in >> 22 || !a->out || a->out >> 22) return VMS_EINVAL;
    if (!a->rank || a->rank > VMS_LOWRANK_MAX_RANK || !a->n_adapters || a->n_adapters > 65535) return VMS_EINVAL;
    if (a->d_starts && a->n_requests >> 16) return VMS_EINVAL;       // (every workgroup looks through them)
    return VMS_OK;
}

// places inside a tile of 128 rows are counted in 32 bits
bool near_ok(u64 ld) { return ld < 1u << 23; }

// How `up` cuts a batch: tiles of 16 * tile16 rows (0: FEW_ROWS, the kernel for single tokens), panels of `trips` trips.
struct UpCut {
    u32 tile16, tiles, trips, panels;
    u64 groups;             // workgroups
};

UpCut up_cut(const vms_lowrank_args *a, u64 cols, bool base)
{
    UpCut c;
    const u64 requests = a->d_starts ? a->n_requests : 1, each = requests ? a->rows / requests : a->rows;
    const bool few = few_of(a);
    c.tile16 = few ? 0 : each >= 512 && a->rank <= 64 && base ? 8 : each >= 48 ? 4 : 1;
    const u64 tiles = few ? few_tiles(a) : tiles_of(a, c.tile16);
    c.tiles = (u32)tiles;
    const u64 trip = few ? 256 : (c.tile16 == 1 ? 4 : 1) * (SLAB_BYTES / type_bytes(a->dtype)), all = (cols + trip - 1) / trip;
    // Workgroups enough for four on every compute unit before one takes a second trip; no more than that where each has to
    // find its request first (24 requests, 6007 rows, 4096 -> 4096, rank 64: 46 us forward, 49 with as many again; one token each of
    // 96 requests, 4096 -> 16384, rank 16: 12 us, 16 with three times as many).
    u64 trips = (all * tiles + (a->d_starts || few ? OPS_CUS * 4 - 1 : 0)) / (OPS_CUS * 4);
    trips = trips < 1 ? 1 : trips > 8 ? 8 : trips;
    c.trips = (u32)trips;
    c.panels = (u32)((all + trips - 1) / trips);
    c.groups = tiles * c.panels;
    return c;
}

// a launch has fewer than 2^32 lanes: of `up` 256 in a workgroup, of `down` 512 (1024 where tiles are few)
bool grid_ok(const UpCut &c) { return c.groups < 1u << 24; }
bool grid_ok(const Cut &c) { return c.tiles < 1u << 23; }

int check_inputs(const vms_lowrank_args *a)
{
    if (!input_ok(a->d_a, a->dtype) || !input_ok(a->d_b, a->dtype)) return VMS_EINVAL;
    if (a->rows && (!input_ok(a->d_x, a->dtype) || !near_ok(a->ldx))) return VMS_EINVAL;
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
    const dim3 grid(tiles, p.h.splits), block(DOWN_WAVES * 64), twice(DOWN_WAVES * 128);
    switch (p.h.padded) {
    case 16: return MR == 4 ? ops_launch(lowrank_down_kernel<T, 4, 1, DOWN_WAVES>, grid, block, 0, p, stream)
                            : ops_launch(lowrank_down_kernel<T, MR == 4 ? 2 : MR, 1, DOWN_WAVES * 2>, grid, twice, 0, p, stream);
    case 32: return MR == 4 ? ops_launch(lowrank_down_kernel<T, 4, 2, DOWN_WAVES>, grid, block, 0, p, stream)
                            : ops_launch(lowrank_down_kernel<T, MR == 4 ? 2 : MR, 2, DOWN_WAVES * 2>, grid, twice, 0, p, stream);
    case 64: return ops_launch(lowrank_down_kernel<T, MR == 4 ? 2 : MR, 4, DOWN_WAVES>, grid, block, 0, p, stream);
    }
    return ops_launch(lowrank_down_kernel<T, 1, 8, DOWN_WAVES>, grid, block, 0, p, stream);
}

template <class T>
int fold(const FoldParams &p, void *stream)
{
    const u32 lanes = (p.rows + 3) / 4 * (p.h[0].padded / 4);
    return ops_launch(lowrank_fold_kernel<T>, dim3((lanes + 63) / 64, 1, 2), dim3(64), 0, p, stream);
}

// The hidden values, whole or in parts that `up` reads; in the order that the products over `in` leave them.
template <class T>
int down(const vms_lowrank_args *a, const Cut &c, const void *x, u64 ldx, const void *w, u64 in, Hidden *h, void *stream)
{
    const DownParams p = { x, w, *h, a->d_scales, requests_of(a), ldx, a->scale, (u32)in, a->rank };
    const dim3 grid(c.tiles, c.splits), block(512);
    int rc;
    switch (c.tile16) {
    case 1: rc = launch_down<T, 1>(p, c.tiles, stream); break;
    case 2: rc = launch_down<T, 2>(p, c.tiles, stream); break;
    case 4: rc = launch_down<T, 4>(p, c.tiles, stream); break;
    default:
        rc = h->padded == 64 ? ops_launch(lowrank_down_shared_kernel<T, 4>, grid, block, 0, p, stream)
                             : ops_launch(lowrank_down_shared_kernel<T, 8>, grid, block, 0, p, stream);
    }
    if (rc || !h->folded) return rc;
    const FoldParams f = { { *h, *h }, { true, false }, { true, false }, (u32)a->rows };
    rc = fold<T>(f, stream);
    h->parts = nullptr;
    return rc;
}

template <class T>
int one(const vms_lowrank_args *a, const Hidden &h, void *stream)
{
    OneParams p = { { a->d_x, a->d_a, h, a->d_scales, requests_of(a), a->ldx, a->scale, (u32)a->in, a->rank },
                    { h, a->d_b, a->d_y, a->d_out, requests_of(a), a->ldy, a->ldo, (u32)a->out, a->rank, 1, 1 } };
    const u32 tiles = (u32)few_tiles(a), all = (u32)((a->out + ONE_WAVES * 64 - 1) / (ONE_WAVES * 64));
    // Panels of columns: a workgroup for each compute unit, two where that leaves four trips for each (32 tokens, 4096 -> 16384
    // at rank 16: 9.1 us with eight panels of four trips, 11.2 with 16 of two).
    u32 panels = min(all / 4, OPS_CUS * 2 / tiles);
    panels = max(max(panels, OPS_CUS / tiles), 1u);
    p.u.trips = (all + panels - 1) / panels;
    p.u.panels = (all + p.u.trips - 1) / p.u.trips;
    const dim3 grid(tiles * p.u.panels), block(ONE_WAVES * 64);
    switch (a->rank / Mma<T>::EPL) {
    case 1: return ops_launch(lowrank_one_kernel<T, 1>, grid, block, 0, p, stream);
    case 2: return ops_launch(lowrank_one_kernel<T, 2>, grid, block, 0, p, stream);
    case 4: return ops_launch(lowrank_one_kernel<T, 4>, grid, block, 0, p, stream);
    case 8: return ops_launch(lowrank_one_kernel<T, 8>, grid, block, 0, p, stream);
    }
    return ops_launch(lowrank_one_kernel<T, 16>, grid, block, 0, p, stream);
}

template <class T, int MR, int WR, bool ONCE = false>
int launch_up(const UpParams &p, u32 grid, void *stream)
{
    const dim3 block(256);
    const int per = Mma<T>::STEP;
    switch (p.h.padded) {
    case 16: return ops_launch(lowrank_up_kernel<T, MR, 1, WR, ONCE>, dim3(grid), block, 0, p, stream);
    case 32: return ops_launch(lowrank_up_kernel<T, MR, 32 / per, WR, ONCE>, dim3(grid), block, 0, p, stream);
    case 64: return ops_launch(lowrank_up_kernel<T, MR, 64 / per, WR, ONCE>, dim3(grid), block, 0, p, stream);
    }
    return ops_launch(lowrank_up_kernel<T, 1, 128 / per, WR, ONCE>, dim3(grid), block, 0, p, stream);
}

template <class T>
int up(const vms_lowrank_args *a, const Hidden &h, const void *w, const void *base, u64 ldb, void *out, u64 ldo, u64 cols, void *stream)
{
    const UpCut c = up_cut(a, cols, base != nullptr);
    const UpParams p = { h, w, base, out, requests_of(a), ldb, ldo, (u32)cols, a->rank, c.trips, c.panels };
    const u32 grid = (u32)c.groups;
    const bool once = passes_by(a->rows * cols * sizeof(T) * (base ? 2 : 1));
    switch (c.tile16) {
    case 1: return launch_up<T, 1, 1>(p, grid, stream);
    case 4: return once ? launch_up<T, 1, 4, true>(p, grid, stream) : launch_up<T, 1, 4>(p, grid, stream);
    case 8: return once ? launch_up<T, 2, 4, true>(p, grid, stream) : launch_up<T, 2, 4>(p, grid, stream);
    }
    const dim3 blocks(grid), block(256);
    switch (a->rank / Mma<T>::EPL) {
    case 1: return ops_launch(lowrank_up_few_kernel<T, 1>, blocks, block, 0, p, stream);
    case 2: return ops_launch(lowrank_up_few_kernel<T, 2>, blocks, block, 0, p, stream);
    case 4: return ops_launch(lowrank_up_few_kernel<T, 4>, blocks, block, 0, p, stream);
    case 8: return ops_launch(lowrank_up_few_kernel<T, 8>, blocks, block, 0, p, stream);
    }
    return ops_launch(lowrank_up_few_kernel<T, 16>, blocks, block, 0, p, stream);
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
    Cut forward, back;          // of the products over `in` and over `out`
};

bool wants_hidden_gradient(const vms_lowrank_backward_args *a) { return a->d_dx || a->d_da; }

Layout layout_of(const vms_lowrank_backward_args *a)
{
    const vms_lowrank_args &f = a->f;
    const size_t e = type_bytes(f.dtype), padded = padded_rank(f.rank);
    Layout l = {};
    size_t end = 0;
    const auto place = [&end](size_t *at, size_t bytes) {
        *at = end;
        end += (bytes + 255) & ~(size_t)255;
    };
    l.forward = forward_cut(&f);
    l.back = cut_of(&f, f.out);
    place(&l.at, a->d_dx ? (size_t)f.n_adapters * f.rank * f.in * e : 0);
    place(&l.bt, wants_hidden_gradient(a) ? (size_t)f.n_adapters * f.rank * f.out * e : 0);
    place(&l.dhidden, wants_hidden_gradient(a) ? hidden_bytes(&f, l.back) : 0);
    place(&l.hfold, a->d_db && l.forward.splits > 1 ? laid_out(&f) : 0);
    place(&l.dfold, a->d_da && l.back.splits > 1 ? laid_out(&f) : 0);
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
    const Layout l = layout_of(a);
    char *const ws = (char *)a->d_workspace;
    Hidden h = hidden_at(&f, l.forward, f.d_hidden), dh = hidden_at(&f, l.back, ws + l.dhidden);
    if (h.folded) h.parts = nullptr;            // the forward pass has put them together
    int rc = VMS_OK;
    if (wants_hidden_gradient(a)) {
        const auto blocks = [](u64 r, u64 k) { return (u32)((r + 31) / 32 * ((k + 31) / 32)); };
        SwapParams s = { { { f.d_b, ws + l.bt, (u32)f.out, f.rank, blocks(f.out, f.rank) }, { f.d_a, ws + l.at, f.rank, (u32)f.in, 0 } } };
        if (a->d_dx) s.job[1].blocks = blocks(f.rank, f.in);
        rc = ops_launch(lowrank_swap_kernel<T>, dim3(s.job[0].blocks + s.job[1].blocks, f.n_adapters), dim3(256), 0, s, stream);
        if (!rc) rc = down<T>(&f, l.back, a->d_dout, a->lddout, ws + l.bt, f.out, &dh, stream);
    }
    const auto dx = [&] { return a->d_dx ? up<T>(&f, dh, ws + l.at, nullptr, 0, a->d_dx, a->lddx, f.in, stream) : VMS_OK; };
    if (rc) return rc;
    if (!(a->d_da || a->d_db)) return dx();
    FoldParams some = { { h, dh }, {}, { a->d_db && h.parts, a->d_da && dh.parts }, (u32)f.rows };
    if (some.outer[0]) h.outer = some.h[0].outer = ws + l.hfold;
    if (some.outer[1]) dh.outer = some.h[1].outer = ws + l.dfold;
    if (some.outer[0] || some.outer[1]) {
        rc = fold<T>(some, stream);
        if (rc) return rc;
    }
    OuterParams o = { { l.db, l.da }, requests_of(&f) };
    o.job[0].v = a->d_dout;
    o.job[0].ldv = a->lddout;
    o.job[0].hidden = h.outer;
    o.job[0].sums = (float *)(ws + l.dbsums);
    o.job[1].v = f.d_x;
    o.job[1].ldv = f.ldx;
    o.job[1].hidden = dh.outer;
    o.job[1].sums = (float *)(ws + l.dasums);
    JoinParams j = { { { o.job[0].sums, a->d_db, (u32)f.out, l.db.chunks, 1 }, { o.job[1].sums, a->d_da, (u32)f.in, l.da.chunks, 0 } },
                     f.rank, padded, (u32)((f.out + 255) / 256) };
    u32 blocks = (u32)((f.in + 255) / 256);
    if (!a->d_db) o.job[0].chunks = j.first_blocks = 0;
    if (!a->d_da) o.job[1].chunks = blocks = 0;
    const u32 grid = o.job[0].panels * o.job[0].chunks + o.job[1].panels * o.job[1].chunks;
    rc = launch_outer<T>(o, padded, dim3(grid, f.n_adapters), stream);
    if (!rc) rc = dx();
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
    return hidden_bytes(a, forward_cut(a));
}

extern "C" int vms_lowrank(const vms_lowrank_args *a, void *stream)
{
    int rc = check(a);
    if (rc) return rc;
    if (!a->rows) return VMS_OK;
    rc = check_inputs(a);
    if (rc) return rc;
    if (!input_ok(a->d_y, a->dtype) || !near_ok(a->ldy) || !output_ok(a->d_out, a->dtype, a->ldo, a->out) || !near_ok(a->ldo)) return VMS_EINVAL;
    if (a->d_y == a->d_out && a->ldy != a->ldo) return VMS_EINVAL;
    if (!grid_ok(up_cut(a, a->out, true))) return VMS_EINVAL;
    const Cut c = forward_cut(a);
    if (!grid_ok(c)) return VMS_EINVAL;
    Hidden h = hidden_at(a, c, a->d_hidden);
    return with_type(a->dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        if (one_launch(a)) return one<T>(a, h, stream);
        const int r = down<T>(a, c, a->d_x, a->ldx, a->d_a, a->in, &h, stream);
        return r ? r : up<T>(a, h, a->d_b, a->d_y, a->ldy, a->d_out, a->ldo, a->out, stream);
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
    if (!input_ok(a->d_dout, f.dtype) || !near_ok(a->lddout)) return VMS_EINVAL;
    if (a->d_dx && (!output_ok(a->d_dx, f.dtype, a->lddx, f.in) || !near_ok(a->lddx))) return VMS_EINVAL;
    if (!a->d_dx && !a->d_da && !a->d_db) return VMS_OK;
    if (a->d_dx && !grid_ok(up_cut(&f, f.in, false))) return VMS_EINVAL;
    if (!grid_ok(cut_of(&f, f.out))) return VMS_EINVAL;
    if (!a->d_workspace || (uintptr_t)a->d_workspace % 16 || a->workspace_bytes < layout_of(a).total) return VMS_EWORKSPACE;
    return with_type(f.dtype, [&](auto *t) { return backward<std::remove_pointer_t<decltype(t)>>(a, stream); });
}
