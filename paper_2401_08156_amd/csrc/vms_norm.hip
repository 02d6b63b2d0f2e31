// vms_layernorm and vms_layernorm_backward (include/vms_ops.h).
//
// Both passes are bound by memory: a row is read once, kept in registers (group g of eight columns in
// lane g mod LANES of those that share the row) and written once.  Mean and variance are taken in one
// go without the cancellation of a difference of squares: every wavefront takes the mean of its part
// and the squares around that, and the parts are joined by
//     M2 = sum M2_w + sum n_w (mean_w - mean)^2.
#include "ops_common.hpp"

namespace {

struct NormParams {
    const void *x, *residual, *weight, *bias;
    void *y, *s;
    float *stats;
    u64 ldx, ldr, ldy, lds;
    u32 rows, cols, groups;         // groups of eight columns
    float eps;
    Mask mask;
};

struct NormBackParams {
    const void *dy, *ds, *s, *weight;
    const float *stats;
    void *dres, *dx;
    float *partial;                 // [workgroups][2][cols]: sums for dweight and dbias
    u64 lddy, ldds, lds, lddres, lddx;
    u32 rows, cols, groups;
    Mask mask;
};

struct NormJoinParams {
    const float *partial;
    void *dweight, *dbias;
    u32 parts, cols;
};

// The sum over a workgroup's lanes, through `part`, which two uses in a row must not share (the barrier between them lies in
// front of the second's reads).
DI float group_sum(float v, float *part)
{
    v = wave_sum(v);
    if (lane_id() == 0) part[wave_of_group()] = v;
    __syncthreads();
    const u32 k = threadIdx.x & 15;
    return row16_sum(k < blockDim.x / 64 ? part[k] : 0.f);
}

// s of eight columns: x, or residual + dropout(x)
template <class T, bool ONCE>
DI void norm_input(const NormParams &p, u64 seed, u32 row, u32 group, float v[8])
{
    const u32 col = group * 8, n = p.cols - col;
    load8<ONCE>((const T *)p.x + row * p.ldx + col, n, v);
    if (p.residual) {
        float r[8];
        load8<ONCE>((const T *)p.residual + row * p.ldr + col, n, r);
        if (p.mask.limit) drop8(p.mask, seed, row, group, v);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] += r[i];
    }
}

// y, and s where it is wanted, of eight columns; w and b: those of weight and bias
template <class T, bool ONCE>
DI void norm_output(const NormParams &p, u32 row, u32 group, const float v[8], const typename Eight<T>::type &w, const typename Eight<T>::type &b,
                    float mean, float rstd)
{
    const u32 col = group * 8, n = p.cols - col;
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; i++) {
        o[i] = (v[i] - mean) * rstd;
        if (p.weight) o[i] *= (float)w[i];
        if (p.bias) o[i] += (float)b[i];
    }
    store8<ONCE>((T *)p.y + row * p.ldy + col, n, o);
    if (p.s) store8<ONCE>((T *)p.s + row * p.lds + col, n, v);
}

// Sum and squares around the mean of a row's part in a wavefront; `mine` columns, the other places hold 0.
template <int NG>
DI void part_stats(const float v[NG][8], const u32 n[NG], u32 mine, float *sum, float *m2)
{
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int g = 0; g < NG; g++)
#pragma unroll
        for (int i = 0; i < 8; i++) a += v[g][i];
    a = wave_sum(a);
    const float mean = mine ? a / (float)mine : 0.f;
#pragma unroll
    for (int g = 0; g < NG; g++) {
        if (LIKELY(n[g] >= 8)) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float d = v[g][i] - mean;
                b += d * d;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float d = v[g][i] - mean;
                if ((u32)i < n[g]) b += d * d;
            }
        }
    }
    *sum = a;
    *m2 = wave_sum(b);
}

// mean and 1 / sqrt(variance + eps) of a row from its parts, one in each lane of 16
DI void join_stats(float sum, float m2, float n, u32 cols, float eps, float *mean, float *rstd)
{
    *mean = row16_sum(sum) / (float)cols;
    const float d = n > 0.f ? sum / n - *mean : 0.f;
    *rstd = 1.f / sqrtf(row16_sum(m2 + n * d * d) / (float)cols + eps);
}

// A row in the registers of a workgroup, NG groups a lane; SINGLE: of a wavefront, four rows a workgroup.
//
// y goes by the sum s as it is in 32 bits.  The statistics for the backward pass are those of s rounded to the type,
// which is what that pass reads: with the others a row of small variance, whose rstd is large, would get a gradient of
// rounding errors, (s rounded - mean) * rstd.
template <class T, bool SINGLE, int NG, bool ONCE>
__global__ __launch_bounds__(SINGLE ? 256 : 1024) void norm_kernel(const NormParams p)
{
    __shared__ float parts[2][5][16];
    const u32 lanes = SINGLE ? 64 : blockDim.x, lane = SINGLE ? lane_id() : threadIdx.x, wave = wave_of_group(), waves = lanes / 64;
    const u32 step = SINGLE ? gridDim.x * 4 : gridDim.x;
    const bool rounded = sizeof(T) == 2 && p.s && p.stats;
    u32 odd = 0;
    const u64 seed = p.mask.limit ? mask_seed(p.mask) : 0;
    u32 n[NG], mine = 0;            // columns of a lane's groups, and of all groups of this wavefront
#pragma unroll
    for (int g = 0; g < NG; g++) {
        const u32 col = (g * lanes + lane) * 8, at = (g * lanes + (SINGLE ? 0 : wave * 64)) * 8;
        n[g] = p.cols > col ? p.cols - col : 0;
        mine += p.cols > at ? min(p.cols - at, 512u) : 0u;
    }
    typedef typename Eight<T>::type Raw;
    for (u32 row = SINGLE ? blockIdx.x * 4 + wave : blockIdx.x; row < p.rows; row += step) {
        // What the row needs is on its way before the first of it is waited for, the weights too where registers hold them
        // (4099 x 5120 in 16 bits: 25 us, 28 with each load waited for before the next).
        const bool AHEAD = NG < 4, WEIGHTS_AHEAD = AHEAD && NG * sizeof(T) <= 8;
        Raw x[NG], r[NG], w[NG], b[NG];
        const auto fetch = [&](int g) {
            const u32 col = (g * lanes + lane) * 8;
            x[g] = r[g] = Raw{};
            if (!n[g]) return;
            x[g] = load8_raw<ONCE>((const T *)p.x + row * p.ldx + col, n[g]);
            if (p.residual) r[g] = load8_raw<ONCE>((const T *)p.residual + row * p.ldr + col, n[g]);
        };
        const auto fetch_weights = [&](int g) {
            const u32 col = (g * lanes + lane) * 8;
            w[g] = b[g] = Raw{};
            if (!n[g]) return;
            if (p.weight) w[g] = load8_raw((const T *)p.weight + col, n[g]);
            if (p.bias) b[g] = load8_raw((const T *)p.bias + col, n[g]);
        };
#pragma unroll
        for (int g = 0; g < NG; g++)
            if (AHEAD) fetch(g);
#pragma unroll
        for (int g = 0; g < NG; g++)
            if (WEIGHTS_AHEAD) fetch_weights(g);
        float v[NG][8];
#pragma unroll
        for (int g = 0; g < NG; g++) {
            if (!AHEAD) fetch(g);
#pragma unroll
            for (int i = 0; i < 8; i++) v[g][i] = (float)x[g][i];
            if (p.mask.limit) drop8(p.mask, seed, row, g * lanes + lane, v[g]);
            if (p.residual) {
#pragma unroll
                for (int i = 0; i < 8; i++) v[g][i] += (float)r[g][i];
            }
        }
        float sum, m2, sum2 = 0.f, m22 = 0.f;
        part_stats<NG>(v, n, mine, &sum, &m2);
        if (rounded) {
            float as_stored[NG][8];
#pragma unroll
            for (int g = 0; g < NG; g++)
#pragma unroll
                for (int i = 0; i < 8; i++) as_stored[g][i] = (float)(T)v[g][i];
            part_stats<NG>(as_stored, n, mine, &sum2, &m22);
        }
        float count = (float)mine;
        if (SINGLE) {               // one part
            const bool one = (lane & 15) == 0;
            sum = one ? sum : 0.f;
            m2 = one ? m2 : 0.f;
            sum2 = one ? sum2 : 0.f;
            m22 = one ? m22 : 0.f;
            count = one ? count : 0.f;
        } else {
            float(&part)[5][16] = parts[odd];       // two places in turn: a wavefront may be one row ahead, not two
            odd ^= 1;
            if (lane_id() == 0) {
                part[0][wave] = sum;
                part[1][wave] = m2;
                part[2][wave] = count;
                part[3][wave] = sum2;
                part[4][wave] = m22;
            }
            __syncthreads();
            const u32 w = lane & 15;
            sum = w < waves ? part[0][w] : 0.f;
            m2 = w < waves ? part[1][w] : 0.f;
            count = w < waves ? part[2][w] : 0.f;
            sum2 = w < waves ? part[3][w] : 0.f;
            m22 = w < waves ? part[4][w] : 0.f;
        }
        float mean, rstd;
        join_stats(sum, m2, count, p.cols, p.eps, &mean, &rstd);
        if (p.stats) {
            float mean2 = mean, rstd2 = rstd;
            if (rounded) join_stats(sum2, m22, count, p.cols, p.eps, &mean2, &rstd2);
            if (lane == 0) {
                p.stats[(u64)row * 2] = mean2;
                p.stats[(u64)row * 2 + 1] = rstd2;
            }
        }
#pragma unroll
        for (int g = 0; g < NG; g++) {
            if (!WEIGHTS_AHEAD) fetch_weights(g);
            if (n[g]) norm_output<T, ONCE>(p, row, g * lanes + lane, v[g], w[g], b[g], mean, rstd);
        }
    }
}

// Rows that no workgroup's registers hold: read three times, the second and third time from a cache near by.
template <class T>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormParams p)
{
    __shared__ float part[4][16];
    const u64 seed = p.mask.limit ? mask_seed(p.mask) : 0;
    const bool rounded = sizeof(T) == 2 && p.s && p.stats;
    for (u32 row = blockIdx.x; row < p.rows; row += gridDim.x) {
        float mean[2] = {}, m2[2] = {}, v[8];
#pragma unroll
        for (int pass = 0; pass < 2; pass++) {
            float acc[2] = {};
            for (u32 group = threadIdx.x; group < p.groups; group += 1024) {
                norm_input<T, false>(p, seed, row, group, v);
                const u32 n = p.cols - group * 8;
                float one[2] = {};              // sums of sums: the rounding errors of a long row stay small
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    const float d = v[i] - mean[0], e = (float)(T)v[i] - mean[1];
                    if ((u32)i < n) {
                        one[0] += pass ? d * d : d;
                        one[1] += pass ? e * e : e;
                    }
                }
                acc[0] += one[0];
                acc[1] += one[1];
            }
            float *const to = pass ? m2 : mean;
            to[0] = group_sum(acc[0], part[pass * 2]) / (float)p.cols;
            to[1] = group_sum(acc[1], part[pass * 2 + 1]) / (float)p.cols;
        }
        const float rstd = 1.f / sqrtf(m2[0] + p.eps);
        if (p.stats && threadIdx.x == 0) {
            p.stats[(u64)row * 2] = mean[rounded];
            p.stats[(u64)row * 2 + 1] = 1.f / sqrtf(m2[rounded] + p.eps);
        }
        for (u32 group = threadIdx.x; group < p.groups; group += 1024) {
            const u32 col = group * 8, n = p.cols - col;
            typename Eight<T>::type w = {}, b = {};
            if (p.weight) w = load8_raw((const T *)p.weight + col, n);
            if (p.bias) b = load8_raw((const T *)p.bias + col, n);
            norm_input<T, false>(p, seed, row, group, v);
            norm_output<T, false>(p, row, group, v, w, b, mean[0], rstd);
        }
    }
}

// What the gradient needs of eight columns: dy, the normalised input, and dy * weight
template <class T>
DI void back_input(const NormBackParams &p, u32 row, u32 group, float mean, float rstd, float dy[8], float h[8])
{
    const u32 col = group * 8, n = p.cols - col;
    load8((const T *)p.dy + row * p.lddy + col, n, dy);
    load8((const T *)p.s + row * p.lds + col, n, h);
#pragma unroll
    for (int i = 0; i < 8; i++) h[i] = (u32)i < n ? (h[i] - mean) * rstd : 0.f;
}

template <class T>
DI void back_weight(const NormBackParams &p, u32 group, float w[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) w[i] = 1.f;
    if (p.weight) load8((const T *)p.weight + group * 8, p.cols - group * 8, w);
}

template <class T, bool ONCE>
DI void back_output(const NormBackParams &p, u64 seed, u32 row, u32 group, const float dy[8], const float h[8], const float w[8],
                    const typename Eight<T>::type &ds, float rstd, float c1, float c2)
{
    const u32 col = group * 8, n = p.cols - col;
    float o[8];
#pragma unroll
    for (int i = 0; i < 8; i++) o[i] = rstd * (dy[i] * w[i] - c1 - h[i] * c2);
    if (p.ds) {
#pragma unroll
        for (int i = 0; i < 8; i++) o[i] += (float)ds[i];
    }
    store8<ONCE>((T *)p.dres + row * p.lddres + col, n, o);
    if (p.dx) {
        if (p.mask.limit) drop8(p.mask, seed, row, group, o);
        store8<ONCE>((T *)p.dx + row * p.lddx + col, n, o);
    }
}

// A workgroup takes every gridDim.x-th row (SINGLE: four rows at a time, a wavefront each) and keeps the sums for the weights'
// gradients in registers until its last row.
template <class T, bool SINGLE, int NG, bool WEIGHTS, bool ONCE>
__global__ __launch_bounds__(SINGLE ? 256 : 1024) void norm_back_kernel(const NormBackParams p)
{
    __shared__ float part[2][2][16];
    __shared__ float joined[SINGLE && WEIGHTS ? 4 * 64 * 8 : 1];
    const u32 lanes = SINGLE ? 64 : blockDim.x, lane = SINGLE ? lane_id() : threadIdx.x, waves = lanes / 64;
    const u32 first = SINGLE ? blockIdx.x * 4 + wave_of_group() : blockIdx.x;
    const u32 step = SINGLE ? gridDim.x * 4 : gridDim.x;
    const u64 seed = p.mask.limit ? mask_seed(p.mask) : 0;
    float w[NG][8], dw[WEIGHTS ? NG : 1][8], db[WEIGHTS ? NG : 1][8];
#pragma unroll
    for (int g = 0; g < NG; g++) {
        const u32 group = g * lanes + lane;
        if (group < p.groups) back_weight<T>(p, group, w[g]);
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (WEIGHTS) dw[g][i] = db[g][i] = 0.f;
    }
    // With one group a lane, what a row's gradient is made of is read while the row before it is worked on (131 us for 16384 x
    // 4096 in 16 bits with residual and dropout, 141 without); the registers do not hold two rows of two.
    const bool AHEAD = NG == 1;
    typedef typename Eight<T>::type Raw;
    Raw dy2 = {}, s2 = {}, ds2 = {};
    const auto fetch = [&](u32 row) {
        const u32 col = lane * 8, n = p.cols - col;
        if (lane >= p.groups) return;
        dy2 = load8_raw<ONCE>((const T *)p.dy + row * p.lddy + col, n);
        s2 = load8_raw<ONCE>((const T *)p.s + row * p.lds + col, n);
        if (p.ds) ds2 = load8_raw<ONCE>((const T *)p.ds + row * p.ldds + col, n);
    };
    if (AHEAD && first < p.rows) fetch(first);
    u32 odd = 0;
    for (u32 row = first; row < p.rows; row += step) {
        const float mean = p.stats[(u64)row * 2], rstd = p.stats[(u64)row * 2 + 1];
        float dy[NG][8], h[NG][8];
        Raw ds = ds2;
        float c1 = 0.f, c2 = 0.f;
#pragma unroll
        for (int g = 0; g < NG; g++) {
            const u32 group = g * lanes + lane, col = group * 8, n = p.cols - col;
#pragma unroll
            for (int i = 0; i < 8; i++) dy[g][i] = h[g][i] = 0.f;
            if (group >= p.groups) continue;
            if (AHEAD) {
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    dy[g][i] = (float)dy2[i];
                    h[g][i] = (float)s2[i];
                }
            } else {
                load8<ONCE>((const T *)p.dy + row * p.lddy + col, n, dy[g]);
                load8<ONCE>((const T *)p.s + row * p.lds + col, n, h[g]);
            }
#pragma unroll
            for (int i = 0; i < 8; i++) {
                h[g][i] = (u32)i < n ? (h[g][i] - mean) * rstd : 0.f;
                const float e = dy[g][i] * w[g][i];
                c1 += e;
                c2 += e * h[g][i];
                if (WEIGHTS) {
                    dw[g][i] += dy[g][i] * h[g][i];
                    db[g][i] += dy[g][i];
                }
            }
        }
        if (AHEAD && row + step < p.rows) fetch(row + step);
        c1 = wave_sum(c1);
        c2 = wave_sum(c2);
        if (!SINGLE) {              // two places in turn: a wavefront may be one row ahead, not two
            if (lane_id() == 0) {
                part[odd][0][wave_of_group()] = c1;
                part[odd][1][wave_of_group()] = c2;
            }
            __syncthreads();
            const u32 k = lane & 15;
            c1 = row16_sum(k < waves ? part[odd][0][k] : 0.f);
            c2 = row16_sum(k < waves ? part[odd][1][k] : 0.f);
            odd ^= 1;
        }
        c1 /= (float)p.cols;
        c2 /= (float)p.cols;
#pragma unroll
        for (int g = 0; g < NG; g++) {
            const u32 group = g * lanes + lane;
            if (group >= p.groups) continue;
            if (!AHEAD && p.ds) ds = load8_raw<ONCE>((const T *)p.ds + row * p.ldds + group * 8, p.cols - group * 8);
            back_output<T, ONCE>(p, seed, row, group, dy[g], h[g], w[g], ds, rstd, c1, c2);
        }
    }
    if (WEIGHTS) {
        float *out = p.partial + (u64)blockIdx.x * 2 * p.cols;
#pragma unroll
        for (int g = 0; g < NG; g++) {
            const u32 group = g * lanes + lane;
#pragma unroll
            for (int k = 0; k < 2; k++) {
                float(&v)[8] = k ? db[g] : dw[g];
                if (SINGLE) {      // the four wavefronts' sums
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < 8; i++) joined[(wave_of_group() * 8 + i) * 64 + lane] = v[i];
                    __syncthreads();
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        v[i] = 0.f;
#pragma unroll
                        for (int u = 0; u < 4; u++) v[i] += joined[(u * 8 + i) * 64 + lane];
                    }
                    if (wave_of_group() != 0) continue;
                }
                if (group < p.groups) store8(out + (u64)k * p.cols + group * 8, p.cols - group * 8, v);
            }
        }
    }
}

// Rows that no workgroup's registers hold: two passes over dy and s, the weights' sums in the workgroup's place in memory,
// where each column belongs to one lane.
template <class T, bool WEIGHTS>
__global__ __launch_bounds__(1024) void norm_back_long_kernel(const NormBackParams p)
{
    __shared__ float part[4][16];
    const u64 seed = p.mask.limit ? mask_seed(p.mask) : 0;
    float *const dw = WEIGHTS ? p.partial + (u64)blockIdx.x * 2 * p.cols : nullptr;
    float dy[8], h[8], w[8];
    u32 odd = 0;
    bool begun = false;
    for (u32 row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const float mean = p.stats[(u64)row * 2], rstd = p.stats[(u64)row * 2 + 1];
        float c1 = 0.f, c2 = 0.f;
        for (u32 group = threadIdx.x; group < p.groups; group += 1024) {
            back_input<T>(p, row, group, mean, rstd, dy, h);
            back_weight<T>(p, group, w);
            float e1 = 0.f, e2 = 0.f;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                e1 += dy[i] * w[i];
                e2 += dy[i] * w[i] * h[i];
            }
            c1 += e1;
            c2 += e2;
            if (WEIGHTS) {
                const u32 n = p.cols - group * 8;
                float a[8] = {}, b[8] = {};
                if (begun) {
                    load8(dw + group * 8, n, a);
                    load8(dw + p.cols + group * 8, n, b);
                }
#pragma unroll
                for (int i = 0; i < 8; i++) {
                    a[i] += dy[i] * h[i];
                    b[i] += dy[i];
                }
                store8(dw + group * 8, n, a);
                store8(dw + p.cols + group * 8, n, b);
            }
        }
        begun = true;
        c1 = group_sum(c1, part[odd]) / (float)p.cols;
        c2 = group_sum(c2, part[odd + 1]) / (float)p.cols;
        odd ^= 2;
        for (u32 group = threadIdx.x; group < p.groups; group += 1024) {
            back_input<T>(p, row, group, mean, rstd, dy, h);
            back_weight<T>(p, group, w);
            typename Eight<T>::type ds = {};
            if (p.ds) ds = load8_raw((const T *)p.ds + row * p.ldds + group * 8, p.cols - group * 8);
            back_output<T, false>(p, seed, row, group, dy, h, w, ds, rstd, c1, c2);
        }
    }
}

// dweight and dbias from the workgroups' sums: 32 columns a workgroup, its 32 rows of lanes take every 32nd part
template <class T>
__global__ __launch_bounds__(1024) void norm_join_kernel(const NormJoinParams p)
{
    __shared__ float sums[32][33];
    const u32 x = threadIdx.x & 31, y = threadIdx.x >> 5, k = blockIdx.y;
    T *const out = (T *)(k ? p.dbias : p.dweight);
    if (!out) return;
    const u32 col = blockIdx.x * 32 + x;
    float v = 0.f;
    if (col < p.cols) {
        const float *from = p.partial + k * (u64)p.cols + col;
        const u64 apart = 2 * (u64)p.cols;
        u32 i = y;
        for (; i + 96 < p.parts; i += 128) {
            float f[4];
#pragma unroll
            for (int u = 0; u < 4; u++) f[u] = from[(i + 32 * u) * apart];
            v += (f[0] + f[1]) + (f[2] + f[3]);
        }
        for (; i < p.parts; i += 32) v += from[i * apart];
    }
    sums[y][x] = v;
    __syncthreads();
    if (y == 0 && col < p.cols) {
#pragma unroll
        for (int i = 1; i < 32; i++) v += sums[i][x];
        out[col] = (T)v;
    }
}

// Which registers hold a row.  Those of one wavefront up to 512 columns (1024 in 16 bits, two groups a lane), those of a
// workgroup beyond, none above 32768.  More than four wavefronts are a multiple of four, for the four units that they are
// spread over.  A lane takes one group up to 2048 columns (6144 in 32 bits), then two or three, as leaves fewer lanes without
// any: 4099 rows of 5120 columns in 16 bits take 24 us with four wavefronts of three groups a lane, 28 with five of two; in 32
// bits 42 with twelve of one, 45 with ten.
// A workgroup for each row: many of them at different stages keep the memory busier than ones that stay and read a row ahead,
// of which fewer fit (16384 x 4096 in 16 bits with residual and dropout take 113 us, 9 us more with such).
template <class T, bool ONCE>
int launch_norm(const NormParams &p, void *stream)
{
    const u32 g = p.groups, most = 1u << 18;      // workgroups; they go on to further rows
    const dim3 quarter(p.rows / 4 < most ? (p.rows + 3) / 4 : most), each(p.rows < most ? p.rows : most);
    const auto fours = [g](u32 groups) { return (g + 256 * groups - 1) / (256 * groups) * 4; };      // wavefronts
    const dim3 one((g <= 256 ? (g + 63) / 64 : fours(1)) * 64), two(fours(2) * 64), three(fours(3) * 64);
    if (g <= 64) return ops_launch(norm_kernel<T, true, 1, ONCE>, quarter, dim3(256), 0, p, stream);
    if constexpr (sizeof(T) == 2)
        if (g <= 128) return ops_launch(norm_kernel<T, true, 2, ONCE>, quarter, dim3(256), 0, p, stream);
    if (g <= (sizeof(T) == 2 ? 256 : 768)) return ops_launch(norm_kernel<T, false, 1, ONCE>, each, one, 0, p, stream);
    if (two.x <= 1024 && two.x * 2 <= three.x * 3) return ops_launch(norm_kernel<T, false, 2, ONCE>, each, two, 0, p, stream);
    if (three.x <= 1024) return ops_launch(norm_kernel<T, false, 3, ONCE>, each, three, 0, p, stream);
    if (g <= 4096) return ops_launch(norm_kernel<T, false, 4, ONCE>, each, dim3(1024), 0, p, stream);
    return ops_launch(norm_long_kernel<T>, each, dim3(1024), 0, p, stream);
}

template <class T, bool WEIGHTS, bool ONCE>
int launch_norm_back(const NormBackParams &p, u32 grid, void *stream)
{
    const u32 g = p.groups;
    if (g <= 64) return ops_launch(norm_back_kernel<T, true, 1, WEIGHTS, ONCE>, dim3(grid), dim3(256), 0, p, stream);
    if (g <= 1024) return ops_launch(norm_back_kernel<T, false, 1, WEIGHTS, ONCE>, dim3(grid), dim3((g + 63) / 64 * 64), 0, p, stream);
    if (g <= 2048) return ops_launch(norm_back_kernel<T, false, 2, WEIGHTS, ONCE>, dim3(grid), dim3((g + 127) / 128 * 64), 0, p, stream);
    return ops_launch(norm_back_long_kernel<T, WEIGHTS>, dim3(grid), dim3(1024), 0, p, stream);
}

bool wants_weights(const vms_layernorm_backward_args *a) { return a->d_dweight || a->d_dbias; }

// Workgroups of the backward pass, each with sums of its own to be joined: 16 wavefronts on a compute unit, 8 in 32 bits, whose
// loads are twice as large (4099 x 5120 in 16 bits: 42 us with 10 wavefronts, 46 with 20, 53 with 40; 2816 x 2048 in 32 bits
// 21 with 8, 22 with 16).
u32 back_grid(u32 dtype, u64 rows, u64 cols)
{
    const u64 groups = (cols + 7) / 8, blocks = groups <= 64 ? (rows + 3) / 4 : rows;
    const u64 waves = groups <= 64 ? 4 : groups <= 1024 ? (groups + 63) / 64 : 16, resident = dtype == VMS_F32 ? 8 : 16, each = waves < resident ? resident / waves : 1;
    return (u32)(blocks < OPS_CUS * each ? blocks : OPS_CUS * each);
}

}  // namespace

extern "C" int vms_layernorm(const vms_layernorm_args *a, void *stream)
{
    if (!a) return VMS_EINVAL;
    if (a->struct_size != sizeof *a) return VMS_ESTRUCT;
    NormParams p;
    int rc = make_mask(a->mask, &p.mask);
    if (rc) return rc;
    if (a->dtype > VMS_BF16 || a->rows >> 31 || a->cols >> 26 || !a->cols || !(a->eps >= 0.0)) return VMS_EINVAL;
    if (!a->rows) return VMS_OK;
    if (!input_ok(a->d_x, a->dtype) || !output_ok(a->d_y, a->dtype, a->ldy, a->cols)) return VMS_EINVAL;
    if (a->d_residual ? !input_ok(a->d_residual, a->dtype) : a->mask.p > 0.0 || a->d_s) return VMS_EINVAL;
    if (a->d_s && !output_ok(a->d_s, a->dtype, a->lds, a->cols)) return VMS_EINVAL;
    if ((a->d_weight && !input_ok(a->d_weight, a->dtype)) || (a->d_bias && !input_ok(a->d_bias, a->dtype))) return VMS_EINVAL;
    if ((uintptr_t)a->d_stats % 4) return VMS_EINVAL;
    if (!stride_ok(a->ldx) || !stride_ok(a->ldr) || !stride_ok(a->ldy) || !stride_ok(a->lds)) return VMS_EINVAL;
    p.x = a->d_x;
    p.residual = a->d_residual;
    p.weight = a->d_weight;
    p.bias = a->d_bias;
    p.y = a->d_y;
    p.s = a->d_s;
    p.stats = a->d_stats;
    p.ldx = a->ldx;
    p.ldr = a->ldr;
    p.ldy = a->ldy;
    p.lds = a->lds;
    p.rows = (u32)a->rows;
    p.cols = (u32)a->cols;
    p.groups = (p.cols + 7) / 8;
    p.eps = (float)a->eps;
    const bool once = passes_by(a->rows * a->cols * type_bytes(a->dtype) * (2 + (a->d_residual != nullptr) + (a->d_s != nullptr)));
    return with_type(a->dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        return once ? launch_norm<T, true>(p, stream) : launch_norm<T, false>(p, stream);
    });
}

extern "C" size_t vms_layernorm_backward_workspace_bytes(const vms_layernorm_backward_args *a)
{
    if (!a || a->struct_size != sizeof *a || a->rows >> 31 || a->cols >> 26 || !wants_weights(a)) return 0;
    return (size_t)back_grid(a->dtype, a->rows, a->cols) * 2 * a->cols * sizeof(float);
}

extern "C" int vms_layernorm_backward(const vms_layernorm_backward_args *a, void *stream)
{
    if (!a) return VMS_EINVAL;
    if (a->struct_size != sizeof *a) return VMS_ESTRUCT;
    NormBackParams p;
    int rc = make_mask(a->mask, &p.mask);
    if (rc) return rc;
    if (a->dtype > VMS_BF16 || a->rows >> 31 || a->cols >> 26 || !a->cols) return VMS_EINVAL;
    const bool weights = wants_weights(a);
    for (const void *d : { a->d_dweight, a->d_dbias })
        if (d && !input_ok(d, a->dtype)) return VMS_EINVAL;
    if (a->rows) {
        if (!input_ok(a->d_dy, a->dtype) || !input_ok(a->d_s, a->dtype) || !output_ok(a->d_dres, a->dtype, a->lddres, a->cols)) return VMS_EINVAL;
        if ((a->d_ds && !input_ok(a->d_ds, a->dtype)) || (a->d_weight && !input_ok(a->d_weight, a->dtype))) return VMS_EINVAL;
        if (a->d_dx && !output_ok(a->d_dx, a->dtype, a->lddx, a->cols)) return VMS_EINVAL;
        if (!a->d_stats || (uintptr_t)a->d_stats % 4) return VMS_EINVAL;
        if (!stride_ok(a->lddy) || !stride_ok(a->ldds) || !stride_ok(a->lds) || !stride_ok(a->lddres) || !stride_ok(a->lddx)) return VMS_EINVAL;
        const size_t need = vms_layernorm_backward_workspace_bytes(a);
        if (need && (!a->d_workspace || (uintptr_t)a->d_workspace % 16 || a->workspace_bytes < need)) return VMS_EWORKSPACE;
    }
    p.dy = a->d_dy;
    p.ds = a->d_ds;
    p.s = a->d_s;
    p.weight = a->d_weight;
    p.stats = a->d_stats;
    p.dres = a->d_dres;
    p.dx = a->d_dx;
    p.partial = (float *)a->d_workspace;
    p.lddy = a->lddy;
    p.ldds = a->ldds;
    p.lds = a->lds;
    p.lddres = a->lddres;
    p.lddx = a->lddx;
    p.rows = (u32)a->rows;
    p.cols = (u32)a->cols;
    p.groups = (p.cols + 7) / 8;
    const u32 grid = back_grid(a->dtype, a->rows, a->cols);
    return with_type(a->dtype, [&](auto *t) {
        typedef std::remove_pointer_t<decltype(t)> T;
        if (a->rows) {
            const bool once = passes_by(a->rows * a->cols * type_bytes(a->dtype) * (3 + (a->d_ds != nullptr) + (a->d_dx != nullptr)));
            if (weights)
                rc = once ? launch_norm_back<T, true, true>(p, grid, stream) : launch_norm_back<T, true, false>(p, grid, stream);
            else
                rc = once ? launch_norm_back<T, false, true>(p, grid, stream) : launch_norm_back<T, false, false>(p, grid, stream);
            if (rc) return rc;
        }
        if (!weights) return (int)VMS_OK;
        const NormJoinParams j = { (const float *)a->d_workspace, a->d_dweight, a->d_dbias, grid, p.cols };
        return ops_launch(norm_join_kernel<T>, dim3((p.cols + 31) / 32, 2), dim3(1024), 0, j, stream);
    });
}
