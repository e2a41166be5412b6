// Norms before and after a block fused with its gate and residual scale, and their gradients.
//
//   b = N(branch; post), res = keep residual + scale gate b, out = N(res; pre)
// forward reads two matrices and writes two; backward reads four and writes two. Both only move memory.
// A row lives in the registers of one team of threads (one to four pieces of 8 neighbouring elements each;
// a team is a wave or part of one for narrow rows and else a block), so every matrix is read once; the row's
// statistics are sums inside the team, formed in two passes over the registers (mean first, then squares
// of the differences). Rows of any width and alignment are read 16 bytes at a time (the hardware takes
// any address).
//
// Gradients, with ^ for the normalised values, i for their factors and mean() over a row:
//   d1 = dout pre, dtot = dres + i_n (d1 - n^ mean(d1 n^) [- mean(d1)]), dresidual = keep dtot
//   db = scale gate dtot, d2 = db post, dbranch = i_o (d2 - o^ mean(d2 o^) [- mean(d2)])
//   dpre = sum_r dout n^, dpost = sum_r db o^, dgate = sum over its rows of scale dtot b
// (brackets: layer norm). res is formed again from residual and branch in fp32, so that out's gradient
// belongs to the out that was computed. A team walks a run of rows with its weights and sums over rows in
// registers and the next row's four pieces on their way; the sums of all blocks are joined by a second
// kernel in a fixed order. Rows of more than 4096 columns take two pieces a thread and keep sums in LDS.
// Forward, 128 MiB a matrix: 3.4 to 5.5 TB/s (bf16, layer, 1001 columns; fp32, RMS, 256). Backward: fp32 4.0 to
// 5.1 TB/s up to 8192 columns, bf16 4.0 to 4.8 where a team's last threads have columns and down to 2.5 where they
// just begin to (1025); 16384, four pieces, in part in scratch memory: RMS 2.9 to 3.4, layer 0.6 to 1.3.
#include "block_internal.h"

namespace enova {

namespace {

constexpr int kPiece = 8;      // neighbouring elements of a row that a thread takes at once

template <class T>
struct Raw {                   // a piece as it lies in memory
    uint4 q[sizeof(T) * kPiece / 16];
};

// Columns c .. c + 7 of a row. Where they go past its end, the row's last eight are read instead and
// unpack() puts them in their places: a load of its own for those threads would make the others, whose
// registers it writes too, wait for theirs (1000 columns: 2.6 TB/s instead of 4.5).
template <class T>
__device__ __forceinline__ Raw<T> load_piece(const T *row, int c, int model)
{
    Raw<T> r = {};
    if (model >= kPiece) {
        const T *const src = row + min(c, model - kPiece);
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(r) / 16); ++i)
            r.q[i] = reinterpret_cast<const Any16 *>(src)[i].v;
    } else if (c == 0) {
        T e[kPiece] = {};
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            if (i < model)
                e[i] = row[i];
        __builtin_memcpy(&r, e, sizeof(r));
    }
    return r;
}
template <class T>
__device__ __forceinline__ void unpack(const Raw<T> &r, int c, int model, bool whole, float (&v)[kPiece])
{
#pragma unroll
    for (int i = 0; i < static_cast<int>(sizeof(r) / 16); ++i) {
        const unsigned u[4] = {r.q[i].x, r.q[i].y, r.q[i].z, r.q[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) {
                v[4 * i + e] = __uint_as_float(u[e]);
            } else {
                v[2 * e] = __uint_as_float(u[e] << 16);
                v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
            }
        }
    }
    if (whole || model < kPiece)       // whole: the team's pieces cover the row exactly
        return;
    const int past = c - min(c, model - kPiece);       // how many elements the piece was read too early
    if (past == 0)                                     // all threads of all waves but a row's last
        return;
    if (model % kPiece) {
#pragma unroll
        for (int d = 1; d < kPiece; d *= 2)
#pragma unroll
            for (int e = 0; e < kPiece; ++e)
                v[e] = past & d ? (e + d < kPiece ? v[e + d] : 0.0f) : v[e];
    }
#pragma unroll
    for (int e = 0; e < kPiece; ++e)
        v[e] = past >= kPiece ? 0.0f : v[e];
}
template <class T>
__device__ __forceinline__ void store_piece(T *row, int c, int model, const float (&v)[kPiece])
{
    T e[kPiece];
#pragma unroll
    for (int i = 0; i < kPiece; ++i)
        e[i] = static_cast<T>(v[i]);
    if (c + kPiece <= model) {
        Raw<T> r;
        __builtin_memcpy(&r, e, sizeof(r));
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(r) / 16); ++i)
            reinterpret_cast<Any16 *>(row + c)[i].v = r.q[i];
    } else {
#pragma unroll
        for (int i = 0; i < kPiece; ++i)
            if (c + i < model)
                row[c + i] = e[i];
    }
}
__device__ __forceinline__ void load_cols(const float *src, int c, int model, bool whole, float fill, float (&v)[kPiece])
{
#pragma unroll
    for (int e = 0; e < kPiece; ++e)
        v[e] = fill;
    if (src)
        unpack(load_piece(src, c, model), c, model, whole, v);
}

// Sums of two values over a team, in a fixed order. A team of several waves is a block; its sums alternate
// between two places, so one barrier a sum is enough.
template <int TEAM>
struct TeamSum {
    float2 (*shared)[16];
    int turn = 0;
    __device__ float2 operator()(float x, float y)
    {
        float2 v = make_float2(x, y);
#pragma unroll
        for (int d = (TEAM < 64 ? TEAM : 64) / 2; d > 0; d >>= 1) {
            v.x += __shfl_xor(v.x, d);
            v.y += __shfl_xor(v.y, d);
        }
        if constexpr (TEAM > 64) {
            float2 *const s = shared[turn];
            turn ^= 1;
            if ((threadIdx.x & 63) == 0)
                s[threadIdx.x >> 6] = v;
            __syncthreads();
            v = s[0];
#pragma unroll
            for (int w = 1; w < TEAM / 64; ++w) {
                v.x += s[w].x;
                v.y += s[w].y;
            }
        }
        return v;
    }
};

template <int TEAM>
constexpr int block_threads() { return TEAM <= 64 ? 256 : TEAM; }

// v's mean (0 for RMS) and factor 1 / sqrt(mean((v - mean)^2) + eps); elements past the row are 0.
template <int TEAM, int P>
__device__ __forceinline__ float2 row_stats(const float (&v)[P][kPiece], const int (&c)[P], int model, int layer, float eps,
                                            TeamSum<TEAM> &sum)
{
    const float inv = 1.0f / model;
    float mean = 0.0f;
    if (layer) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < kPiece; ++e)
                s += v[i][e];
        mean = sum(s, 0.0f).x * inv;
    }
    float q = 0.0f;
    const auto squares = [&](bool all) {
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int e = 0; e < kPiece; ++e) {
                const float d = v[i][e] - mean;
                q += all || c[i] + e < model ? d * d : 0.0f;
            }
    };
    if (model == TEAM * P * kPiece || !layer)      // without a mean the elements past the row are still 0
        squares(true);
    else
        squares(false);
    q = sum(q, 0.0f).x * inv;
    return make_float2(mean, 1.0f / sqrtf(q + eps));
}

template <class T, int TEAM, int P>
__global__ void __launch_bounds__(block_threads<TEAM>()) k_resnorm_forward(NormParams p, int64_t first_block)
{
    __shared__ float2 shared[2][16];
    constexpr int kTeams = block_threads<TEAM>() / TEAM;
    if (TEAM > 16)
        __builtin_assume(p.model >= kPiece);
    const int t = threadIdx.x % TEAM;
    const int64_t row = (first_block + blockIdx.x) * kTeams + threadIdx.x / TEAM;
    if (row >= p.rows)                 // a whole team
        return;
    const int64_t at = row * p.model;
    TeamSum<TEAM> sum{shared};
    const bool whole = p.model == TEAM * P * kPiece;
    int c[P];
    Raw<T> branch[P], residual[P];
    float o[P][kPiece], r[P][kPiece], w[kPiece];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        c[i] = (i * TEAM + t) * kPiece;
        branch[i] = load_piece(static_cast<const T *>(p.branch) + at, c[i], p.model);
        residual[i] = load_piece(static_cast<const T *>(p.residual) + at, c[i], p.model);
    }
    // The weights are on their way while the statistics are summed (a team of 1024 has no registers for them).
    constexpr bool kEarly = P == 1 && TEAM < 1024;
    const float *const gate = p.gate ? p.gate + row / p.group * p.model : nullptr;
    const float *const from[5] = {p.post, p.post_bias, gate, p.pre, p.pre_bias};
    Raw<float> q[P][5];
    const auto ask = [&](int i, int k) {
        q[i][k] = {};
        if (from[k])
            q[i][k] = load_piece(from[k], c[i], p.model);
    };
    const auto weights = [&](int i, int k, float fill) {
        if (!kEarly)
            ask(i, k);
        unpack(q[i][k], c[i], p.model, whole, w);
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            w[e] = from[k] ? w[e] : fill;
    };
    if (kEarly)
#pragma unroll
        for (int i = 0; i < P; ++i)
#pragma unroll
            for (int k = 0; k < 5; ++k)
                ask(i, k);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        unpack(branch[i], c[i], p.model, whole, o[i]);
        unpack(residual[i], c[i], p.model, whole, r[i]);
    }
    // In place, a row's last eight values may lie in the piece of another wave's thread as well: nobody stores before all
    // have read. (With a first norm its sums are that barrier.)
    if (TEAM > 64 && !p.post && p.res == p.residual)
        __syncthreads();
    float2 so = make_float2(0.0f, 1.0f);
    if (p.post)
        so = row_stats<TEAM, P>(o, c, p.model, p.layer, p.eps, sum);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        if (p.post) {
            weights(i, 0, 1.0f);
#pragma unroll
            for (int e = 0; e < kPiece; ++e)
                o[i][e] = (o[i][e] - so.x) * so.y * w[e];
            if (p.post_bias) {
                weights(i, 1, 0.0f);
#pragma unroll
                for (int e = 0; e < kPiece; ++e)
                    o[i][e] += w[e];
            }
        }
        weights(i, 2, 1.0f);
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            r[i][e] = p.keep * r[i][e] + p.scale * w[e] * o[i][e];
        store_piece(static_cast<T *>(p.res) + at, c[i], p.model, r[i]);
    }
    const float2 sn = row_stats<TEAM, P>(r, c, p.model, p.layer, p.eps, sum);
#pragma unroll
    for (int i = 0; i < P; ++i) {
        weights(i, 3, 1.0f);
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            r[i][e] = (r[i][e] - sn.x) * sn.y * w[e];
        if (p.pre_bias) {
            weights(i, 4, 0.0f);
#pragma unroll
            for (int e = 0; e < kPiece; ++e)
                r[i][e] += w[e];
        }
        store_piece(static_cast<T *>(p.out) + at, c[i], p.model, r[i]);
    }
    if (p.stats && t == 0)
        *reinterpret_cast<float4 *>(p.stats + 4 * row) = make_float4(so.x, so.y, sn.x, sn.y);
}

// The teams of a block add their sums up; a block that is one team has nothing to add.
template <int TEAM>
__device__ __forceinline__ void store_sums(float *dst, int model, int c, float (&s)[kPiece], float *lds)
{
    if constexpr (TEAM <= 64) {
        const int t = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            lds[(team * kPiece + e) * TEAM + t] = s[e];
        __syncthreads();
        if (team)
            return;
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            for (int k = 1; k < 256 / TEAM; ++k)
                s[e] += lds[(k * kPiece + e) * TEAM + t];
    }
    store_piece(dst, c, model, s);
}

// One sum over rows of a thread's columns: in registers, or for wide rows in LDS, where each thread has places
// of its own (a row's update takes a tenth of the time that its loads take).
template <int P, bool LDS>
struct RowSum {
    float v[P][kPiece] = {};
    __device__ void init(float4 *) {}
    __device__ void add(int i, const float (&x)[kPiece])
    {
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            v[i][e] += x[e];
    }
    __device__ void get(int i, float (&x)[kPiece]) const
    {
#pragma unroll
        for (int e = 0; e < kPiece; ++e)
            x[e] = v[i][e];
    }
};
template <int P>
struct RowSum<P, true> {
    float4 *at;
    __device__ void init(float4 *lds)
    {
        at = lds + threadIdx.x;
#pragma unroll
        for (int i = 0; i < 2 * P; ++i)
            at[i * blockDim.x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    __device__ void add(int i, const float (&x)[kPiece])
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float4 v = at[(2 * i + h) * blockDim.x];
            v.x += x[4 * h];
            v.y += x[4 * h + 1];
            v.z += x[4 * h + 2];
            v.w += x[4 * h + 3];
            at[(2 * i + h) * blockDim.x] = v;
        }
    }
    __device__ void get(int i, float (&x)[kPiece]) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 v = at[(2 * i + h) * blockDim.x];
            x[4 * h] = v.x;
            x[4 * h + 1] = v.y;
            x[4 * h + 2] = v.z;
            x[4 * h + 3] = v.w;
        }
    }
};

// Rows of more than 4096 columns keep sums in LDS: two for a plain RMS norm, else four where they fit.
template <int TEAM, int P, bool FULL>
constexpr int lds_sums() { return P == 1 ? 0 : FULL && TEAM * P * kPiece <= 8192 ? 4 : 2; }
template <int TEAM, int P, bool FULL>
constexpr size_t lds_sum_bytes() { return size_t{4} * lds_sums<TEAM, P, FULL>() * TEAM * P * kPiece; }

// FULL: layer norms, or biases; else plain RMS norms, which need neither means nor two of the sums.
// AHEAD: the next row is read while this one is worked on. Two pieces a thread have the registers for it only for
// plain RMS norms of bf16 (8192 columns, layer, bf16: 228 us with it, in part in scratch memory, 194 without).
template <class T, int TEAM, int P, bool FULL, bool AHEAD = P == 1 || (P == 2 && !FULL && sizeof(T) == 2)>
__global__ void __launch_bounds__(block_threads<TEAM>()) k_resnorm_backward(NormParams p)
{
    __shared__ float2 shared[2][16];
    __shared__ float joined[TEAM <= 64 ? 256 * kPiece : 1];
    extern __shared__ float4 row_sums[];
    constexpr int kTeams = block_threads<TEAM>() / TEAM;
    if (TEAM > 16)                     // narrower rows have the smallest team
        __builtin_assume(p.model >= kPiece);
    const int t = threadIdx.x % TEAM;
    const int64_t team = static_cast<int64_t>(blockIdx.x) * kTeams + (kTeams > 1 ? threadIdx.x / TEAM : 0);
    const int64_t item0 = min(team * p.items_per_team, p.items), item1 = min(item0 + p.items_per_team, p.items);
    const float inv = 1.0f / p.model;
    TeamSum<TEAM> sum{shared};
    const bool whole = p.model == TEAM * P * kPiece;
    int c[P];
    // Rows of four pieces a thread read their weights again for each row (from the caches) rather than keep them.
    constexpr bool kKeep = P <= 2, kAhead = AHEAD;
    constexpr int kInLds = lds_sums<TEAM, P, FULL>(), kSumPlace = 2 * P * TEAM;
    float post[P][kPiece], post_bias[P][kPiece], pre[P][kPiece], gate[P][kPiece], s_gate[P][kPiece] = {};
    RowSum<P, (kInLds > 0)> s_post, s_pre;
    RowSum<P, (kInLds > 2)> s_pb, s_nb;
    s_post.init(row_sums);
    s_pre.init(row_sums + kSumPlace);
    if (FULL) {
        s_pb.init(row_sums + 2 * kSumPlace);
        s_nb.init(row_sums + 3 * kSumPlace);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        c[i] = (i * TEAM + t) * kPiece;
        load_cols(nullptr, c[i], p.model, whole, 1.0f, gate[i]);
    }
    // All loads before the first use; a weight that is not there reads this block's place for its sums instead and
    // drops what it read, so that no load waits behind a branch.
    float *const part = p.part + static_cast<int64_t>(blockIdx.x) * kNormSums * p.model;
    const auto weights = [&](int i, const float *g, bool with_gate) {
        const Raw<float> q0 = load_piece(p.post ? p.post : part, c[i], p.model), q1 = load_piece(p.pre ? p.pre : part, c[i], p.model);
        Raw<float> q2, q3;
        if (FULL)
            q2 = load_piece(p.post_bias ? p.post_bias : part, c[i], p.model);
        if (with_gate)
            q3 = load_piece(g ? g : part, c[i], p.model);
        const auto put = [&](const Raw<float> &q, bool there, float fill, float (&v)[kPiece]) {
            unpack(q, c[i], p.model, whole, v);
#pragma unroll
            for (int e = 0; e < kPiece; ++e)
                v[e] = there ? v[e] : fill;
        };
        put(q0, p.post, 1.0f, post[i]);
        put(q1, p.pre, 1.0f, pre[i]);
        if (FULL)
            put(q2, p.post_bias, 0.0f, post_bias[i]);
        if (with_gate)
            put(q3, g, 1.0f, gate[i]);
    };
    if (kKeep)
#pragma unroll
        for (int i = 0; i < P; ++i)
            weights(i, nullptr, false);
    // The rows of an item: part `sub` of a group's, or of all.
    const auto rows_of = [&](int64_t item, int64_t &first, int64_t &end) {
        const int64_t grp = p.gate ? item / p.items_per_group : 0, sub = item - grp * p.items_per_group;
        first = (p.gate ? grp * p.group : 0) + (p.gate ? sub : item) * p.item_rows;
        end = min(first + p.item_rows, p.rows);
        if (p.gate)
            end = min(end, (grp + 1) * p.group);
    };
    Raw<T> ro[P], rr[P], rn[P], rt[P];
    float4 rs;
    const auto fetch = [&](int64_t row) {
        const int64_t at = row * p.model;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            ro[i] = load_piece(static_cast<const T *>(p.branch) + at, c[i], p.model);
            rr[i] = load_piece(static_cast<const T *>(p.residual) + at, c[i], p.model);
            rn[i] = load_piece(static_cast<const T *>(p.dout) + at, c[i], p.model);
            rt[i] = load_piece(static_cast<const T *>(p.dres) + at, c[i], p.model);
        }
        rs = *reinterpret_cast<const float4 *>(p.stats + 4 * row);
    };
    for (int64_t item = item0; item < item1; ++item) {
        int64_t first, end;
        rows_of(item, first, end);
        const float *const gate_row = p.gate ? p.gate + item / p.items_per_group * p.model : nullptr;
        if (p.gate) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if (kKeep)
                    load_cols(gate_row, c[i], p.model, whole, 1.0f, gate[i]);
#pragma unroll
                for (int e = 0; e < kPiece; ++e)
                    s_gate[i][e] = 0.0f;
            }
        }
        if (kAhead && first < end)
            fetch(first);
        for (int64_t row = first; row < end; ++row) {
            const int64_t at = row * p.model;
            // The columns seem new in every row, or the compiler would keep some dozen addresses of a thread's pieces
            // and step them along.
#pragma unroll
            for (int i = 0; i < P; ++i)
                asm volatile("" : "+v"(c[i]));
            if (!kAhead)
                fetch(row);
            float o[P][kPiece], r[P][kPiece], dn[P][kPiece], dt[P][kPiece];
#pragma unroll
            for (int i = 0; i < P; ++i) {
                unpack(ro[i], c[i], p.model, whole, o[i]);
                unpack(rr[i], c[i], p.model, whole, r[i]);
                unpack(rn[i], c[i], p.model, whole, dn[i]);
                unpack(rt[i], c[i], p.model, whole, dt[i]);
            }
            const float4 st = rs;
            if (kAhead && row + 1 < end)
                fetch(row + 1);
            float sx = 0.0f, sy = 0.0f;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if (!kKeep) {          // one piece's weights at a time
                    __builtin_amdgcn_sched_barrier(0);
                    asm volatile("" ::: "memory");
                    weights(i, gate_row, true);
                }
                float v_pre[kPiece];
#pragma unroll
                for (int e = 0; e < kPiece; ++e) {
                    if (p.post)
                        o[i][e] = FULL ? (o[i][e] - st.x) * st.y : o[i][e] * st.y;
                    const float b = o[i][e] * post[i][e] + (FULL ? post_bias[i][e] : 0.0f);
                    const float v = p.keep * r[i][e] + p.scale * gate[i][e] * b;
                    r[i][e] = FULL ? (v - st.z) * st.w : v * st.w;
                    const float d1 = dn[i][e] * pre[i][e];       // 0 past the row, where dn is
                    sx += d1 * r[i][e];
                    sy += d1;
                    v_pre[e] = dn[i][e] * r[i][e];
                }
                s_pre.add(i, v_pre);
                if (FULL)
                    s_nb.add(i, dn[i]);
            }
            float2 s = sum(sx, sy);
            const float a1 = s.x * inv, a2 = FULL && p.layer ? s.y * inv : 0.0f;
            sx = sy = 0.0f;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                if (!kKeep) {          // one piece's weights at a time
                    __builtin_amdgcn_sched_barrier(0);
                    asm volatile("" ::: "memory");
                    weights(i, gate_row, true);
                }
                float v_post[kPiece], v_pb[kPiece];
#pragma unroll
                for (int e = 0; e < kPiece; ++e) {
                    float d = dt[i][e] + st.w * (dn[i][e] * pre[i][e] - r[i][e] * a1 - a2);
                    if (FULL)          // without a mean it is 0 past the row already
                        d = c[i] + e < p.model ? d : 0.0f;
                    const float sd = p.scale * d, db = sd * gate[i][e];
                    s_gate[i][e] += sd * (o[i][e] * post[i][e] + (FULL ? post_bias[i][e] : 0.0f));
                    v_post[e] = db * o[i][e];
                    v_pb[e] = db;
                    const float d2 = db * post[i][e];
                    sx += d2 * o[i][e];
                    sy += d2;
                    r[i][e] = p.keep * d;
                    dn[i][e] = d2;
                }
                s_post.add(i, v_post);
                if (FULL)
                    s_pb.add(i, v_pb);
                store_piece(static_cast<T *>(p.dresidual) + at, c[i], p.model, r[i]);
            }
            if (p.post) {
                s = sum(sx, sy);
                const float b1 = s.x * inv, b2 = FULL && p.layer ? s.y * inv : 0.0f;
#pragma unroll
                for (int i = 0; i < P; ++i)
#pragma unroll
                    for (int e = 0; e < kPiece; ++e)
                        dn[i][e] = st.y * (dn[i][e] - o[i][e] * b1 - b2);
            }
#pragma unroll
            for (int i = 0; i < P; ++i)
                store_piece(static_cast<T *>(p.dbranch) + at, c[i], p.model, dn[i]);
        }
        if (p.gate_part)
#pragma unroll
            for (int i = 0; i < P; ++i)
                store_piece(p.gate_part + item * p.model, c[i], p.model, s_gate[i]);
    }
    const auto leave = [&](int which, const auto &sums) {
        if (p.want >> which & 1u)
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float v[kPiece];
                sums.get(i, v);
                store_sums<TEAM>(part + which * static_cast<int64_t>(p.model), p.model, c[i], v, joined);
            }
    };
    leave(0, s_post);
    if (FULL)
        leave(1, s_pb);
    leave(2, s_pre);
    if (FULL)
        leave(3, s_nb);
}

// A block sums 64 columns of one output row: 16 waves take every 16th partial row each, in order, and are
// joined in order. Output row y is job y's, or with one job the sum of partial rows y per .. (y + 1) per - 1.
__global__ void __launch_bounds__(1024) k_norm_sums(NormSumJobs jobs, int64_t stride, int64_t per, int64_t total, int model)
{
    __shared__ float s[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
    const int64_t y = blockIdx.y;
    const float *const src = jobs.n > 1 ? jobs.src[y] : jobs.src[0];
    float *const out = jobs.n > 1 ? jobs.out[y] : jobs.out[0] + y * model;
    const int64_t first = jobs.n > 1 ? 0 : y * per, end = min(first + per, total);
    float v = 0.0f;
    if (c < model) {
#pragma unroll 8
        for (int64_t j = first + wave; j < end; j += 16)
            v += src[j * stride + c];
    }
    s[wave][lane] = v;
    __syncthreads();
    if (wave == 0 && c < model) {
#pragma unroll
        for (int w = 1; w < 16; ++w)
            v += s[w][lane];
        out[c] = v;
    }
}

template <class T, int TEAM, int P>
hipError_t launch_forward(const NormParams &p, hipStream_t st)
{
    constexpr int kThreads = block_threads<TEAM>(), kTeams = kThreads / TEAM;
    return launch_in_runs((p.rows + kTeams - 1) / kTeams, kThreads, [&](int64_t from, unsigned n) {
        k_resnorm_forward<T, TEAM, P><<<n, kThreads, 0, st>>>(p, from);
    });
}

// A power of two of pieces, one a thread, up to 4096 columns; three a thread where the columns fill no more than 3/4 of
// that, and three or four beyond it: a team with few waves wastes less where some have no columns, and they wait at
// every sum (layer norms of bf16, 128 MiB a matrix: 1500 columns 174 us with one piece, 129 with three; 6000 columns
// 163 with two of 512 threads, 124 with three of 256; 16384 the same with two of 1024 and four of 512).
template <class T>
hipError_t launch_forward(const NormParams &p, hipStream_t st)
{
    const int m = p.model;
    if (m > 8192)
        return m <= 12288 ? launch_forward<T, 512, 3>(p, st) : launch_forward<T, 1024, 2>(p, st);
    if (m > 4096)
        return m <= 6144 ? launch_forward<T, 256, 3>(p, st) : launch_forward<T, 256, 4>(p, st);
    switch (norm_team(m)) {
    case 16: return launch_forward<T, 16, 1>(p, st);
    case 32: return launch_forward<T, 32, 1>(p, st);
    case 64: return m <= 384 ? launch_forward<T, 16, 3>(p, st) : launch_forward<T, 64, 1>(p, st);
    case 128: return m <= 768 ? launch_forward<T, 32, 3>(p, st) : launch_forward<T, 128, 1>(p, st);
    case 256: return m <= 1536 ? launch_forward<T, 64, 3>(p, st) : launch_forward<T, 256, 1>(p, st);
    default: return m <= 2 * 1536 ? launch_forward<T, 128, 3>(p, st) : launch_forward<T, 512, 1>(p, st);
    }
}

// Rows of P pieces a thread, with sums in LDS.
template <class T, int P, bool FULL>
hipError_t launch_wide_backward(const NormParams &p, unsigned n, hipStream_t st)
{
    constexpr size_t kLds = lds_sum_bytes<512, P, FULL>();
    const hipError_t ready = allow_lds(reinterpret_cast<const void *>(k_resnorm_backward<T, 512, P, FULL>), kLds);
    if (ready != hipSuccess)
        return ready;
    k_resnorm_backward<T, 512, P, FULL><<<n, 512, kLds, st>>>(p);
    return hipGetLastError();
}

template <class T, bool FULL>
hipError_t launch_backward(const NormParams &p, unsigned n, hipStream_t st)
{
    switch (norm_team(p.model)) {
    case 16: k_resnorm_backward<T, 16, 1, FULL><<<n, 256, 0, st>>>(p); break;
    case 32: k_resnorm_backward<T, 32, 1, FULL><<<n, 256, 0, st>>>(p); break;
    case 64: k_resnorm_backward<T, 64, 1, FULL><<<n, 256, 0, st>>>(p); break;
    case 128: k_resnorm_backward<T, 128, 1, FULL><<<n, 128, 0, st>>>(p); break;
    case 256: k_resnorm_backward<T, 256, 1, FULL><<<n, 256, 0, st>>>(p); break;
    case 512: k_resnorm_backward<T, 512, 1, FULL><<<n, 512, 0, st>>>(p); break;
    default: return p.model <= 8192 ? launch_wide_backward<T, 2, FULL>(p, n, st) : launch_wide_backward<T, 4, FULL>(p, n, st);
    }
    return hipGetLastError();
}

}  // namespace

int norm_team(int model)
{
    return model <= 128 ? 16 : model <= 256 ? 32 : model <= 512 ? 64 : model <= 1024 ? 128 : model <= 2048 ? 256 : model <= 4096 ? 512 : 1024;
}

hipError_t launch_resnorm_forward(const NormParams &p, int dtype, hipStream_t st)
{
    return dtype == ENOVA_F32 ? launch_forward<float>(p, st) : launch_forward<__bf16>(p, st);
}

hipError_t launch_resnorm_backward(const NormParams &p, int dtype, int64_t blocks, hipStream_t st)
{
    const unsigned n = static_cast<unsigned>(blocks);
    const bool full = p.layer || p.post_bias || (p.want & 10u);
    if (dtype == ENOVA_F32)
        return full ? launch_backward<float, true>(p, n, st) : launch_backward<float, false>(p, n, st);
    return full ? launch_backward<__bf16, true>(p, n, st) : launch_backward<__bf16, false>(p, n, st);
}

hipError_t launch_norm_sums(const NormSumJobs &jobs, int64_t stride, int64_t per, int64_t total, int64_t rows, int model,
                            hipStream_t st)
{
    const dim3 grid((model + 63) / 64, static_cast<unsigned>(rows));
    k_norm_sums<<<grid, 1024, 0, st>>>(jobs, stride, per, total, model);
    return hipGetLastError();
}

}  // namespace enova
