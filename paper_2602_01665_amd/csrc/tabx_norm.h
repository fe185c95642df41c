// Layer norm of rows and its gradients.
//
// A row of W elements is held in registers by LANES lanes, PIECES pieces of four consecutive elements each, so the mean
// and the sum of squared differences from it are two passes over registers and one over memory.  Piece q of lane l starts
// at element 4 (q LANES + l), but no later than W - 4: a last piece that would not be whole, and those behind the row's
// end, are the row's last four elements once more.  Such a piece counts in sums only for the elements that no piece
// before has (`Cut`), and what it stores is what others store there too.  A form (LANES, PIECES) is used for rows that
// fill all pieces but the last in all lanes, so only the last one is ever cut.
//
// A team (a wavefront, or a workgroup where a row takes more lanes) walks through a run of rows, 64 / LANES of them at a
// time; rows that are masked out are sorted out 64 at a time and cost their mask byte.  The next rows' loads are under way
// while it works on the present ones.  That needs every load and store of a turn to be issued in every turn and lane: the
// one counter that a wavefront waits by takes what might not have been issued as not issued, and then waits for
// everything.  So there is no branch around them: lanes without a row of their own repeat the first one of the turn, and
// behind the end of its run a team loads its last rows once more.
#pragma once
#include "tabx_rows.h"

#pragma clang fp contract(off)

namespace tabx {

struct NormArgs {
    const void *x;
    void       *y;                 // forward: the result; backward: the input's gradient, or nullptr
    const void *grad_y;            // backward only
    const uint8_t *row_mask;
    const float *weight, *bias;
    float      *mean, *rstd;       // forward: written; backward: read
    float      *partial;           // backward: [workgroup][2][width], or nullptr
    float      *grad_weight, *grad_bias;   // backward of a single workgroup, if `partial` is nullptr
    int64_t     rows, x_stride, y_stride, g_stride;
    int64_t     team_rows, lap;    // a team's rows are runs of at most 64 of them, `lap` rows from one run to the next
    int32_t     width, x_type, y_type, g_type;
    float       eps, inv_width;
    int32_t     stream;            // forward: the result goes past the caches
};

// Rows of up to a wavefront's lanes: four teams to a workgroup; else a workgroup is a team.
constexpr int threads_of(int lanes) { return lanes > 64 ? lanes : 256; }

// Wavefronts of the backward pass that a SIMD holds: its registers go with the pieces (28 of them for each, two rows of
// both inputs among them, and some 50 more).
constexpr int grad_wavefronts(int pieces) { return pieces <= 2 ? 4 : pieces == 3 ? 3 : 2; }

// Where a lane's pieces are, and what counts of its last one.
template <int LANES, int PIECES>
struct Cut {
    int lane, start;               // of the last piece
    int skip;                      // elements of the last piece that count elsewhere, all four if skip >= 4

    __device__ __forceinline__ Cut(int width) : lane((int)threadIdx.x % LANES)
    {
        const int j = 4 * ((PIECES - 1) * LANES + lane);
        start = LANES == 1 ? 0 : min(j, width - 4);
        skip = j - start;
        if (LANES == 1) skip = width;              // one lane per row of up to four elements: those from `width` on are none
    }
    __device__ __forceinline__ int at(int q) const { return q < PIECES - 1 ? 4 * (q * LANES + lane) : start; }
    __device__ __forceinline__ bool counts(int i) const { return LANES == 1 ? i < skip : i >= skip; }
    __device__ __forceinline__ f32x4 counted(f32x4 v) const
    {
        return f32x4{counts(0) ? v.x : 0.0f, counts(1) ? v.y : 0.0f, counts(2) ? v.z : 0.0f, counts(3) ? v.w : 0.0f};
    }
};

// A row as it lies in memory, elements of BYTES bytes.  It stays so until it is worked on, so that nothing waits for it.
template <int BYTES>
struct RawPiece;
template <>
struct RawPiece<4> {
    typedef f32x4 four;
    typedef f32x4 anywhere __attribute__((aligned(4)));
};
template <>
struct RawPiece<2> {
    typedef u32x2 four;
    typedef u32x2 anywhere __attribute__((aligned(2)));
};
template <int BYTES, int PIECES>
struct RawRow {
    typename RawPiece<BYTES>::four v[PIECES];
};

// ONCE: read by nobody else, so that it need not stay in the caches.
template <bool ONCE = false, int LANES, int BYTES, int PIECES>
__device__ __forceinline__ void load_raw(RawRow<BYTES, PIECES> &raw, const void *data, int64_t offset, const Cut<LANES, PIECES> &cut,
                                         int width)
{
    const char *row = (const char *)data + offset * BYTES;
    if constexpr (LANES == 1) {                    // rows of one to four elements: one by one
        const int b = min(1, width - 1), c = min(2, width - 1), d = width - 1;
        if constexpr (BYTES == 4) {
            const float *e = (const float *)row;
            raw.v[0] = f32x4{e[0], e[b], e[c], e[d]};
        } else {
            const uint16_t *e = (const uint16_t *)row;
            raw.v[0] = u32x2{(uint32_t)e[b] << 16 | e[0], (uint32_t)e[d] << 16 | e[c]};
        }
    } else {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            const auto *at = (const typename RawPiece<BYTES>::anywhere *)(row + cut.at(q) * BYTES);
            raw.v[q] = ONCE ? __builtin_nontemporal_load(at) : *at;
        }
    }
}

template <int BYTES, int PIECES>
__device__ __forceinline__ void unpack(f32x4 (&v)[PIECES], const RawRow<BYTES, PIECES> &raw, int type)
{
    if constexpr (BYTES == 4) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] = raw.v[q];
    } else if (type == TABX_BF16) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            const uint32_t a = raw.v[q].x, b = raw.v[q].y;
            v[q] = f32x4{__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16),
                         __uint_as_float(b & 0xffff0000u)};
        }
    } else {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            f16x4 h;
            __builtin_memcpy(&h, &raw.v[q], 8);
            v[q] = __builtin_convertvector(h, f32x4);
        }
    }
}

template <int TYPE, bool STREAM, int LANES, int PIECES>
__device__ __forceinline__ void store_pieces(const f32x4 (&v)[PIECES], void *data, int64_t offset, const Cut<LANES, PIECES> &cut,
                                             int width)
{
    typedef typename Element<TYPE>::one T;
    T *row = (T *)data + offset;
    if constexpr (LANES == 1) {
        row[0] = (T)v[0].x;
        if (width > 1) row[1] = (T)v[0].y;
        if (width > 2) row[2] = (T)v[0].z;
        if (width > 3) row[3] = (T)v[0].w;
    } else {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) store_four<TYPE, STREAM>(row + cut.at(q), v[q]);
    }
}

template <bool STREAM = false, int LANES, int PIECES>
__device__ __forceinline__ void store_row(const f32x4 (&v)[PIECES], void *data, int type, int64_t offset,
                                          const Cut<LANES, PIECES> &cut, int width)
{
    if (type == TABX_F32) store_pieces<TABX_F32, STREAM>(v, data, offset, cut, width);
    else if (type == TABX_BF16) store_pieces<TABX_BF16, STREAM>(v, data, offset, cut, width);
    else store_pieces<TABX_F16, STREAM>(v, data, offset, cut, width);
}

// Per-column values: `other` where there are none.
template <int LANES, int PIECES>
__device__ __forceinline__ void load_columns(f32x4 (&v)[PIECES], const float *columns, float other, const Cut<LANES, PIECES> &cut,
                                             int width)
{
    if (columns) {
        RawRow<4, PIECES> raw;
        load_raw(raw, columns, 0, cut, width);
        unpack(v, raw, TABX_F32);
    } else {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] = f32x4{other, other, other, other};
    }
}

// Sum over the lanes of a row; rows of more than a wavefront meet in `slots` (one float per wavefront; a call uses
// slots that no wavefront can still be reading: those of the call before the last).
template <int LANES>
__device__ __forceinline__ float row_sum(float v, float *slots)
{
    v = lanes_sum<(LANES < 64 ? LANES : 64)>(v);
    if (LANES > 64) {
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) v += slots[w];
    }
    return v;
}

__device__ __forceinline__ float sum_of(f32x4 v) { return (v.x + v.y) + (v.z + v.w); }

__device__ __forceinline__ f32x4 fma4(f32x4 a, f32x4 b, f32x4 c)
{
    return f32x4{fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y), fmaf(a.z, b.z, c.z), fmaf(a.w, b.w, c.w)};
}

// A team's way through its rows.
template <int LANES>
struct Walk {
    static constexpr int kAtOnce = LANES < 64 ? 64 / LANES : 1;
    const uint8_t *mask;
    int64_t  base, next, rows, lap;   // the run at hand, the one after it, where the rows end
    int      run;                  // rows of a run
    uint64_t on, off;              // which of the run's rows count and have not been taken; which are masked out
    int      sub;                  // which of the rows worked on at a time is this lane's

    __device__ __forceinline__ Walk(const NormArgs &a)
    {
        const int wave = LANES <= 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0;
        const int64_t team = (int64_t)blockIdx.x * (LANES <= 64 ? threads_of(LANES) / 64 : 1) + wave;
        mask = a.row_mask;
        run = (int)a.team_rows;
        next = team * a.team_rows;
        rows = a.rows;
        lap = a.lap;
        base = 0;
        on = off = 0;
        sub = ((int)threadIdx.x & 63) / (LANES < 64 ? LANES : 64);
    }
    // Another run; false if there is none.
    __device__ __forceinline__ bool refill()
    {
        if (next >= rows) return false;
        const int lane = (int)threadIdx.x & 63;
        const bool there = lane < run && next + lane < rows;
        const uint64_t all = __ballot(there);
        on = mask ? __ballot(there && mask[there ? next + lane : next] != 0) : all;
        off = all & ~on;
        base = next;
        next += lap;
        return true;
    }
    // More rows to take: of the run at hand, or of those behind.  skipped(): called for every run.
    template <typename Skipped>
    __device__ __forceinline__ bool more(Skipped skipped)
    {
        while (on == 0) {
            if (!refill()) return false;
            skipped();
        }
        return true;
    }
    // This lane's row among the next kAtOnce of a set that is not empty; the first of them, and own = false, if there
    // are not so many.
    __device__ __forceinline__ int64_t take(uint64_t &set, bool &own)
    {
        int mine = __builtin_ctzll(set);
        own = true;
        if constexpr (LANES == 1) {
            own = set >> sub & 1;
            mine = own ? sub : mine;
            set = 0;
        } else {
            set &= set - 1;
            if (kAtOnce > 1) own = sub == 0;
#pragma unroll
            for (int k = 1; k < kAtOnce; ++k) {
                const bool some = set != 0;
                const int bit = some ? __builtin_ctzll(set) : 0;
                mine = some && sub == k ? bit : mine;
                own = own || (some && sub == k);
                set &= set - 1;
            }
        }
        return base + mine;
    }
};

// Whether a team's next rows are under way while it works on the present ones.  Workgroups as teams cover each other's
// waits (forward, rows of 2048: 282 us, 334 with the next row under way, whose registers cost a workgroup per CU), but
// for the widest, of which a CU holds one (backward, rows of 6000: 206 us, 181 with it).
template <int LANES>
constexpr bool kNormAhead = LANES <= 64;
template <int LANES>
constexpr bool kGradAhead = LANES <= 64 || LANES == 1024;

// Works on all rows of a run: `more` says whether there are any (and makes them the ones to be taken), `fetch` loads them,
// with the loads of those behind under way; two sets of registers take turns, so that none is copied (a copy would wait
// for the loads).
template <bool AHEAD, typename Rows, typename More, typename Fetch, typename Work>
__device__ __forceinline__ void walk_through(More more, Fetch fetch, Work work)
{
    Rows first;
    if constexpr (!AHEAD) {
        while (more()) {
            fetch(first, true, first);
            work(first);
        }
    } else {
        Rows second;
        if (!more()) return;
        fetch(first, true, first);
        for (;;) {
            const bool some = more();
            fetch(second, some, first);
            work(first);
            if (!some) return;
            const bool again = more();
            fetch(first, again, second);
            work(second);
            if (!again) return;
        }
    }
}

// Bound by HBM.  Rows go through the machine in the order of their addresses: a team has few rows, and the next
// workgroup's lie behind its own (a wavefront of 64 rows: 85 us, of 4: 76, 10v10 x 16384, half of the rows).  71 us, 5.1
// TB/s of x and y (a large copy on this card: 5.2); 64v64 x 1024, all rows, 281 us, 5.7 TB/s.
template <int LANES, int PIECES, int X_BYTES>
__global__ __launch_bounds__(threads_of(LANES)) void tabx_norm_kernel(const NormArgs a)
{
    constexpr int THREADS = threads_of(LANES);
    __shared__ float slots[4][THREADS / 64];
    const Cut<LANES, PIECES> cut(a.width);
    Walk<LANES> walk(a);
    f32x4 w[PIECES], b[PIECES];
    load_columns(w, a.weight, 1.0f, cut, a.width);
    load_columns(b, a.bias, 0.0f, cut, a.width);
    int turn = 0;
    struct Rows {
        RawRow<X_BYTES, PIECES> x;
        int64_t r;
    };
    const auto more = [&] { return walk.more([] {}); };
    const auto fetch = [&](Rows &h, bool some, const Rows &last) {
        bool own;
        h.r = some ? walk.take(walk.on, own) : last.r;
        load_raw(h.x, a.x, h.r * a.x_stride, cut, a.width);
    };
    const auto work = [&](const Rows &h) {
        f32x4 v[PIECES];
        unpack(v, h.x, a.x_type);
        f32x4 sum = cut.counted(v[PIECES - 1]);
#pragma unroll
        for (int q = 0; q < PIECES - 1; ++q) sum += v[q];
        const float mean = row_sum<LANES>(sum_of(sum), slots[turn]) * a.inv_width;
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] -= mean;
        const f32x4 last = cut.counted(v[PIECES - 1]);
        f32x4 squares = last * last;
#pragma unroll
        for (int q = 0; q < PIECES - 1; ++q) squares = fma4(v[q], v[q], squares);
        const float rstd = rsqrtf(fmaf(row_sum<LANES>(sum_of(squares), slots[turn + 1]), a.inv_width, a.eps));
        turn ^= 2;
        if (a.mean && cut.lane == 0) {
            a.mean[h.r] = mean;
            a.rstd[h.r] = rstd;
        }
#pragma unroll
        for (int q = 0; q < PIECES; ++q) v[q] = fma4(v[q] * rstd, w[q], b[q]);
        if (a.stream) store_row<true>(v, a.y, a.y_type, h.r * a.y_stride, cut, a.width);
        else store_row(v, a.y, a.y_type, h.r * a.y_stride, cut, a.width);
    };
    walk_through<kNormAhead<LANES>, Rows>(more, fetch, work);
}

// INPUTS: the input's gradient is wanted.  Each workgroup adds up its rows' parts of the weight's and the bias's
// gradient in registers, one column set per lane, and leaves them in a.partial (if that is given).  Bound by HBM: a
// workgroup stays, for the sake of its sums, but its teams take short runs of rows a lap apart, so that the machine goes
// through the rows in the order of their addresses all the same (200000 rows of 512 in bf16 136 us with a long run per
// team, 121 with runs of four rows, 5.1 TB/s; 85051 rows 61 and 56).
// ONCE: more is read than the memory-side cache holds, so nothing of it is kept (10v10 x 16384 without the input's
// gradient, 364 MB: 64 us, 5.7 TB/s, 69 without; 66 MB: 14.4 and 13.3; with the input's gradient it is slower, 182 us
// and 171, 200000 rows of 700).  Rows that are masked out count, as the host does not see them; a call that reads half of
// that gains too (132 MB of 265: 28.6 us and 31.3).
template <int LANES, int PIECES, int X_BYTES, int G_BYTES, bool INPUTS, bool ONCE>
__global__ __launch_bounds__(threads_of(LANES), grad_wavefronts(PIECES)) void tabx_norm_grad_kernel(const NormArgs a)
{
    constexpr int THREADS = threads_of(LANES);
    constexpr int WAVES = THREADS / 64;
    __shared__ float slots[4][WAVES];
    __shared__ f32x4 meet[LANES <= 64 ? WAVES : 1][LANES <= 64 ? LANES : 1];
    const Cut<LANES, PIECES> cut(a.width);
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    Walk<LANES> walk(a);
    f32x4 w[INPUTS ? PIECES : 1], dw[PIECES], db[PIECES];
    if constexpr (INPUTS) load_columns(w, a.weight, 1.0f, cut, a.width);
#pragma unroll
    for (int q = 0; q < PIECES; ++q) dw[q] = zero, db[q] = zero;
    const bool sums = !INPUTS || a.partial || a.grad_weight || a.grad_bias;
    // a row's mean and rstd are the same for a whole wavefront; without a lane's own address they would be moved to
    // scalar registers as soon as they are loaded, and waited for
    int here = 0;
    asm("v_mov_b32 %0, 0" : "=v"(here));
    int turn = 0;
    struct Rows {
        RawRow<X_BYTES, PIECES> x;
        RawRow<G_BYTES, PIECES> g;
        float   mean, rstd;
        int64_t r;
        bool    own;
    };
    const auto more = [&] {
        return walk.more([&] {
            if constexpr (INPUTS) {                // rows that are masked out have no gradient
                f32x4 none[PIECES];
#pragma unroll
                for (int q = 0; q < PIECES; ++q) none[q] = zero;
                while (walk.off) {
                    bool own;
                    store_row(none, a.y, a.y_type, walk.take(walk.off, own) * a.y_stride, cut, a.width);
                }
            }
        });
    };
    const auto fetch = [&](Rows &h, bool some, const Rows &last) {
        h.r = some ? walk.take(walk.on, h.own) : last.r;
        h.mean = (a.mean + h.r)[here];
        h.rstd = (a.rstd + h.r)[here];
        load_raw<ONCE>(h.x, a.x, h.r * a.x_stride, cut, a.width);
        load_raw<ONCE>(h.g, a.grad_y, h.r * a.g_stride, cut, a.width);
    };
    const auto work = [&](const Rows &h) {
        f32x4 x[PIECES], g[PIECES];
        unpack(x, h.x, a.x_type);
        unpack(g, h.g, a.g_type);
#pragma unroll
        for (int q = 0; q < PIECES; ++q) x[q] = (x[q] - h.mean) * h.rstd;
        const f32x4 last = cut.counted(g[PIECES - 1]);
        if (sums && (LANES >= 64 || h.own)) {
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                const f32x4 t = q < PIECES - 1 ? g[q] : last;
                dw[q] = fma4(t, x[q], dw[q]);
                db[q] += t;
            }
        }
        if constexpr (INPUTS) {
            f32x4 total = last * w[PIECES - 1], along = total * x[PIECES - 1];
#pragma unroll
            for (int q = 0; q < PIECES; ++q) {
                g[q] *= w[q];
                if (q < PIECES - 1) {
                    total += g[q];
                    along = fma4(g[q], x[q], along);
                }
            }
            const float sg = row_sum<LANES>(sum_of(total), slots[turn]) * a.inv_width;
            const float sh = row_sum<LANES>(sum_of(along), slots[turn + 1]) * a.inv_width;
            turn ^= 2;
#pragma unroll
            for (int q = 0; q < PIECES; ++q) g[q] = (fma4(x[q], f32x4{-sh, -sh, -sh, -sh}, g[q]) - sg) * h.rstd;
            store_row(g, a.y, a.y_type, h.r * a.y_stride, cut, a.width);
        }
    };
    walk_through<kGradAhead<LANES>, Rows>(more, fetch, work);
    if (!sums) return;
    // the rows worked on side by side in a wavefront, then the wavefronts
    const int64_t part = (int64_t)blockIdx.x * 2 * a.width;
    float *const outs[2] = {a.partial ? a.partial + part : a.grad_weight, a.partial ? a.partial + part + a.width : a.grad_bias};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        float *const out = outs[half];
        if (!out) continue;                        // (the same for all)
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            f32x4 v = half ? db[q] : dw[q];
            if (LANES <= 64) {
#pragma unroll
                for (int d = LANES; d < 64; d *= 2) {
                    v.x += __shfl_xor(v.x, d);
                    v.y += __shfl_xor(v.y, d);
                    v.z += __shfl_xor(v.z, d);
                    v.w += __shfl_xor(v.w, d);
                }
                __syncthreads();                   // the piece before has been read
                if ((int)(threadIdx.x & 63) < LANES) meet[LANES <= 64 ? threadIdx.x >> 6 : 0][LANES <= 64 ? cut.lane : 0] = v;
                __syncthreads();
                if ((int)threadIdx.x >= LANES) continue;
                v = meet[0][LANES <= 64 ? cut.lane : 0];
#pragma unroll
                for (int k = 1; k < WAVES; ++k) v += meet[LANES <= 64 ? k : 0][LANES <= 64 ? cut.lane : 0];
            }
            float *at = out + cut.at(q);
            if (q < PIECES - 1) {
                store_four<TABX_F32>(at, v);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (cut.counts(i)) at[i] = v[i];
            }
        }
    }
}

// Adds up the workgroups' parts: 32 columns per workgroup, 32 runs of parts side by side, always in the same order.
__global__ __launch_bounds__(1024) void tabx_norm_join_kernel(const float *partial, int parts, int width, float *grad_weight,
                                                              float *grad_bias)
{
    __shared__ float meet[32][33];
    const int c = (int)threadIdx.x & 31, run = (int)threadIdx.x >> 5;
    const int j = (int)blockIdx.x * 32 + c;
    float s = 0.0f;
    if (j < 2 * width) {
#pragma unroll 8
        for (int k = run; k < parts; k += 32) s += partial[(int64_t)k * 2 * width + j];
    }
    meet[run][c] = s;
    __syncthreads();
    if (run != 0 || j >= 2 * width) return;
#pragma unroll
    for (int k = 1; k < 32; ++k) s += meet[k][c];
    float *const out = j < width ? grad_weight : grad_bias;
    if (out) out[j < width ? j : j - width] = s;
}

} // namespace tabx
