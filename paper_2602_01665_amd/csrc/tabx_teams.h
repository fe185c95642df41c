// Rows in the registers of the lanes that share them, and a team's way through its rows (the norms' kernels).
//
// A row of W elements is held in registers by LANES lanes, PIECES pieces of four consecutive elements each, so a row's
// statistics are passes over registers, and there is one over memory.  Piece q of lane l starts at element
// 4 (q LANES + l), but no later than W - 4: a last piece that would not be whole, and those behind the row's end, are the
// row's last four elements once more.  Such a piece counts in sums only for the elements that no piece before has (`Cut`),
// and what it stores is what others store there too.  A form (LANES, PIECES) is used for rows that
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

    template <typename Args>                       // rows, row_mask, team_rows, lap
    __device__ __forceinline__ Walk(const Args &a)
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

} // namespace tabx
