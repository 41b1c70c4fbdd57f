// embed.hip -- rows of a table by their codes, scaled, and the table's gradient
// (finc_embed_* of finc.h).
//
// Both are bound by memory.  The gradient sorts the codes (a radix sort that keeps their
// order, so that its sums have a fixed one), then sums runs of equal codes: tiles of the
// sorted list side by side, and what runs on over a tile's end is joined afterwards.
// Rows that no code names are zeros: of a short list's table all of it beside the sort, in
// which one workgroup has work, of a long one's the rows that are not in the list.
#include "seq_common.h"

namespace {

using namespace finc_seq;

constexpr int kThreads = 256;
constexpr int kVec = 8;   // elements a thread takes of a row

struct Ids {
    const void *p;
    int wide, V;
    // the code, or V for padding
    __device__ unsigned key(long long m) const {
        const long long v = wide ? ((const long long *)p)[m] : ((const int *)p)[m];
        return v < 0 || v >= V ? (unsigned)V : (unsigned)v;
    }
};

// Eight elements a thread, all of a row's loads under way at once.
template <typename E, typename R>
__global__ __launch_bounds__(kThreads) void embed_kernel(Ids ids, const R *table, long long st,
                                                         E *y, long long sy, int M, int D,
                                                         FastDiv by_vecs, int vecs, float scale) {
    const long long i = block_of() * (long long)kThreads + threadIdx.x;
    if (i >= (long long)M * vecs)
        return;
    const int m = fdiv((int)i, by_vecs), col = ((int)i - m * vecs) * kVec;
    const unsigned k = ids.key(m);
    const int count = min(D - col, kVec);
    float v[kVec] = {};
    if (k < (unsigned)ids.V)
        load_upto<R, kVec>(table + k * st + col, count, v);
#pragma unroll
    for (int j = 0; j < kVec; ++j)
        v[j] *= scale;
    if (k >= (unsigned)ids.V)
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            v[j] = 0.0f;
    store_upto<E, kVec>(y + m * sy + col, count, v);
}

// ---- the sort ----------------------------------------------------------------------
// Eight bits a pass from the lowest on.  A block of the list goes to one workgroup, each
// of whose waves takes a run of it, 64 entries at a time: the lanes of one digit find
// each other by ballots, and the wave's next place for it is kept in LDS.

constexpr int kDigits = 256, kWaves = kThreads / 64;
// Entries of a block at least, and blocks at most: a block reads every block's counts, and
// its waves take their entries in turns (a pass over 32768 codes, 2.8 us of counts and 6.2 of
// places in 64 blocks of 512, 4.0 and 10.7 in 16 of 2048).
constexpr int kSortBlock = 512, kMostBlocks = 128;

struct Sort {
    Ids ids;
    const unsigned *key_in;   // NULL: the ids themselves, in order
    const int *at_in;
    unsigned *key_out;
    int *at_out;
    int *counts;              // (blocks, 256)
    int M, per, blocks, shift;
    float *zeros;             // of a short list: the table's gradient
    long long zero_count;
};

__device__ inline unsigned sort_key(const Sort &s, int i) {
    return s.key_in ? s.key_in[i] : s.ids.key(i);
}

__global__ __launch_bounds__(kThreads) void count_kernel(Sort s) {
    __shared__ int n[kDigits];
    n[threadIdx.x] = 0;
    __syncthreads();
    const long long first = (long long)blockIdx.x * s.per;
    const int end = (int)min(first + s.per, (long long)s.M);
    for (int i = (int)first + threadIdx.x; i < end; i += kThreads)
        atomicAdd(&n[sort_key(s, i) >> s.shift & 255u], 1);
    __syncthreads();
    s.counts[blockIdx.x * kDigits + threadIdx.x] = n[threadIdx.x];
}

// Sum of the values of the threads before this one, of the first 256 (all of the
// workgroup's threads call).
__device__ inline int before(int v, int (&waves)[4]) {
    const int t = threadIdx.x, lane = t & 63;
    int s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int u = __shfl_up(s, d);
        s += lane >= d ? u : 0;
    }
    if (lane == 63 && t < 256)
        waves[t >> 6] = s;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i)
        s += t >> 6 > i ? waves[i] : 0;
    return s - v;
}

// The lanes (of those that are `in`) with this lane's digit.
__device__ inline unsigned long long peers(unsigned digit, bool in) {
    unsigned long long mask = __ballot(in);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const unsigned long long have = __ballot(digit >> b & 1u);
        mask &= digit >> b & 1u ? have : ~have;
    }
    return mask;
}

__global__ __launch_bounds__(kThreads) void place_kernel(Sort s) {
    __shared__ int place[kWaves][kDigits], sums[4];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, block = blockIdx.x;
    // this digit's place: all of the smaller ones, and those of the blocks before
    int all = 0, earlier = 0;
#pragma unroll 16
    for (int b = 0; b < s.blocks; ++b) {
        const int n = s.counts[b * kDigits + t];
        all += n;
        earlier += b < block ? n : 0;
    }
    const int start = before(all, sums) + earlier;
#pragma unroll
    for (int i = 0; i < kWaves; ++i)
        place[i][t] = 0;
    __syncthreads();
    const long long first = (long long)block * s.per;
    const int n = (int)(min(first + s.per, (long long)s.M) - first);
    const int share = (n + kWaves - 1) / kWaves;   // of one wave
    const int lo = min(w * share, n), hi = min(lo + share, n);
    for (int i = lo + lane; i < hi; i += 64)
        atomicAdd(&place[w][sort_key(s, (int)first + i) >> s.shift & 255u], 1);
    __syncthreads();
    int at = start;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
        const int c = place[i][t];
        place[i][t] = at;
        at += c;
    }
    __syncthreads();
    for (int base = lo; base < hi; base += 64) {
        const int i = base + lane;
        const bool in = i < hi;
        const unsigned key = in ? sort_key(s, (int)first + i) : 0u;
        const unsigned digit = key >> s.shift & 255u;
        const unsigned long long same = peers(digit, in);
        const int rank = __popcll(same & ((1ull << lane) - 1ull));
        const int to = in ? place[w][digit] + rank : 0;
        wave_exchange();
        if (in) {
            s.key_out[to] = key;
            s.at_out[to] = s.at_in ? s.at_in[(int)first + i] : (int)first + i;
            if (rank == 0)
                place[w][digit] += __popcll(same);
        }
        wave_exchange();
    }
}

// Short lists in one launch: a workgroup keeps them in LDS from pass to pass.  The others
// write zeros (4096 codes of 70000 rows of 64: 39 us with a search for the rows that are
// not in the list, 32 so).
constexpr int kShort = 4096, kShortThreads = 1024, kShortWaves = kShortThreads / 64;
constexpr int kZeroed = 16384;   // elements of a workgroup

__global__ __launch_bounds__(kShortThreads) void sort_short_kernel(Sort s) {
    __shared__ unsigned key[2][kShort];
    __shared__ int at[2][kShort];
    __shared__ int place[kShortWaves][kDigits], totals[4];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    if (block_of() > 0) {
        const float zero[4] = {0, 0, 0, 0};
        const long long first = (block_of() - 1) * (long long)kZeroed + t * 4;
        for (int i = 0; i < kZeroed; i += kShortThreads * 4) {
            const long long left = s.zero_count - first - i;
            store_upto<float, 4>(s.zeros + first + i, (int)max(min(left, 4ll), 0ll), zero);
        }
        return;
    }
    for (int i = t; i < s.M; i += kShortThreads) {
        key[0][i] = s.ids.key(i);
        at[0][i] = i;
    }
    const int share = (s.M + kShortWaves - 1) / kShortWaves;
    const int lo = min(w * share, s.M), hi = min(lo + share, s.M);
    int from = 0;
    for (int shift = 0; shift < 32 && (shift == 0 || s.ids.V >> shift); shift += 8) {
        for (int i = t; i < kShortWaves * kDigits; i += kShortThreads)
            (&place[0][0])[i] = 0;
        __syncthreads();
        for (int i = lo + lane; i < hi; i += 64)
            atomicAdd(&place[w][key[from][i] >> shift & 255u], 1);
        __syncthreads();
        // a digit's first place, then that of every wave
        int all = 0, of[kShortWaves];
        if (t < kDigits)
#pragma unroll
            for (int i = 0; i < kShortWaves; ++i)
                all += of[i] = place[i][t];
        int first = before(all, totals);
        if (t < kDigits)
#pragma unroll
            for (int i = 0; i < kShortWaves; ++i) {
                place[i][t] = first;
                first += of[i];
            }
        __syncthreads();
        for (int base = lo; base < hi; base += 64) {
            const int i = base + lane;
            const bool in = i < hi;
            const unsigned k = in ? key[from][i] : 0u, digit = k >> shift & 255u;
            const unsigned long long same = peers(digit, in);
            const int rank = __popcll(same & ((1ull << lane) - 1ull));
            const int to = in ? place[w][digit] + rank : 0;
            wave_exchange();
            if (in) {
                key[from ^ 1][to] = k;
                at[from ^ 1][to] = at[from][i];
                if (rank == 0)
                    place[w][digit] += __popcll(same);
            }
            wave_exchange();
        }
        __syncthreads();
        from ^= 1;
    }
    for (int i = t; i < s.M; i += kShortThreads) {
        s.key_out[i] = key[from][i];
        s.at_out[i] = at[from][i];
    }
}

// ---- the sums -------------------------------------------------------------------------

// Entries of the sorted list that one wave's lanes add up: few of a short list, whose tiles
// do not fill the card and where the chain of loads counts (2048 codes of 64 columns: 26 us
// with 32 entries, 21 with 8; 14306 of 16384 rows of 23 46 and 39), more of a long one, whose
// runs over several tiles are read again (16384 codes of 256 rows of 512: 31 us with either;
// 65536 of two rows 75 with 32, 183 with 8).
constexpr int kAhead = 8;
int lanes_of(int D) {   // of a row: a power of two, up to a wave
    int n = 1;
    while (n < 64 && n * kVec < D)
        n *= 2;
    return n;
}
int tile_of(int M, int D) {
    return M <= 16384 && M * lanes_of(D) <= 1 << 19 ? kAhead : 4 * kAhead;
}

struct Sum {
    const unsigned *key;
    const int *at;
    const void *dy;
    long long sdy;
    float *dtable, *head, *tail;   // a tile's first and last run where they pass its ends
    float scale;
    int M, V, D, tile, tiles, lanes, slices;   // lanes of a row, slices of its columns
    long long sum_blocks;
};

// A lane's eight columns of a row of D, from `own` on.  Loads have no branches, which would
// wait for each: a lane that passes the row's end takes the row's last eight columns and
// stores those that are its own (D = 126: the sums of 434 codes 20 us before, 5 now).
struct Columns {
    int col, skip, D;
    bool narrow;
    __device__ Columns(int own, int d)
        : col(d < kVec ? 0 : min(own, d - kVec)), skip(own - col), D(d), narrow(d < kVec) {}
    template <typename E>
    __device__ typename Vec<E, kVec>::type load(const E *row) const {
        typename Vec<E, kVec>::type v;
        if (narrow)
#pragma unroll
            for (int j = 0; j < kVec; ++j)
                v[j] = row[min(j, D - 1)];
        else
            v = *(const typename Vec<E, kVec>::type *)(row + col);
        return v;
    }
    __device__ void store(float *row, const float *v) const {
        if (skip == 0)
            store_upto<float, kVec>(row + col, D - col, v);
        else
#pragma unroll
            for (int j = 1; j < kVec; ++j)
                if (j >= skip)
                    row[col + j] = v[j];
    }
};

// A group of lanes takes a tile of the list and up to 8 columns a lane.
template <typename E>
__device__ void sum_tiles(const Sum &s, long long group, int lane) {
    const int tile = (int)(group / s.slices), slice = (int)(group - (long long)tile * s.slices);
    if (tile >= s.tiles)
        return;
    const int own = (slice * s.lanes + lane) * kVec;
    if (own >= s.D)
        return;
    const Columns cols(own, s.D);
    const int first = tile * s.tile, n = min(s.tile, s.M - first);
    const unsigned V = (unsigned)s.V;
    const unsigned prior = first > 0 ? s.key[first - 1] : ~0u;
    const unsigned next = first + n < s.M ? s.key[first + n] : ~0u;
    const E *dy = (const E *)s.dy;
    float sum[kVec] = {};
    unsigned run = s.key[first];
    bool headed = prior == run;   // the run began before the tile
    auto flush = [&](bool open) {
        if (run >= V)
            return;
        float *to = headed ? s.head + (long long)tile * s.D
                           : (open ? s.tail + (long long)tile * s.D
                                   : s.dtable + (long long)run * s.D);
        const float f = headed || open ? 1.0f : s.scale;
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            sum[j] *= f;
        cols.store(to, sum);
    };
    unsigned k[kAhead];
    int at[kAhead];
    auto look = [&](int e) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            k[i] = s.key[first + min(e + i, n - 1)];
            at[i] = s.at[first + min(e + i, n - 1)];
        }
    };
    look(0);
    for (int e = 0; e < n; e += kAhead) {
        typename Vec<E, kVec>::type v[kAhead];
        unsigned of[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            of[i] = k[i];
            v[i] = cols.load(dy + at[i] * s.sdy);
        }
        look(e + kAhead);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (e + i < n) {
                if (of[i] != run) {
                    flush(false);
                    run = of[i];
                    headed = false;
#pragma unroll
                    for (int j = 0; j < kVec; ++j)
                        sum[j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < kVec; ++j)
                    sum[j] += (float)v[i][j];
            }
    }
    flush(next == run);
}

// Rows that no code of a long list names: zeros.  A wave looks for a few rows in the list, a
// lane each.
constexpr int kFillRows = 8;
__device__ inline void fill_rows(const Sum &s, long long wave, int lane) {
    const long long v0 = wave * kFillRows;
    if (v0 >= s.V)
        return;
    const int v = (int)min(v0 + (lane & (kFillRows - 1)), (long long)s.V - 1);
    int lo = 0, hi = s.M;   // the first entry of at least v
    while (lo < hi) {
        const int mid = lo + (hi - lo) / 2;
        if (s.key[mid] < (unsigned)v)
            lo = mid + 1;
        else
            hi = mid;
    }
    const bool there = lo < s.M && s.key[lo] == (unsigned)v;
    unsigned long long absent = __ballot(lane < kFillRows && v0 + lane < s.V && !there);
    const float zero[4] = {0, 0, 0, 0};
    while (absent) {
        const int i = __ffsll((long long)absent) - 1;
        absent &= absent - 1;
        float *p = s.dtable + (v0 + i) * s.D;
        for (int c = lane * 4; c < s.D; c += 256)
            store_upto<float, 4>(p + c, min(s.D - c, 4), zero);
    }
}

template <typename E>
__global__ __launch_bounds__(kThreads) void sum_kernel(Sum s) {
    const long long block = block_of();
    const int t = threadIdx.x;
    if (block < s.sum_blocks) {
        const int groups = kThreads / s.lanes;
        sum_tiles<E>(s, block * groups + t / s.lanes, t & (s.lanes - 1));
    } else
        fill_rows(s, (block - s.sum_blocks) * kWaves + (t >> 6), t & 63);
}

// Runs over several tiles: a workgroup for the one that begins in its tile and passes the
// end.  Its groups of lanes take a contiguous share of the tiles each.
__global__ __launch_bounds__(kThreads) void join_runs_kernel(Sum s) {
    __shared__ float part[kThreads * kVec];
    __shared__ int more;
    const int at = block_of(), tile = at / s.slices, slice = at - tile * s.slices;
    if (tile + 1 >= s.tiles)
        return;
    const int t = threadIdx.x, first = tile * s.tile, last = first + s.tile - 1;
    const unsigned run = s.key[last];
    if (run >= (unsigned)s.V || s.key[last + 1] != run || (first > 0 && s.key[first - 1] == run))
        return;
    // the tiles that begin with the run
    int n = 0;
    for (;;) {
        if (t == 0)
            more = kThreads;
        __syncthreads();
        const long long u = (long long)tile + 1 + n + t;
        if (u >= s.tiles || s.key[u * s.tile] != run)
            atomicMin(&more, t);
        __syncthreads();
        const int got = more;
        __syncthreads();
        n += got;
        if (got < kThreads)
            break;
    }
    const int groups = kThreads / s.lanes, g = t / s.lanes, lane = t & (s.lanes - 1);
    const int own = (slice * s.lanes + lane) * kVec;
    const Columns cols(own, s.D);
    const int share = (n + groups - 1) / groups, lo = min(g * share, n), hi = min(lo + share, n);
    float sum[kVec] = {};
    if (g == 0) {
        const auto v = cols.load(s.tail + (long long)tile * s.D);
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            sum[j] = v[j];
    }
    for (int i = lo; i < hi; i += kAhead) {
        Vec<float, kVec>::type v[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            v[e] = cols.load(s.head + ((long long)tile + 1 + min(i + e, hi - 1)) * s.D);
#pragma unroll
        for (int e = 0; e < kAhead; ++e)
            if (i + e < hi)
#pragma unroll
                for (int j = 0; j < kVec; ++j)
                    sum[j] += v[e][j];
    }
#pragma unroll
    for (int j = 0; j < kVec; ++j)
        part[j * kThreads + t] = sum[j];
    __syncthreads();
    if (g == 0) {
        for (int i = 1; i < groups; ++i)
#pragma unroll
            for (int j = 0; j < kVec; ++j)
                sum[j] += part[j * kThreads + i * s.lanes + lane];
#pragma unroll
        for (int j = 0; j < kVec; ++j)
            sum[j] *= s.scale;
        if (own < s.D)
            cols.store(s.dtable + (long long)run * s.D, sum);
    }
}

// ---- the host ----------------------------------------------------------------------------

// The columns of a row's last slice, up to 512, count within 31 bits too.
bool embed_shape(int M, int V, int D) {
    return M >= 0 && V >= 0 && D >= 1 && D <= INT32_MAX - 511 &&
           (long long)M * ((D + 7) / 8) < (1ll << 31) && (long long)V * ((D + 7) / 8) < (1ll << 37) &&
           M < (1 << 30) && V < (1 << 30);
}
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
Region rows(const void *p, long long step, long long M, int D, int size) {
    return {p, M, step, 1, 0, D, size};
}
int tiles_of(int M, int D) { return (int)cdivll(M, tile_of(M, D)); }

}  // namespace

extern "C" {

int finc_embed_forward(int type, int ttype, const void *ids, int wide, const void *table,
                       long long st, void *y, long long sy, int M, int V, int D, double scale,
                       hipStream_t stream) {
    if (!type_size(type) || (ttype != type && ttype != FINC_F32) || !embed_shape(M, V, D))
        return FINC_EINVAL;
    const Region in[] = {flat(ids, M, wide ? 8 : 4), rows(table, st, V, D, type_size(ttype))};
    const Region out[] = {rows(y, sy, M, D, type_size(type))};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    if (!writable(out[0]) || !disjoint(in, out))
        return FINC_EINVAL;
    if (M == 0)
        return FINC_OK;
    const int vecs = (D + kVec - 1) / kVec;
    const dim3 grid = grid_of(cdivll((long long)M * vecs, kThreads));
    const Ids i = {ids, wide, V};
    with_type(type, [&](auto e) {
        typedef decltype(e) E;
        if (ttype == type)
            embed_kernel<E, E><<<grid, kThreads, 0, stream>>>(i, (const E *)table, st, (E *)y, sy, M,
                                                              D, make_fastdiv(vecs), vecs,
                                                              (float)scale);
        else
            embed_kernel<E, float><<<grid, kThreads, 0, stream>>>(
                i, (const float *)table, st, (E *)y, sy, M, D, make_fastdiv(vecs), vecs,
                (float)scale);
    });
    return launched();
}

size_t finc_embed_workspace_bytes(int M, int V, int D) {
    if (!embed_shape(M, V, D))
        return 0;
    return 4 * round256((size_t)M * 4) + round256((size_t)kMostBlocks * kDigits * 4) +
           2 * round256((size_t)tiles_of(M, D) * D * 4);
}

int finc_embed_backward(int type, const void *ids, int wide, const void *dy, long long sdy,
                        float *dtable, int M, int V, int D, double scale, void *workspace,
                        hipStream_t stream) {
    if (!type_size(type) || !embed_shape(M, V, D) || ((uintptr_t)workspace & 255u))
        return FINC_EINVAL;
    const size_t space = finc_embed_workspace_bytes(M, V, D);
    const Region in[] = {flat(ids, M, wide ? 8 : 4), rows(dy, sdy, M, D, type_size(type))};
    const Region out[] = {flat(dtable, (long long)V * D, 4), flat(workspace, (long long)space, 1)};
    for (const Region &r : in)
        if (!readable(r))
            return FINC_EINVAL;
    for (const Region &r : out)
        if (!readable(r))
            return FINC_EINVAL;
    if (!disjoint(in, out))
        return FINC_EINVAL;
    if (V == 0)
        return FINC_OK;
    char *ws = (char *)workspace;
    auto take = [&](size_t bytes) {
        char *p = ws;
        ws += round256(bytes);
        return p;
    };
    unsigned *keys[2];
    int *at[2];
    for (int i = 0; i < 2; ++i) {
        keys[i] = (unsigned *)take((size_t)M * 4);
        at[i] = (int *)take((size_t)M * 4);
    }
    Sort o = {};
    o.ids = {ids, wide, V};
    o.counts = (int *)take((size_t)kMostBlocks * kDigits * 4);
    o.M = M;
    o.per = (int)cdivll(M, kMostBlocks);
    o.per = o.per < kSortBlock ? kSortBlock : o.per;
    o.blocks = (int)cdivll(M, o.per);
    int from = 0;
    if (M > 0 && M <= kShort) {
        o.key_out = keys[0];
        o.at_out = at[0];
        o.zeros = dtable;
        o.zero_count = (long long)V * D;
        sort_short_kernel<<<grid_of(1 + cdivll(o.zero_count, kZeroed)), kShortThreads, 0,
                            stream>>>(o);
    } else if (M > 0)
        for (o.shift = 0; o.shift < 32 && (o.shift == 0 || V >> o.shift); o.shift += 8) {
            o.key_out = keys[from ^ 1];
            o.at_out = at[from ^ 1];
            count_kernel<<<o.blocks, kThreads, 0, stream>>>(o);
            place_kernel<<<o.blocks, kThreads, 0, stream>>>(o);
            from ^= 1;
            o.key_in = keys[from];
            o.at_in = at[from];
        }
    Sum s = {};
    s.key = keys[from];
    s.at = at[from];
    s.dy = dy;
    s.sdy = sdy;
    s.dtable = dtable;
    s.tile = tile_of(M, D);
    s.tiles = tiles_of(M, D);
    s.head = (float *)take((size_t)s.tiles * D * 4);
    s.tail = (float *)take((size_t)s.tiles * D * 4);
    s.scale = (float)scale;
    s.M = M;
    s.V = V;
    s.D = D;
    s.lanes = lanes_of(D);
    s.slices = (D + s.lanes * kVec - 1) / (s.lanes * kVec);
    s.sum_blocks = cdivll((long long)s.tiles * s.slices, kThreads / s.lanes);
    const bool filled = M > 0 && M <= kShort;
    const long long blocks = s.sum_blocks + (filled ? 0 : cdivll(V, kFillRows * kWaves));
    with_type(type, [&](auto e) {
        sum_kernel<decltype(e)><<<grid_of(blocks), kThreads, 0, stream>>>(s);
    });
    if (s.tiles > 1)
        join_runs_kernel<<<grid_of((long long)s.tiles * s.slices), kThreads, 0, stream>>>(s);
    return launched();
}

}  // extern "C"
