// Range attention: how a call is cut and where its workspace lies, and the
// dispatch by row type (include/frog.h: frog_attend, frog_attend_backward).

#include <algorithm>

#include "attend_launch.h"
#include "attend_tile.h"

namespace frog {
namespace {

int64_t take(int64_t* at, int64_t bytes) {
    const int64_t here = *at;
    *at = (here + bytes + 255) / 256 * 256;
    return here;
}

int launched(const char* what, hipError_t e = hipGetLastError()) {
    return e == hipSuccess ? FROG_OK : fail(FROG_EHIP, "%s: %s", what, hipGetErrorString(e));
}

// (the kernels below take the number of their launch's first workgroup)
__global__ void copy_weights(const float* in, float* out, int64_t n, int64_t first) {
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
    if (i < n) out[i] = in ? in[i] : 0.f;
}

// a tensor of rows set to 0: [batch][tokens][heads][d values], pieces of 16 bytes
__global__ void clear_rows(char* p, int64_t s0, int64_t s1, int64_t s2, int64_t tokens, int heads, int pieces, int64_t total, int64_t first) {
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
    if (i >= total) return;
    const int c = (int)(i % pieces);
    const int64_t r = i / pieces, h = r % heads, t = r / heads % tokens, b = r / heads / tokens;
    *(uint4*)(p + b * s0 + t * s1 + h * s2 + 16 * c) = make_uint4(0, 0, 0, 0);
}

hipError_t clear(void* p, const int64_t (&st)[3], int64_t batch, int64_t tokens, int heads, int d, int size, hipStream_t s) {
    const int pieces = d * size / 16;
    const int64_t total = batch * tokens * heads * pieces, s0 = st[0] * size, s1 = st[1] * size, s2 = st[2] * size;
    return in_launches((total + 255) / 256, 256, [&](int64_t first, dim3 grid) { clear_rows<<<grid, 256, 0, s>>>((char*)p, s0, s1, s2, tokens, heads, pieces, total, first); });
}

}  // namespace

constexpr int64_t kCUs = 256;

// parts, at most `most`, of each of `blocks` workgroups until there are `want`
int parts_until(int64_t want, int64_t blocks, int64_t most) {
    return (int)std::max<int64_t>(1, std::min((want + blocks - 1) / std::max<int64_t>(blocks, 1), most));
}

// A few-rows pass over at most kWholeKeys keys that is not split: one launch
// instead of two, but a workgroup walks all keys of a kv head, and a CU takes in
// about 60 GB/s (fp32, whose workgroups have half the wavefronts: 40).  With 256
// workgroups or more that is at least as fast at every size (256 caches of 1,024
// keys, bf16, d = 128: 26 us, split 30).  With fewer it is as long as it takes no
// more than the host takes for two launches, 14 us: while the keys of a kv head
// are at most kWholeBytes (fp32: half of it).  us a call in a stream of calls,
// whole and split, and by the device alone, as in a replayed graph: bf16, d = 128,
// 512 keys 12.0, 14.0 and 9.1, 8.9; 1,001 keys 13.9, 14.8 and 13.4, 8.8 (what a
// program that replays graphs loses); 1,300 keys 18.2, 14.3; fp32, d = 128, 256 keys
// 13.7, 14.6 and 11.6, 11.8; 512 keys 20.0, 14.7 and 18.0, 11.8; 1,024 keys 31.3, 14.6.
// A shared prefix and a tail are two such passes: 4 requests over 700 and 60 keys,
// bf16, d = 128, 16.1, 16.2; over 900 and 60 18.0, 16.0.
constexpr int64_t kWholeKeys = 1024, kWholeBytes = 256 << 10, kWholeSharedBytes = 192 << 10;
bool whole_pays(int64_t keys, int64_t blocks, int d, int type, int64_t bytes) {
    return keys <= kWholeKeys && (blocks >= kCUs || keys * d * (type == FROG_STORAGE_F32 ? 8 : 2) <= bytes);
}

// Schedules are made where intervals may differ (lr), and a call is long enough
// for what they win: a workgroup's work is anything from one step to hundreds, and
// the longest one decides.  Sizes alone do not tell packed documents, which win,
// from windows and causal masks, which the order without a schedule serves as well
// (16-bit rows), so the bounds are set where documents win about what the others
// lose; a launch costs 6 to 10 us.  One sequence, bf16, d = 128, 16 query and 4 kv
// heads, forward and gradients, us with and without:
//   tokens     4,096              6,000              8,192               16,384
//   documents  68, 61; 216, 216   64, 70; 278, 299   105, 115; 432, 497  292, 312; 1,354, 1,546
//   causal     99, 97; 400, 392   166, 159; 697, 686 286, 293; 1,178, 1,196  1,048, 1,043; 4,566, 4,707
//   window     38, 32; 176, 166   52, 45; 244, 231   63, 56; 281, 262    111, 102; 504, 468
// The same lengths of narrower rows are worth less (d = 64, two sequences of 6,144
// tokens: 81, 85; 290, 333), fp32 rows some 16 times as much (4,096 tokens, d = 64:
// documents 134, 157; 434, 518, causal masks 325, 406; 1,207, 1,381): kScheduleWork
// in query-key pairs times d.  Short sequences balance by their number (4 of 3,000
// tokens: 85, 82; 345, 354).  One workgroup makes a schedule, so its tiles are
// bounded: of 64 sequences of 2,048 tokens it took 72 us of 500, of 4,096 half of
// 11 ms, of 8 of 8,192 (512 tiles of keys) as much as it won.
constexpr double kScheduleWork = 60e9;
constexpr int64_t kScheduleRowTiles = 1024, kScheduleKeyTiles = 256;
SchedulePlan schedule_plan(const frog_attend_t& a, int64_t tiles, int parts, int64_t least, int64_t most) {
    SchedulePlan p{};
    const bool f32 = a.type == FROG_STORAGE_F32;
    const int64_t length = std::min(a.keys, a.queries);
    if (!a.lr || length < (f32 ? 2048 : 4096) || a.batch * a.kv_heads * tiles < least || a.batch * tiles > most) return p;
    if ((double)a.batch * a.heads * length * length * a.d * (f32 ? 16 : 1) < kScheduleWork) return p;
    p.tiles = tiles;
    p.parts = parts;
    p.bytes = a.batch * tiles * 4;
    return p;
}
// Row tiles: above two workgroups for each CU, which start all at once (16-bit rows,
// 512 workgroups: 79 us with, 73 without).  fp32 workgroups differ by so much that
// one a CU is enough in the forward pass (256 workgroups, causal: 188, 224).
SchedulePlan schedule_rows_plan(const frog_attend_t& a, int64_t tiles, int parts, bool forward) {
    return schedule_plan(a, tiles, parts, a.type == FROG_STORAGE_F32 ? (forward ? kCUs : kCUs + 1) : 2 * kCUs + 1, kScheduleRowTiles);
}
// Key tiles are cut in parts: half a tile (fp32: a quarter) for each CU and more.
SchedulePlan schedule_keys_plan(const frog_attend_t& a, int64_t tiles, int parts) {
    return schedule_plan(a, tiles, parts, a.type == FROG_STORAGE_F32 ? kCUs / 4 : kCUs / 2 + 1, kScheduleKeyTiles);
}

ForwardPlan forward_plan(const frog_attend_t& a) {
    ForwardPlan p{};
    const int64_t group = a.heads / a.kv_heads, pairs = a.batch * a.kv_heads;
    p.rows = a.queries * group;
    p.few = p.rows <= 32;
    p.groups = p.rows <= 16 ? 1 : 2;
    p.tiles = (int)((p.rows + kTileRows - 1) / kTileRows);
    // parts of the keys until the card's 256 CUs have four workgroups each
    // (two of the larger tile's), none of less than a step of its wavefronts
    // (128 keys; 256 of the tiles', whose parts cost 4 D bytes a row)
    const int64_t blocks = pairs * (p.few ? 1 : p.tiles), want = p.few ? 4 * kCUs : 2 * kCUs, least = p.few ? 128 : 256;
    p.splits = parts_until(want, blocks, (a.keys + least - 1) / least);
    // (with key weights too, where a second launch follows in any case, so that
    // they do not change the output: 512 keys 17.3 us whole, 16.3 split)
    if (p.few && p.groups == 1 && whole_pays(a.keys, pairs, a.d, a.type, kWholeBytes)) p.splits = 1;
    if (!p.few) p.plan = schedule_rows_plan(a, p.tiles, p.splits, true);
    int64_t at = 0;
    p.plan.at = take(&at, p.plan.bytes);
    if (p.splits > 1) {
        p.o = take(&at, p.splits * pairs * p.rows * a.d * 4);
        p.ml = take(&at, p.splits * pairs * p.rows * 8);
    }
    if (a.w_out) {
        if (!a.lse) p.lse = take(&at, a.batch * a.heads * a.queries * 4);
        if (p.few) p.scores = take(&at, a.batch * a.heads * a.queries * a.keys * 4);
        else p.pack = take(&at, pack_plan(a, false).bytes);
    }
    p.bytes = at;
    return p;
}

PackPlan pack_plan(const frog_attend_t& a, bool grad) {
    PackPlan p{};
    p.tiles = (a.queries * (a.heads / a.kv_heads) + 31) / 32;
    // Parts of the query rows until there are four workgroups for each of the
    // 256 CUs, which hold two at a time, of 8 tiles at least: a workgroup's keys
    // see anything from all rows to a few (causal: the first keys twice the
    // mean).  Their fp32 sums cost 16 d bytes a key and part.  Two, four and eight
    // workgroups a CU, us a step, 16 and 4 heads of d = 128:
    //   tokens       4,096           8,192                 16,384
    //   causal       542, 483, 558   1,726, 1,441, 1,504   7,002, 5,599, 5,346
    //   documents    402, 347, 408   695, 541, 574         1,612, 1,163, 1,094
    //   window       179, 202, 267   302, 329, 402         516, 568, 640
    //   every key    722, 757, 869   2,638, 2,672, 2,794   10,234, 10,276, 10,489
    // Equal work pays 5 to 20 % for the others' gain; sizes do not tell them apart.
    const int64_t blocks = a.batch * a.kv_heads * ((a.keys + kTileRows - 1) / kTileRows);
    p.parts = parts_until(4 * kCUs, blocks, p.tiles / 8);
    const int64_t key_tiles = (a.keys + kTileRows - 1) / kTileRows, row_tiles = (p.tiles + 3) / 4;
    p.keys_plan = schedule_keys_plan(a, key_tiles, p.parts);
    if (grad) p.rows_plan = schedule_rows_plan(a, row_tiles, 1, false);
    int64_t at = 0;
    p.keys_plan.at = take(&at, p.keys_plan.bytes);
    p.rows_plan.at = take(&at, p.rows_plan.bytes);
    p.rows = take(&at, a.batch * a.kv_heads * p.tiles * 192 * 4);
    p.bounds = take(&at, a.batch * p.tiles * 16);
    p.zeros = take(&at, 512);
    if (p.parts > 1) p.o = take(&at, p.parts * a.batch * key_tiles * a.kv_heads * kTileRows * (grad ? 2 * a.d : 1) * 4);
    p.bytes = at;
    return p;
}

namespace {

// a pass without a query or without a key
bool empty(const frog_attend_t& a) { return a.batch == 0 || a.queries == 0 || a.keys == 0; }

template <typename F>
void by_type(int type, F&& f) {
    if (type == FROG_STORAGE_F32) f(AttendLaunch<float>{});
    else if (type == FROG_STORAGE_F16) f(AttendLaunch<f16_t>{});
    else f(AttendLaunch<bf16_t>{});
}

// A launch takes fewer than 2^32 threads.  (Joining passes are not looked at:
// an axis is cut only where there are a few hundred workgroups.)
int check_grid(int64_t blocks, int threads = 256) {
    return blocks > 0xffffffffll / threads ? fail(FROG_EUNSUPPORTED, "%lld workgroups of %d threads: more than one launch takes", (long long)blocks, threads) : FROG_OK;
}

// the passes that own keys
int check_keys(const frog_attend_t& a, const PackPlan& p) {
    const int64_t pairs = a.batch * a.kv_heads;
    return check_grid(std::max((pairs * p.tiles + 3) / 4, pairs * ((a.keys + kTileRows - 1) / kTileRows) * p.parts));
}

int check_forward(const frog_attend_t& a, const ForwardPlan& p) {
    const int64_t pairs = a.batch * a.kv_heads;
    int rc = p.few ? check_grid(pairs * p.splits, 512) : check_grid(pairs * p.splits * p.tiles);
    if (rc != FROG_OK || !a.w_out) return rc;
    return p.few ? check_grid((pairs * p.rows + 3) / 4 + (a.keys + 255) / 256 * pairs) : check_keys(a, pack_plan(a, false));
}

int check_backward(const frog_attend_t& a, const PackPlan& p) {
    const int64_t rows = a.queries * (a.heads / a.kv_heads);
    int rc = check_grid(a.batch * a.kv_heads * ((rows + kTileRows - 1) / kTileRows));
    return rc != FROG_OK ? rc : check_keys(a, p);
}

int check_shared(const frog_attend_shared_t& a, const SharedPlan& p) {
    int rc = check_grid(p.tail_blocks + (p.few ? (int64_t)a.kv_heads * p.head_splits : 0), p.whole ? 512 : 256);
    if (rc == FROG_OK && !p.whole && !p.few) rc = check_grid((int64_t)a.kv_heads * p.head_splits * p.tiles);
    return rc != FROG_OK || p.whole ? rc : check_grid((a.batch * a.heads + 3) / 4);
}

__global__ void fill_lse(float* lse, int64_t n, int64_t first) {
    const int64_t i = (first + blockIdx.x) * 256 + threadIdx.x;
    if (i < n) lse[i] = -INFINITY;
}

}  // namespace

namespace {

// Tiles longest first, by one workgroup counting in 1,024 classes of equal width
// (of a class in any order: it changes no result).  The workgroups of the first
// `wave` tiles take a CU each; those of the next `wave`, which join them there,
// come shortest first, so that the CU with the longest gets the shortest beside
// it.  length(tile) is called by whole wavefronts (WAVE) or by single threads.
constexpr int kSortBlock = 1024;
template <bool WAVE, typename F>
__device__ inline void longest_first(int tiles, int wave, int* order, F&& length) {
    __shared__ int held[kScheduleRowTiles], hist[kSortBlock], wave_sum[kSortBlock / 64], most;
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int first = WAVE ? w : t, step = WAVE ? kSortBlock / 64 : kSortBlock;
    const bool writes = !WAVE || lane == 0;
    hist[t] = 0;
    if (t == 0) most = 1;
    __syncthreads();
    int top = 0;
    for (int i = first; i < tiles; i += step) {
        const int n = length(i);
        if (writes) held[i] = n;          // read back by the same thread
        top = max(top, n);
    }
    if (writes) atomicMax(&most, top);
    __syncthreads();
    const float scale = (float)(kSortBlock - 1) / (float)most;
    auto bin = [&](int i) {
        return kSortBlock - 1 - min((int)((float)held[i] * scale), kSortBlock - 1);
    };
    if (writes)
        for (int i = first; i < tiles; i += step) atomicAdd(&hist[bin(i)], 1);
    __syncthreads();
    const int own = hist[t];
    int x = own;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 63) wave_sum[w] = x;
    __syncthreads();
    for (int i = 0; i < w; ++i) x += wave_sum[i];
    hist[t] = x - own;
    __syncthreads();
    if (writes)
        for (int i = first; i < tiles; i += step) {
            const int at = atomicAdd(&hist[bin(i)], 1), end = min(2 * wave, tiles);
            order[at >= wave && at < end ? wave + end - 1 - at : at] = i;
        }
}

// Lengths of row tiles: the keys from the first to the last that the first,
// middle and last token of a tile see.
__global__ __launch_bounds__(kSortBlock) void schedule_row_tiles(frog_attend_t a, int group, int tiles, int wave, int* order) {
    longest_first<false>((int)a.batch * tiles, wave, order, [&](int item) {
        const int64_t b = item / tiles, rows = a.queries * group, r0 = (int64_t)(item % tiles) * kTileRows, r1 = min(rows, r0 + kTileRows) - 1;
        const int64_t t0 = r0 / group, t1 = r1 / group, tokens[3] = {t0, (t0 + t1) / 2, t1};
        int first = INT_MAX, last = -1;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            int lo, hi;
            interval(a, b, tokens[i], &lo, &hi);
            if (lo > hi) continue;
            first = min(first, lo);
            last = max(last, hi);
        }
        return last < 0 ? 0 : last - first + 1;
    });
}

// Lengths of key tiles: how many of at most 256 of the sequence's row tiles
// (evenly spread) see one of its keys.
__global__ __launch_bounds__(kSortBlock) void schedule_key_tiles(frog_attend_t a, int tiles, const int4* bounds, int row_tiles, int wave, int* order) {
    const int lane = threadIdx.x & 63, stride = (row_tiles + 255) / 256;
    longest_first<true>((int)a.batch * tiles, wave, order, [&](int item) {
        const int4* of = bounds + (int64_t)(item / tiles) * row_tiles;
        const int first = item % tiles * kTileRows, last = (int)min((int64_t)first + kTileRows, a.keys) - 1;
        int n = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t t = (int64_t)(u * 64 + lane) * stride;
            const int4 bd = of[min(t, (int64_t)row_tiles - 1)];
            n += __popcll(__ballot(t < row_tiles && bd.x <= last && bd.y >= first));
        }
        return n;
    });
}

}  // namespace

// tiles whose workgroups (of all kv heads) are one for each of the 256 CUs; all of
// them where a CU holds one workgroup (shortest first after the longest, a causal
// pass of 4,096 fp32 tokens, d = 128, took 770 us instead of 639)
static int cu_tiles(const frog_attend_t& a, const SchedulePlan& p, bool alone) {
    return alone ? (int)(a.batch * p.tiles) : (int)std::max<int64_t>(1, kCUs / ((int64_t)a.kv_heads * p.parts));
}

void schedule_rows(const frog_attend_t& a, const SchedulePlan& p, bool alone, char* ws, hipStream_t s) {
    schedule_row_tiles<<<dim3(1), kSortBlock, 0, s>>>(a, a.heads / a.kv_heads, (int)p.tiles, cu_tiles(a, p, alone), (int*)(ws + p.at));
}

void schedule_keys(const frog_attend_t& a, const SchedulePlan& p, bool alone, const int4* bounds, int row_tiles, char* ws, hipStream_t s) {
    schedule_key_tiles<<<dim3(1), kSortBlock, 0, s>>>(a, (int)p.tiles, bounds, row_tiles, cu_tiles(a, p, alone), (int*)(ws + p.at));
}

int64_t attend_ws(const frog_attend_t& a) {
    if (empty(a)) return 0;
    const ForwardPlan p = forward_plan(a);
    const int rc = check_forward(a, p);
    return rc != FROG_OK ? rc : p.bytes;
}

int launch_attend(const frog_attend_t& a, void* ws, hipStream_t stream) {
    const int size = a.type == FROG_STORAGE_F32 ? 4 : 2;
    if (empty(a)) {
        const int64_t rows = a.batch * a.heads * a.queries, cols = a.batch * a.kv_heads * a.keys;
        hipError_t e = clear(a.out, a.out_stride, a.batch, a.queries, a.heads, a.d, size, stream);
        if (e == hipSuccess && a.out_low && size == 2) e = clear(a.out_low, a.out_stride, a.batch, a.queries, a.heads, a.d, size, stream);
        if (e == hipSuccess && a.lse) e = in_launches((rows + 255) / 256, 256, [&](int64_t first, dim3 grid) { fill_lse<<<grid, 256, 0, stream>>>(a.lse, rows, first); });
        if (e == hipSuccess && a.w_out && a.w_out != a.w_in)
            e = in_launches((cols + 255) / 256, 256, [&](int64_t first, dim3 grid) { copy_weights<<<grid, 256, 0, stream>>>(a.w_in, a.w_out, cols, first); });
        return launched("attention launch", e);
    }
    const ForwardPlan p = forward_plan(a);
    by_type(a.type, [&](auto l) { l.forward(a, p, (char*)ws, stream); });
    return launched("attention launch");
}

int64_t attend_bwd_ws(const frog_attend_t& a) {
    if (empty(a)) return 0;
    const PackPlan p = pack_plan(a, true);
    const int rc = check_backward(a, p);
    return rc != FROG_OK ? rc : p.bytes;
}

int launch_attend_bwd(const frog_attend_t& a, void* ws, hipStream_t stream) {
    const int size = a.type == FROG_STORAGE_F32 ? 4 : 2;
    if (empty(a)) {
        hipError_t e = clear(a.dq, a.dq_stride, a.batch, a.queries, a.heads, a.d, size, stream);
        if (e == hipSuccess) e = clear(a.dk, a.dk_stride, a.batch, a.keys, a.kv_heads, a.d, size, stream);
        if (e == hipSuccess) e = clear(a.dv, a.dv_stride, a.batch, a.keys, a.kv_heads, a.d, size, stream);
        return launched("attention gradient launch", e);
    }
    by_type(a.type, [&](auto l) { l.backward(a, (char*)ws, stream); });
    return launched("attention gradient launch");
}

SharedPlan shared_plan(const frog_attend_shared_t& a) {
    SharedPlan p{};
    const int64_t group = a.heads / a.kv_heads, rows = a.batch * group, all = a.batch * a.heads;
    const int64_t most = a.pages_per_request * a.page;
    const int whole_groups = group <= 16 ? 1 : 2;
    const int64_t whole_blocks = a.batch * a.kv_heads * ((group + 16 * whole_groups - 1) / (16 * whole_groups));
    // (the prefix of more than 32 rows would take tiles, one more launch: 16
    // requests over 900 and 60 keys, bf16, d = 128: 18.6 us whole, 23.6 in parts)
    if (a.prefix + most <= kWholeKeys && a.batch * a.prefix <= 16 * kWholeKeys &&
        ((a.prefix > 0 && rows > 32) || whole_pays(a.prefix + most, whole_blocks, a.d, a.type, kWholeSharedBytes))) {
        p.whole = true;
        p.groups = whole_groups;
        p.tail_blocks = whole_blocks;
        return p;
    }
    // parts as in forward_plan
    if (a.prefix > 0) {
        p.few = rows <= 32;
        p.tiles = (int)((rows + kTileRows - 1) / kTileRows);
        const int64_t blocks = (int64_t)a.kv_heads * (p.few ? 1 : p.tiles), want = p.few ? 4 * kCUs : 2 * kCUs, least = p.few ? 128 : 256;
        p.head_splits = parts_until(want, blocks, (a.prefix + least - 1) / least);
    }
    p.groups = std::max(p.few ? rows : 0, std::min<int64_t>(group, 32)) <= 16 ? 1 : 2;
    if (most > 0) {
        const int64_t blocks = a.batch * a.kv_heads * ((group + 16 * p.groups - 1) / (16 * p.groups));
        p.tail_splits = parts_until(4 * kCUs, blocks, (most + 127) / 128);
        p.tail_blocks = blocks * p.tail_splits;
    }
    int64_t at = 0;
    p.ho = take(&at, p.head_splits * all * a.d * 4);
    p.hml = take(&at, p.head_splits * all * 8);
    p.to = take(&at, p.tail_splits * all * a.d * 4);
    p.tml = take(&at, p.tail_splits * all * 8);
    if (a.slopes && p.head_splits && !p.few) {
        p.at_q = take(&at, a.batch * 4);
        p.at_k = take(&at, a.prefix * 4);
    }
    p.bytes = at;
    return p;
}

int64_t attend_shared_ws(const frog_attend_shared_t& a) {
    if (a.batch == 0) return 0;
    const SharedPlan p = shared_plan(a);
    const int rc = check_shared(a, p);
    return rc != FROG_OK ? rc : p.bytes;
}

int launch_attend_shared(const frog_attend_shared_t& a, void* ws, hipStream_t stream) {
    if (a.batch == 0) return FROG_OK;
    const SharedPlan p = shared_plan(a);
    by_type(a.type, [&](auto l) { l.shared(a, p, (char*)ws, stream); });
    return launched("shared attention launch");
}

}  // namespace frog
