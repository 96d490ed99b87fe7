// bp_evict_by_weight: lists over their budget lose the entries of the lowest accumulated weight.
#include <algorithm>

#include "common.h"

namespace bp {
namespace {

constexpr int64_t kMaxLists = int64_t(1) << 24;

struct EvictArgs {
    const int64_t* bag_off;
    const int32_t* bag_len;
    int64_t n, bags;
    int32_t budget, sinks, recent;
    const float* weight;
    const int64_t* ids;
    const int32_t *slots, *pos;
    float* kept_weight;
    int64_t* kept_ids;
    int32_t *kept_slots, *kept_pos, *kept_len;
    int64_t* evict_ids;
    int32_t* evict_slots;
    int64_t list_capacity;
    int64_t* evict_off;
    int32_t scanned;               // evict_off is there already
    int32_t split;                 // lists are taken by pieces of kPiece entries, else whole
    uint32_t parts;                // pieces, or lists
    struct Choice* choice;         // [parts]
    uint2* begins;                 // [parts][kStretches]: ties, and entries that leave, of the list before a stretch
    uint32_t* hist;                // [parts][kDigits][kBins] of lists of several pieces
};

// The entries [first, first + count) of a list; offsets and lengths that point outside the arrays use nothing there.
__device__ __forceinline__ void list_span(const EvictArgs& a, int64_t bag, int64_t* first, int64_t* count) {
    int64_t f = a.bag_off[bag], e = a.bag_off[bag + 1];
    if (f < 0) f = 0;
    if (e > a.n) e = a.n;
    int64_t c = e > f ? e - f : 0;
    if (a.bag_len) {
        const int64_t used = a.bag_len[bag];
        if (used < c) c = used > 0 ? used : 0;
    }
    *first = f;
    *count = c;
}

// Weights as unsigned keys of the same order: -0 as 0, NaN above everything.
__device__ __forceinline__ uint32_t weight_key(float w) {
    if (w != w) return 0xffffffffu;
    const uint32_t u = __float_as_uint(w + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// ---- selection -----------------------------------------------------------------------------------------------------------
// The weight up to which a list's entries leave is found eleven bits at a time by counting.  A workgroup takes a list, whose keys
// stay in its registers (up to 32 a thread, so the list is read once; longer ones are read again for every digit); or, where
// lists are long, a piece of one, and the pieces of a list meet over three launches, each of which adds up the counts that the
// one before left.  A wavefront's entries lie side by side, 64 a step: its stretch.
constexpr int kDigits = 3, kBins = 2048, kStretches = 16;
constexpr int kPieceShift = 15, kPiece = 1 << kPieceShift;        // what 1,024 threads hold
constexpr int kShift[kDigits] = {21, 10, 0}, kWidth[kDigits] = {11, 11, 10};

constexpr int kFew = 8;           // up to so many leave: found one by one, a barrier each (of 1,025 entries one: 8.7 us, four 11.0, eight
                                  // 14.1, sixteen 20.1), instead of the digits' nine (14.1 to 14.6)

struct Choice {
    uint32_t key;             // the largest key that leaves
    uint32_t ties;            // how many of the entries with that key leave: the earliest
    int64_t before;           // entries that leave earlier lists
};

// What a workgroup works on: a list, or a piece of one.
struct Part {
    int64_t bag, first;             // the list
    int32_t count;
    int32_t begin, end;             // the part's places in it
    uint32_t first_id, of, number;  // the list's parts
};
__device__ __forceinline__ uint32_t first_part(const EvictArgs& a, int64_t bag) {
    int64_t at = a.bag_off[bag];
    if (at < 0) at = 0;
    if (at > a.n) at = a.n;
    return (uint32_t)(at >> kPieceShift) + (uint32_t)bag;
}
__device__ __forceinline__ Part find_part(const EvictArgs& a, uint32_t id) {
    Part p;
    p.first = 0;
    p.count = p.begin = p.end = 0;
    p.bag = id;
    p.first_id = id;
    p.of = 1;
    p.number = 0;
    if (id >= a.parts || a.bags == 0) {
        p.bag = a.bags;
        return p;
    }
    if (a.split) {                    // the last list that begins no later, 64 lists a step
        const uint32_t lane = threadIdx.x % 64;
        uint32_t lo = 0, hi = (uint32_t)a.bags;
        while (hi - lo > 1) {
            const uint32_t step = (hi - lo + 63) / 64, i = lo + (lane + 1) * step;
            lo += __popcll(__ballot(i < hi && first_part(a, i) <= id)) * step;
            hi = min(hi, lo + step);
        }
        p.bag = lo;
        p.first_id = first_part(a, lo);
        p.number = id - p.first_id;
    }
    int64_t count;
    list_span(a, p.bag, &p.first, &count);
    p.count = p.end = (int32_t)count;
    if (a.split) {
        p.of = (uint32_t)max(int64_t(1), min((count + kPiece - 1) >> kPieceShift, (int64_t)a.parts - p.first_id));
        if (p.number >= p.of) {
            p.begin = p.count;                                    // a number without a piece
        } else {
            p.begin = (int32_t)(p.number << kPieceShift);
            if (p.number + 1 < p.of) p.end = p.begin + kPiece;
        }
    }
    return p;
}

// Sum over the workgroup of v over the threads before this one, and over all.
template <int BLOCK>
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t* waves, uint32_t* all) {
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t upto = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const uint32_t x = __shfl_up(upto, off);
        if (lane >= off) upto += x;
    }
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    uint32_t before = upto - v, total = 0;
#pragma unroll
    for (int w = 0; w < BLOCK / 64; ++w) {
        if (w < wave) before += waves[w];
        total += waves[w];
    }
    *all = total;
    return before;
}

// The digit in which the need-th smallest key lies, and how many are left to count in it (into LDS; read behind a barrier).
template <int BLOCK>
__device__ __forceinline__ void find_digit(const uint32_t (&c)[kBins / BLOCK], uint32_t need, uint32_t* waves, uint32_t* found, uint32_t* rest) {
    uint32_t sum = 0, all;
#pragma unroll
    for (int i = 0; i < kBins / BLOCK; ++i) sum += c[i];
    uint32_t before = sum_before<BLOCK>(sum, waves, &all);
    if (before < need && need <= before + sum) {                   // one thread
#pragma unroll
        for (int i = 0; i < kBins / BLOCK; ++i) {
            if (before < need && need <= before + c[i]) {
                *found = (kBins / BLOCK) * threadIdx.x + i;
                *rest = need - before;
            }
            before += c[i];
        }
    }
}

// ---- what stays and what leaves, of one wavefront's stretch ------------------------------------------------------------------
// Ranks are popcounts of ballots; kAhead steps' loads are in flight together.  Places are unsigned here and wherever steps of 64 go past
// a stretch's end: a list may end at 2^31 - 1.
constexpr int kAhead = 4;
__device__ __forceinline__ void move_stretch(const EvictArgs& a, const Part& p, const Choice& c, uint32_t begin, uint32_t end, uint32_t tie, uint32_t gone) {
    const int lane = threadIdx.x % 64;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    const bool over = p.count > a.budget;
    const uint32_t may0 = a.sinks, may1 = over ? p.count - a.recent : 0;
    for (uint32_t e0 = begin; e0 < end; e0 += 64 * kAhead) {
        float w[kAhead];
        int64_t id[kAhead];
        int32_t slot[kAhead], pos[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t e = e0 + i * 64 + lane;
            const int64_t from = p.first + e;
            if (e >= end) continue;
            w[i] = a.weight[from];
            id[i] = a.ids ? a.ids[from] : 0;
            slot[i] = a.slots[from];
            pos[i] = a.pos ? a.pos[from] : 0;
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const uint32_t e = e0 + i * 64 + lane;
            const bool in = e < end, may = over && in && e >= may0 && e < may1;
            const uint32_t k = weight_key(w[i]);
            const uint64_t ties = __ballot(may && k == c.key);
            const bool leaves = may && (k < c.key || (k == c.key && tie + __popcll(ties & below) < c.ties));
            const uint64_t leaving = __ballot(leaves);
            const uint32_t left = gone + __popcll(leaving & below);        // entries of the list that leave before this one
            if (leaves) {
                const int64_t to = c.before + left;
                if (to < a.list_capacity) {
                    if (a.evict_ids) a.evict_ids[to] = id[i];
                    a.evict_slots[to] = slot[i];
                }
            } else if (in) {
                const int64_t to = p.first + e - left;
                if (a.kept_weight) a.kept_weight[to] = w[i];
                if (a.kept_ids) a.kept_ids[to] = id[i];
                a.kept_slots[to] = slot[i];
                if (a.kept_pos) a.kept_pos[to] = pos[i];
            }
            tie += __popcll(ties);
            gone += __popcll(leaving);
        }
    }
}

// The evict lists behind the last entry, a share a workgroup.
template <int BLOCK>
__device__ __forceinline__ void clear_rest(const EvictArgs& a, int64_t all) {
    for (int64_t e = all + (int64_t)blockIdx.x * BLOCK + threadIdx.x; e < a.list_capacity; e += (int64_t)gridDim.x * BLOCK) {
        if (a.evict_ids) a.evict_ids[e] = -1;
        a.evict_slots[e] = -1;
    }
}

template <int BLOCK>
struct Stretch {
    int steps;
    uint32_t begin, end;
    __device__ __forceinline__ Stretch(const Part& p, int wave) {
        const int places = p.end - p.begin;
        steps = places / BLOCK + (places % BLOCK != 0);
        begin = p.begin + (uint32_t)min((int64_t)places, (int64_t)wave * steps * 64);
        end = (uint32_t)min((int64_t)p.end, (int64_t)begin + steps * 64);
    }
};

// PASS 0: offsets, lengths, the evict lists' rest, and the first digit; lists of one part go on to the end.  PASS 1, 2: the next digits
// of lists of several pieces; PASS 3: their ranks.  FUSED: entries are moved here too (lists of one part).
template <int BLOCK, bool FUSED, int PASS>
__global__ __launch_bounds__(BLOCK) void evict_select_kernel(EvictArgs a) {
    constexpr int kHeld = BLOCK == 1024 ? 32 : 16, WAVES = BLOCK / 64, COPIES = BLOCK == 1024 ? 4 : 2, PER = kBins / BLOCK;
    __shared__ uint32_t hist[COPIES][kBins + 1], found, rest, waves[WAVES];
    __shared__ uint32_t counts[2][WAVES];
    __shared__ int64_t sums[2][WAVES];
    __shared__ uint64_t lows[2][WAVES];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const Part p = find_part(a, blockIdx.x);
    if (PASS > 0 && (p.of == 1 || p.number >= p.of)) return;
    const int over = max(0, p.count - a.budget);
    const Stretch<BLOCK> mine(p, wave);
    const bool held = mine.steps <= kHeld;
    uint32_t key[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const uint32_t e = mine.begin + i * 64 + lane;
        key[i] = over && held && e < mine.end ? weight_key(a.weight[p.first + e]) : 0;
    }
    Choice c{0, (uint32_t)over, 0};
    if (PASS == 0) {
        // what leaves the lists before this one, and all lists
        int64_t before = 0, all = 0;
        if (a.scanned) {
            before = a.evict_off[min(p.bag, a.bags)];
            all = a.evict_off[a.bags];
        } else {
            for (int64_t b = threadIdx.x; b < a.bags; b += BLOCK) {
                int64_t f, n;
                list_span(a, b, &f, &n);
                const int64_t o = max(int64_t(0), n - a.budget);
                all += o;
                if (b < p.bag) before += o;
            }
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) {
                before += __shfl_xor(before, off);
                all += __shfl_xor(all, off);
            }
            if (lane == 0) {
                sums[0][wave] = before;
                sums[1][wave] = all;
            }
            __syncthreads();
            before = all = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                before += sums[0][w];
                all += sums[1][w];
            }
            if (threadIdx.x == 0 && p.bag < a.bags && p.number == 0) a.evict_off[p.bag] = before;
            if (threadIdx.x == 0 && blockIdx.x == 0) a.evict_off[a.bags] = all;
        }
        c.before = before;
        if (threadIdx.x == 0 && p.bag < a.bags && p.number == 0) a.kept_len[p.bag] = (int32_t)(p.count - over);
        if (FUSED) clear_rest<BLOCK>(a, all);
        if (p.begin >= p.end) return;
    } else {
        c = a.choice[blockIdx.x];
    }
    const int may0 = a.sinks, may1 = p.count - a.recent;
    // f(place, key) for the stretch, 64 places at a time; places past its end come as the list's length
    const auto each = [&](auto&& f) {
        const uint32_t end = mine.end;
        if (held) {
#pragma unroll
            for (int i = 0; i < kHeld; ++i)
                if (i < mine.steps) {
                    const uint32_t e = mine.begin + i * 64 + lane;
                    f(e < end ? (int)e : p.count, key[i]);
                }
        } else {
            for (uint32_t e = mine.begin + lane; e - lane < end; e += 64) f(e < end ? (int)e : p.count, e < end ? weight_key(a.weight[p.first + e]) : 0u);
        }
    };
    const auto count_digit = [&](int digit) {
        for (int i = threadIdx.x; i < COPIES * (kBins + 1); i += BLOCK) (&hist[0][0])[i] = 0;
        __syncthreads();
        const int shift = kShift[digit], above = shift + kWidth[digit];
        each([&](int e, uint32_t k) {
            if (e >= may0 && e < may1 && (digit == 0 || (k ^ c.key) >> above == 0)) atomicAdd(&hist[lane % COPIES][k >> shift & ((1 << kWidth[digit]) - 1)], 1u);
        });
        __syncthreads();
    };
    const auto take_digit = [&](int digit, const uint32_t (&n)[PER]) {
        find_digit<BLOCK>(n, c.ties, waves, &found, &rest);
        __syncthreads();
        c.key |= found << kShift[digit];
        c.ties = rest;
    };
    uint32_t tie = 0, gone = 0;                       // of the list, before this part
    if (over && p.of == 1 && over <= kFew) {          // one after the other: the lowest key, of those the earliest place
        uint64_t last = 0;
        c.ties = 0;
        for (int round = 0; round < over; ++round) {
            uint64_t low = ~uint64_t(0);
            each([&](int e, uint32_t k) {
                const uint64_t v = (uint64_t)k << 32 | (uint32_t)e;
                if (e >= may0 && e < may1 && (round == 0 || v > last)) low = min(low, v);
            });
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) low = min(low, (uint64_t)__shfl_xor(low, off));
            if (lane == 0) lows[round % 2][wave] = low;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) low = min(low, lows[round % 2][w]);
            c.ties = round > 0 && (uint32_t)(low >> 32) == (uint32_t)(last >> 32) ? c.ties + 1 : 1;
            last = low;
        }
        c.key = (uint32_t)(last >> 32);
    } else if (over && p.of == 1) {
#pragma unroll
        for (int digit = 0; digit < kDigits; ++digit) {
            count_digit(digit);
            uint32_t n[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                n[i] = 0;
#pragma unroll
                for (int k = 0; k < COPIES; ++k) n[i] += hist[k][PER * threadIdx.x + i];
            }
            take_digit(digit, n);
        }
    }
    if (over && p.of > 1) {
        if (PASS > 0) {                               // the digit that the pass before counted, over the list's pieces
            uint32_t n[PER], mine_before = 0, all;
#pragma unroll
            for (int i = 0; i < PER; ++i) n[i] = 0;
            for (uint32_t q = 0; q < p.of; ++q) {
                const uint32_t* const h = a.hist + ((int64_t)(p.first_id + q) * kDigits + PASS - 1) * kBins + PER * threadIdx.x;
#pragma unroll
                for (int i = 0; i < PER; ++i) n[i] += h[i];
            }
            take_digit(PASS - 1, n);
            if (PASS == kDigits) {                    // entries of the pieces before that have a lower key, or the same
                for (uint32_t q = 0; q < p.number; ++q)
#pragma unroll
                    for (int d = 0; d < kDigits; ++d) {
                        const uint32_t* const h = a.hist + ((int64_t)(p.first_id + q) * kDigits + d) * kBins;
                        const uint32_t digit = c.key >> kShift[d] & ((1 << kWidth[d]) - 1);
                        for (uint32_t i = threadIdx.x; i < digit; i += BLOCK) mine_before += h[i];
                        if (d == kDigits - 1) tie += h[digit];
                    }
                __syncthreads();
                sum_before<BLOCK>(mine_before, waves, &all);
                gone = all;
                __syncthreads();
            }
        }
        if (PASS < kDigits) {
            count_digit(PASS);
            for (int i = threadIdx.x; i < kBins; i += BLOCK) {
                uint32_t n = 0;
#pragma unroll
                for (int k = 0; k < COPIES; ++k) n += hist[k][i];
                a.hist[((int64_t)blockIdx.x * kDigits + PASS) * kBins + i] = n;
            }
            if (threadIdx.x == 0) a.choice[blockIdx.x] = c;
            return;
        }
    }
    // ranks: ties before this wavefront, and what leaves before it
    uint32_t n_tie = 0, n_less = 0;
    if (over)
        each([&](int e, uint32_t k) {
            const bool may = e >= may0 && e < may1;
            n_tie += __popcll(__ballot(may && k == c.key));
            n_less += __popcll(__ballot(may && k < c.key));
        });
    if (lane == 0) {
        counts[0][wave] = n_tie;
        counts[1][wave] = n_less;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        tie += counts[0][w];
        gone += counts[1][w];
    }
    gone += min(tie, c.ties);
    if (FUSED) {
        move_stretch(a, p, c, mine.begin, mine.end, tie, gone);
    } else {
        if (lane == 0) a.begins[(int64_t)blockIdx.x * kStretches + wave] = make_uint2(tie, gone);
        if (threadIdx.x == 0) a.choice[blockIdx.x] = c;
    }
}

// A wavefront a stretch of 1,024 threads' selection.
constexpr int kMoveBlock = 256;
__global__ __launch_bounds__(kMoveBlock) void evict_move_kernel(EvictArgs a) {
    const uint32_t job = blockIdx.x * (kMoveBlock / 64) + threadIdx.x / 64, part = job / kStretches;
    const Part p = find_part(a, part);
    const Stretch<1024> mine(p, job % kStretches);
    clear_rest<kMoveBlock>(a, a.evict_off[a.bags]);
    if (mine.begin >= mine.end) return;
    const Choice c = a.choice[part];
    const uint2 b = a.begins[job];
    move_stretch(a, p, c, mine.begin, mine.end, b.x, b.y);
}

// Offsets of the evict lists where there are too many lists for every workgroup to add them up.
__global__ __launch_bounds__(1024) void evict_scan_kernel(EvictArgs a) {
    __shared__ int64_t sums[16];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int64_t total = 0;
    for (int64_t b0 = 0; b0 < a.bags; b0 += 1024) {
        const int64_t b = b0 + threadIdx.x;
        int64_t f, n = 0;
        if (b < a.bags) list_span(a, b, &f, &n);
        const int64_t o = max(int64_t(0), n - a.budget);
        int64_t upto = o;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int64_t x = __shfl_up(upto, off);
            if (lane >= off) upto += x;
        }
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        int64_t before = total + upto - o;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            if (w < wave) before += sums[w];
            total += sums[w];
        }
        if (b < a.bags) a.evict_off[b] = before;
        __syncthreads();
    }
    if (threadIdx.x == 0) a.evict_off[a.bags] = total;
}

constexpr int64_t kManyLists = 4096;
// Lists of up to 2,048 entries in the mean: 256 threads a list, one launch.  Longer ones: 1,024 threads choose, and a second launch
// moves, 16 wavefronts a list wherever there is room (lists of 4,000: 512 of them 23 us in one launch and 30 in two, 32 of them 11.3 and
// 10.2; of 64 of 16,000 the longest would hold a CU up while others have none).  From 16,384 on (a workgroup holds twice that) by pieces
// (64 of 22,000: 31 us, whole 42; 8 of 31,000: 32 and 43).
bool lists_short(int64_t n, int64_t bags) { return n <= 2048 * std::max<int64_t>(bags, 1); }
bool lists_long(int64_t n, int64_t bags) { return n > (kPiece / 2) * std::max<int64_t>(bags, 1) && n > kPiece; }

struct EvictScratch {
    Choice* choice;
    uint2* begins;
    uint32_t* hist;
    size_t bytes;
    EvictScratch(void* ws, int64_t n, int64_t bags) {
        // room for any n and number of lists up to these
        const int64_t pieces = (n >> kPieceShift) + std::min(bags, (n >> (kPieceShift - 1)) + 1), whole = std::min(bags, n / 2048 + 1);
        Carver c(ws, 0);
        choice = c.take<Choice>((size_t)std::max(pieces, whole));
        begins = c.take<uint2>((size_t)std::max(pieces, whole) * kStretches);
        hist = c.take<uint32_t>(n > kPiece ? (size_t)pieces * kDigits * kBins : 0);
        bytes = c.used();
    }
};

int launch_evict(EvictArgs a, hipStream_t stream) {
    a.scanned = a.bags > kManyLists;
    if (a.scanned) BP_LAUNCH(K_EVICT_SELECT, evict_scan_kernel, dim3(1), dim3(1024), 0, stream, a);
    a.split = lists_long(a.n, a.bags);
    a.parts = (uint32_t)(a.split ? (a.n >> kPieceShift) + a.bags : a.bags);
    const unsigned parts = std::max(a.parts, 1u);
    // enough workgroups for the evict lists' rest, too
    const auto grid = [&](int64_t groups, int block) { return dim3((unsigned)std::max(groups, std::min<int64_t>(ceil_div(a.list_capacity, 8 * block), 1024))); };
    if (lists_short(a.n, a.bags)) {
        BP_LAUNCH(K_EVICT_SELECT, (evict_select_kernel<256, true, 0>), grid(parts, 256), dim3(256), 0, stream, a);
        return BP_OK;
    }
    BP_LAUNCH(K_EVICT_SELECT, (evict_select_kernel<1024, false, 0>), dim3(parts), dim3(1024), 0, stream, a);
    if (a.split) {
        BP_LAUNCH(K_EVICT_SELECT, (evict_select_kernel<1024, false, 1>), dim3(a.parts), dim3(1024), 0, stream, a);
        BP_LAUNCH(K_EVICT_SELECT, (evict_select_kernel<1024, false, 2>), dim3(a.parts), dim3(1024), 0, stream, a);
        BP_LAUNCH(K_EVICT_SELECT, (evict_select_kernel<1024, false, 3>), dim3(a.parts), dim3(1024), 0, stream, a);
    }
    BP_LAUNCH(K_EVICT_MOVE, evict_move_kernel, grid(ceil_div((int64_t)parts * kStretches, kMoveBlock / 64), kMoveBlock), dim3(kMoveBlock), 0, stream, a);
    return BP_OK;
}

}  // namespace
}  // namespace bp

using namespace bp;

BP_EXPORT int bp_evict_by_weight_workspace_bytes(int64_t n, int64_t bags, size_t* bytes) {
    if (!bytes) return fail(BP_ERR_INVALID_ARG, "bytes is NULL");
    if (n < 0 || bags < 0) return fail(BP_ERR_INVALID_ARG, "negative size");
    if (n >= (int64_t(1) << 31) || bags >= kMaxLists) return fail(BP_ERR_UNSUPPORTED, "n >= 2^31 or bags >= 2^24");
    *bytes = EvictScratch(nullptr, n, bags).bytes;
    return BP_OK;
}

BP_EXPORT int bp_evict_by_weight(const int64_t* bag_offsets, const int32_t* bag_lengths, int64_t n, int64_t bags, int32_t budget, int32_t sinks,
                                 int32_t recent, const float* weight, const int64_t* ids, const int32_t* slots, const int32_t* pos,
                                 float* kept_weight, int64_t* kept_ids, int32_t* kept_slots, int32_t* kept_pos, int32_t* kept_lengths,
                                 int64_t* evict_ids, int32_t* evict_slots, int64_t list_capacity, int64_t* evict_offsets, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    size_t need = 0;
    BP_TRY(bp_evict_by_weight_workspace_bytes(n, bags, &need));
    if (budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget)
        return fail(BP_ERR_INVALID_ARG, "budget %d, sinks %d, recent %d: at least 1, 0 and 0, sinks + recent <= budget", budget, sinks, recent);
    if (list_capacity < 0) return fail(BP_ERR_INVALID_ARG, "negative list_capacity");
    if (!evict_offsets || (bags && (!bag_offsets || !kept_lengths))) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (n && bags && (!weight || !slots || !kept_slots)) return fail(BP_ERR_INVALID_ARG, "NULL pointer");
    if (n && ((ids != nullptr) != (kept_ids != nullptr) || (pos != nullptr) != (kept_pos != nullptr)))
        return fail(BP_ERR_INVALID_ARG, "kept_ids goes with ids, kept_pos with pos");
    if (list_capacity && (!evict_slots || (n && (ids != nullptr) != (evict_ids != nullptr))))
        return fail(BP_ERR_INVALID_ARG, "evict_slots is NULL, or only one of ids and evict_ids is given");
    if ((((uintptr_t)bag_offsets | (uintptr_t)ids | (uintptr_t)kept_ids | (uintptr_t)evict_ids | (uintptr_t)evict_offsets) & 7) ||
        (((uintptr_t)bag_lengths | (uintptr_t)weight | (uintptr_t)slots | (uintptr_t)pos | (uintptr_t)kept_weight | (uintptr_t)kept_slots |
          (uintptr_t)kept_pos | (uintptr_t)kept_lengths | (uintptr_t)evict_slots) & 3))
        return fail(BP_ERR_INVALID_ARG, "an array is not aligned to its elements");
    const void* const from[4] = {weight, ids, slots, pos};
    const void* const to[4] = {kept_weight, kept_ids, kept_slots, kept_pos};
    const size_t wide[4] = {4, 8, 4, 4};
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (from[i] && to[j] && (uintptr_t)from[i] < (uintptr_t)to[j] + n * wide[j] && (uintptr_t)to[j] < (uintptr_t)from[i] + n * wide[i])
                return fail(BP_ERR_INVALID_ARG, "the kept arrays overlap the input arrays");
    if (bags && kept_lengths == bag_lengths) return fail(BP_ERR_INVALID_ARG, "kept_lengths is bag_lengths");
    if (need && (!workspace || ((uintptr_t)workspace & 255))) return fail(BP_ERR_INVALID_ARG, "workspace NULL or not 256-byte aligned");
    if (workspace_bytes < need) return fail(BP_ERR_WORKSPACE_TOO_SMALL, "workspace %zu < required %zu bytes", workspace_bytes, need);
    const EvictScratch w(workspace, n, bags);
    return launch_evict(EvictArgs{bag_offsets, bag_lengths, n, bags, budget, sinks, recent, weight, ids, slots, pos, kept_weight, kept_ids,
                                  kept_slots, kept_pos, kept_lengths, evict_ids, evict_slots, list_capacity, evict_offsets, 0, 0, 0, w.choice,
                                  w.begins, w.hist},
                        (hipStream_t)stream);
}
