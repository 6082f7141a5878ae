// Block tables of a paged cache (wg_kv_* of wg.h): room for new tokens, tokens given back, and tables that
// follow a beam search's selection.
//
// State of a pool: ref[b] = how many table rows name block b, and one bit per block that is set while
// ref[b] == 0.  "The k-th free block" is then a prefix sum over the bits' population counts, and what
// is taken does not depend on the order in which blocks came free: whatever order the atomics of a
// call ran in, the counts and bits after it are the same.
#include <new>

#include "wg_divide.cuh"
#include "wg_host.h"

namespace {

constexpr int PLAN_THREADS = 1024;      // one block: plans of a whole batch
constexpr int FILL_THREADS = 256;
constexpr int MOVE_THREADS = 128;       // columns of a table per block
constexpr int SHRINK_THREADS = 128;
constexpr int COPY_THREADS = 256;
constexpr int WORDS_PER_THREAD = 4;     // words of free bits a thread counts per round

struct PoolDev {
    int32_t *ref;         // [n_blocks]
    uint32_t *free_bits;  // [n_words], padded with zero words to a whole round of a thread
    int32_t *n_free;
    int32_t n_blocks, n_words;
    Divisor block;        // tokens of a block
    // per-call scratch
    int32_t *taken;       // [n_blocks] blocks handed out by the call, in order
    int32_t *first;       // [max_seqs] where a sequence's blocks begin in `taken`, or -1: refused
    int32_t *old_len;     // [max_seqs] lengths before the call
    int32_t *new_len;     // [max_seqs]
    int32_t *src;         // [max_seqs] a reorder's rows: the block to copy, or -1
    int4 *copy;           // [max_seqs] its copies, one after the other: from, to, tokens, column
    int32_t *n_copies;
    int32_t *arrived;     // blocks of the reorder's first kernel that have finished; zero between calls
};

__device__ __forceinline__ void kv_enter() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// A length (>= 0) in whole blocks and the tokens beyond them.
struct Blocks {
    int32_t whole, rest;
    __device__ __forceinline__ Blocks(const PoolDev &pool, int32_t len)
        : whole((int32_t)pool.block.quotient((uint32_t)len)), rest(len - whole * (int32_t)pool.block.d) {}
    __device__ __forceinline__ int32_t held() const { return whole + (rest != 0); }
};

__device__ __forceinline__ int up(int x, int o) { return __shfl_up_sync(0xFFFFFFFFu, x, o); }

// Inclusive prefix sum over the block, and the block's total.  `warps`: shared, 32 entries.
template <typename T>
__device__ __forceinline__ T block_scan(T x, T *warps, T &total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = (int)(blockDim.x >> 5);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const T y = up(x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) warps[warp] = x;
    __syncthreads();
    if (warp == 0) {
        T w = lane < n_warps ? warps[lane] : T{};
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const T y = up(w, o);
            if (lane >= o) w += y;
        }
        if (lane < n_warps) warps[lane] = w;
    }
    __syncthreads();
    total = warps[n_warps - 1];
    const T before = warp > 0 ? warps[warp - 1] : T{};
    __syncthreads();   // `warps` may be used again
    return x + before;
}

__device__ __forceinline__ int nth_set_bit(uint32_t w, int n) {   // position of the n-th set bit (0-based)
    int at = 0;
#pragma unroll
    for (int half = 16; half > 0; half >>= 1) {
        const int c = __popc((w >> at) & ((1u << half) - 1u));
        if (n >= c) {
            n -= c;
            at += half;
        }
    }
    return at;
}

// Called by a whole block: takes the `n` lowest free blocks (n <= the number of free ones; the caller has
// seen to that) with count 1 and calls got(k, id) for the k-th of them.  Every round a thread counts
// four words of free bits; after the scan the warps go over the threads' words, a lane per bit.
// `w`: the thread's words of the first round, asked for early.
template <int THREADS>
struct TakeShared {
    uint4 words[THREADS];
    int32_t before[THREADS];      // free blocks before a thread's words
    int32_t warps[32];
};

__device__ __forceinline__ uint4 free_words(const PoolDev &pool, int at) {
    return at < pool.n_words ? __ldcg(reinterpret_cast<const uint4 *>(pool.free_bits + at)) : make_uint4(0, 0, 0, 0);
}

template <int THREADS, typename Got>
__device__ __forceinline__ void take_blocks(const PoolDev &pool, TakeShared<THREADS> &sh, int n, uint4 w, const Got &got) {
    const int lane = threadIdx.x & 31;
    int done = 0;
#pragma unroll 1
    for (int w0 = 0; done < n && w0 < pool.n_words; w0 += THREADS * WORDS_PER_THREAD) {
        const int mine = w0 + (int)threadIdx.x * WORDS_PER_THREAD;
        if (w0 > 0) w = free_words(pool, mine);
        sh.words[threadIdx.x] = w;
        const int count = __popc(w.x) + __popc(w.y) + __popc(w.z) + __popc(w.w);
        int total;
        const int before = block_scan(count, sh.warps, total) - count;
        sh.before[threadIdx.x] = before;
        __syncthreads();
        const int here = min(total, n - done);
#pragma unroll 1
        for (int g = threadIdx.x >> 5; g < THREADS; g += THREADS / 32) {
            int k = sh.before[g];
            if (k >= here) break;
            const uint32_t *words = reinterpret_cast<const uint32_t *>(&sh.words[g]);
#pragma unroll 1
            for (int i = 0; i < WORDS_PER_THREAD; ++i) {
                const uint32_t word = words[i];
                const int at = k + __popc(word & ((1u << lane) - 1u));
                if (((word >> lane) & 1u) && at < here) {
                    const int id = (w0 + g * WORDS_PER_THREAD + i) * 32 + lane;
                    pool.ref[id] = 1;
                    got(done + at, id);
                }
                k += __popc(word);
            }
        }
        int drop = min(count, here - before);         // of this thread's blocks, the lowest `drop` are gone
        if (drop > 0) {
            uint32_t v[WORDS_PER_THREAD] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int i = 0; i < WORDS_PER_THREAD; ++i) {
                const int c = __popc(v[i]);
                if (drop >= c) v[i] = 0u;
                else if (drop > 0) v[i] &= ~((1u << nth_set_bit(v[i], drop)) - 1u);
                drop -= c;
            }
            *reinterpret_cast<uint4 *>(pool.free_bits + mine) = make_uint4(v[0], v[1], v[2], v[3]);
        }
        done += here;
        __syncthreads();                              // the shared words are free for the next round
    }
}

__device__ __forceinline__ bool id_ok(const PoolDev &pool, int32_t id) { return id >= 0 && id < pool.n_blocks; }

__device__ __forceinline__ void add_freed(const PoolDev &pool, int freed) {   // called by whole warps
    freed = __reduce_add_sync(0xFFFFFFFFu, freed);
    if ((threadIdx.x & 31) == 0 && freed) atomicAdd(pool.n_free, freed);
}

// ---------------------------------------------------------------------------------------
// Pool set-up
// ---------------------------------------------------------------------------------------
// refs == NULL: all blocks free.  A thread per word of bits.
__global__ void pool_load_kernel(PoolDev pool, const int32_t *refs) {
    const int w = blockIdx.x * blockDim.x + threadIdx.x;
    uint32_t bits = 0;
    if (w < pool.n_words) {
        for (int i = 0; i < 32; ++i) {
            const int id = w * 32 + i;
            if (id >= pool.n_blocks) break;
            const int32_t r = refs ? max(refs[id], 0) : 0;
            pool.ref[id] = r;
            if (r == 0) bits |= 1u << i;
        }
        pool.free_bits[w] = bits;
    }
    add_freed(pool, __popc(bits));
}

// ---------------------------------------------------------------------------------------
// Extend
// ---------------------------------------------------------------------------------------
struct ExtendArgs {
    int32_t *table;
    int64_t stride;
    int32_t max_blocks;
    int32_t *len;
    const int32_t *n_new;
    int32_t n_seq;
    int32_t *cu;
    int64_t *slot;
    int32_t *pos, *seq;
    int32_t n_tokens;
    int32_t *status;
};

// Token t of the call: its sequence by bisection over cu, its block from the table or, for a new
// block, from the blocks taken.  The token at a block's first position also enters the block into the
// table (new blocks begin where the old length's last block ends, so each holds exactly one such token).
__device__ __forceinline__ void extend_token(const PoolDev &pool, const ExtendArgs &a, int t, int n_used,
                                             const int32_t *cu, const int32_t *old_len, const int32_t *first,
                                             const int32_t *taken) {
    int64_t slot = -1;
    int32_t pos = -1, s = -1;
    if (t < n_used) {
        int lo = 0, hi = a.n_seq - 1;      // the sequence that begins at or before t and ends after it
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (cu[mid + 1] > t) hi = mid; else lo = mid + 1;
        }
        s = lo;
        const int32_t len = old_len[s];
        pos = len + (t - cu[s]);
        if (first[s] >= 0) {
            const Blocks at(pool, pos);
            const int32_t held = Blocks(pool, len).held(), col = at.whole;
            int32_t *entry = a.table + (int64_t)s * a.stride + col;
            int32_t id;
            if (col < held) {
                id = *entry;
            } else {
                id = taken[first[s] + col - held];
                if (at.rest == 0) *entry = id;
            }
            if (id_ok(pool, id)) slot = (int64_t)id * (int64_t)pool.block.d + at.rest;
        }
    }
    a.slot[t] = slot;
    a.pos[t] = pos;
    a.seq[t] = s;
}

// A batch of up to this many tokens in at most PLAN_THREADS sequences is placed by the planning block
// itself, everything it needs for that in shared memory (one launch less).
constexpr int32_t FILL_IN_PLAN = 2048;

struct PlanSums {
    long long tokens, wanted;
    __device__ __forceinline__ PlanSums operator+(const PlanSums &o) const { return {tokens + o.tokens, wanted + o.wanted}; }
    __device__ __forceinline__ PlanSums &operator+=(const PlanSums &o) { return *this = *this + o; }
};
__device__ __forceinline__ PlanSums up(const PlanSums &x, int o) {
    return {__shfl_up_sync(0xFFFFFFFFu, x.tokens, o), __shfl_up_sync(0xFFFFFFFFu, x.wanted, o)};
}

// One block: who gets how many blocks, which ones, and where each sequence's tokens begin.  A block is
// enough: a batch has few thousand sequences, and what it takes lies at the front of the free bits.
// Bound by latency: lengths, scan, free words, scan, table entry.  Measured, with the tokens taken back again
// (the shrink): 7.6 us for one token of each of 1024 sequences, 9.6 us for 64 prompts of 8192 tokens
// in all, whose tokens the fill kernel places in parallel.
template <bool FILL>
__global__ void __launch_bounds__(PLAN_THREADS, 1)
extend_plan_kernel(PoolDev pool, ExtendArgs a) {
    __shared__ TakeShared<PLAN_THREADS> take;
    __shared__ PlanSums warps[32];
    __shared__ int32_t sh_cu[FILL ? PLAN_THREADS + 1 : 1], sh_len[FILL ? PLAN_THREADS : 1];
    __shared__ int32_t sh_first[FILL ? PLAN_THREADS : 1], sh_taken[FILL ? FILL_IN_PLAN : 1];
    kv_enter();
    const uint4 free0 = free_words(pool, (int)threadIdx.x * WORDS_PER_THREAD);
    const int n_free = *pool.n_free;
    PlanSums before{0, 0};               // of the rounds done
    int granted = 0;                     // blocks granted: the largest prefix that is
    const int64_t room = min((int64_t)a.max_blocks * pool.block.d, (int64_t)INT32_MAX);   // lengths have 32 bits
    for (int s0 = 0; s0 < a.n_seq; s0 += PLAN_THREADS) {
        const int s = s0 + (int)threadIdx.x;
        int32_t len = 0, add = 0, need = 0, st = WG_OK;
        if (s < a.n_seq) {
            len = a.len[s];
            add = a.n_new[s];
            if (len < 0 || len > room || add < 0 || (int64_t)len + add > room) {
                st = WG_ERR_ARG;
                add = 0;
            } else {
                need = Blocks(pool, len + add).held() - Blocks(pool, len).held();
            }
        }
        PlanSums total;
        const PlanSums upto = block_scan(PlanSums{add, need}, warps, total) + before;
        int last = 0;                    // blocks granted up to and including this sequence
        if (s < a.n_seq) {
            const bool fits = st == WG_OK &&
                              (add == 0 || (upto.tokens <= a.n_tokens && (need == 0 || upto.wanted <= n_free)));
            if (st == WG_OK && !fits) st = WG_ERR_CAPACITY;
            const int32_t cu = (int32_t)min(upto.tokens, (long long)a.n_tokens);
            const int32_t first = fits ? (int32_t)min(upto.wanted - need, (long long)n_free) : -1;
            a.cu[s + 1] = cu;
            if (FILL) {
                sh_cu[s + 1] = cu;
                sh_len[s] = len;
                sh_first[s] = first;
            } else {
                pool.old_len[s] = len;
                pool.first[s] = first;
            }
            if (fits) {
                a.len[s] = len + add;
                if (need > 0) last = (int)upto.wanted;
            }
            if (a.status) a.status[s] = st;
        }
        granted = max(granted, __reduce_max_sync(0xFFFFFFFFu, last));
        before += total;
    }
    if (threadIdx.x == 0) {
        a.cu[0] = 0;
        if (FILL) sh_cu[0] = 0;
    }
    if ((threadIdx.x & 31) == 0) take.warps[threadIdx.x >> 5] = granted;
    __syncthreads();
    granted = __reduce_max_sync(0xFFFFFFFFu, take.warps[threadIdx.x & 31]);
    __syncthreads();
    if (granted > 0) {
        take_blocks(pool, take, granted, free0, [&](int k, int id) {
            if (FILL) sh_taken[k] = id;
            else pool.taken[k] = id;
        });
        if (threadIdx.x == 0) *pool.n_free = n_free - granted;
    }
    if (FILL) {
        __syncthreads();
        const int n_used = sh_cu[a.n_seq];
        for (int t = threadIdx.x; t < a.n_tokens; t += PLAN_THREADS)
            extend_token(pool, a, t, n_used, sh_cu, sh_len, sh_first, sh_taken);
    }
}

__global__ void __launch_bounds__(FILL_THREADS)
extend_fill_kernel(PoolDev pool, ExtendArgs a) {
    kv_enter();
    const int n_used = a.cu[a.n_seq];
    const int t = blockIdx.x * FILL_THREADS + (int)threadIdx.x;
    if (t < a.n_tokens) extend_token(pool, a, t, n_used, a.cu, pool.old_len, pool.first, pool.taken);
}

// ---------------------------------------------------------------------------------------
// Shrink: a block per sequence.  A count that reaches zero sets the block's free bit; a sequence's blocks are
// counted down four to a thread, all in flight together, since each waits for what the atomic returns.
// Measured in the extend's figures above.
// ---------------------------------------------------------------------------------------
__global__ void __launch_bounds__(SHRINK_THREADS)
shrink_kernel(PoolDev pool, int32_t *table, int64_t stride, int32_t max_blocks, int32_t *len,
              const int32_t *keep, int32_t *status) {
    kv_enter();
    const int s = blockIdx.x;
    const int32_t have = len[s], want = keep[s];
    const bool ok = have >= 0 && have <= (int64_t)max_blocks * pool.block.d && want >= 0 && want <= have;
    if (threadIdx.x == 0 && status) status[s] = ok ? WG_OK : WG_ERR_ARG;
    if (!ok) return;
    const int32_t end = Blocks(pool, have).held();
    int32_t *row = table + (int64_t)s * stride;
    int freed = 0;
    constexpr int AT_ONCE = 4;
    for (int c0 = Blocks(pool, want).held() + (int)threadIdx.x; c0 < end; c0 += AT_ONCE * SHRINK_THREADS) {
        int32_t id[AT_ONCE], left[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int c = c0 + u * SHRINK_THREADS;
            id[u] = c < end ? row[c] : -1;
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) left[u] = id_ok(pool, id[u]) ? atomicSub(&pool.ref[id[u]], 1) - 1 : -1;
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            if (c0 + u * SHRINK_THREADS < end) row[c0 + u * SHRINK_THREADS] = -1;
            if (left[u] == 0) {
                atomicOr(&pool.free_bits[id[u] >> 5], 1u << (id[u] & 31));
                ++freed;
            }
        }
    }
    add_freed(pool, freed);
    __syncthreads();                       // everybody has read the length
    if (threadIdx.x == 0) len[s] = want;
}

// ---------------------------------------------------------------------------------------
// Reorder
// ---------------------------------------------------------------------------------------
struct MoveArgs {
    int32_t *table;
    int64_t stride;
    int32_t max_blocks;
    int32_t *len;
    const int32_t *parent;
    int32_t n_req, n_beam;
    int32_t *copy_src, *copy_dst, *status;
};

// What a request's rows become; filled by the block for its request.
struct MoveShared {
    int32_t parent[WG_BEAM_MAX_BEAMS];    // -1: the sequence ends
    int32_t len[WG_BEAM_MAX_BEAMS];       // old lengths, 0 where they lie outside the table
    int32_t blocks[WG_BEAM_MAX_BEAMS];    // columns in use
    int32_t partly[WG_BEAM_MAX_BEAMS];    // the column of a partly filled last block, or -1
    int32_t children[WG_BEAM_MAX_BEAMS];
    int32_t first[WG_BEAM_MAX_BEAMS];     // first child, or n_beam
    int32_t bad[WG_BEAM_MAX_BEAMS];       // the length lay outside
    int32_t most, alive;                  // columns in use by any row; rows that have a parent
};

constexpr int MOVE_ROWS = 4;              // rows a thread of the last block takes per round

// First kernel: grid = (tiles of MOVE_THREADS columns, requests); a thread holds one column of all the
// request's rows, so the rows move in place with no other thread in the way.  Row b's block of the
// column was held once and is held by its children afterwards: the count changes by children - 1 (a
// partly filled last block stays with one child only).  A count never reaches zero before the last row that
// named the block has been dealt with: what is not yet dealt with still counts 1 for each row.  In a
// column that all rows share (a prompt's) the changes cancel.  The block that finishes last hands out the
// blocks for the copies.  Bound by latency (a chain of lengths, table, counts, the finished blocks' counter,
// free bits): 28 us for 64 x 8 beams with their copies, which are about 18 of them, and 9.8 us for 4 x 4.
// Divisions by a block's length are multiplications; they and counts in flight together made 22 of 29 us
// (with the planes in L2).
__global__ void __launch_bounds__(MOVE_THREADS)
move_rows_kernel(PoolDev pool, MoveArgs a) {
    extern __shared__ int32_t column[];   // [n_beam][MOVE_THREADS]
    __shared__ MoveShared sh;
    __shared__ TakeShared<MOVE_THREADS> take;
    __shared__ int32_t is_last;
    kv_enter();
    const int K = a.n_beam, row0 = blockIdx.y * K;
    const int64_t room = (int64_t)a.max_blocks * pool.block.d;
    if ((int)threadIdx.x < K) {
        const int32_t p = a.parent[row0 + threadIdx.x], l = a.len[row0 + threadIdx.x];
        const int32_t len = l >= 0 && l <= room ? l : 0;
        const Blocks n(pool, len);
        sh.parent[threadIdx.x] = p >= 0 && p < K ? p : -1;
        sh.len[threadIdx.x] = len;
        sh.bad[threadIdx.x] = len != l;
        sh.blocks[threadIdx.x] = n.held();
        sh.partly[threadIdx.x] = n.rest != 0 ? n.whole : -1;
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        int children = 0, first = K, most = 0;
        if ((int)threadIdx.x < K) {
#pragma unroll 1
            for (int j = K - 1; j >= 0; --j)
                if (sh.parent[j] == (int)threadIdx.x) {
                    ++children;
                    first = j;
                }
            sh.children[threadIdx.x] = children;
            sh.first[threadIdx.x] = first;
            most = sh.blocks[threadIdx.x];
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        const int alive = __reduce_add_sync(0xFFFFFFFFu, children);
        if (threadIdx.x == 0) {
            sh.most = most;
            sh.alive = alive;
        }
    }
    __syncthreads();
    // what the last block needs of a row: its length, and that there is nothing to copy (where there is,
    // the thread that holds the column says so below)
    if (blockIdx.x == 0 && (int)threadIdx.x < K) {
        const int j = threadIdx.x, p = sh.parent[j];
        pool.new_len[row0 + j] = p >= 0 ? sh.len[p] : 0;
        if (a.status) a.status[row0 + j] = p >= 0 && sh.bad[p] ? WG_ERR_ARG : WG_OK;
        if (p < 0 || sh.partly[p] < 0 || sh.first[p] == j) pool.src[row0 + j] = -1;
    }
    int freed = 0;
    const int c = blockIdx.x * MOVE_THREADS + (int)threadIdx.x;
    if (c < sh.most) {
        constexpr int AT_ONCE = 8;
        int32_t *col = a.table + (int64_t)row0 * a.stride + c;
        int32_t *v = column + threadIdx.x;
        const int alive = sh.alive;
        bool same = true, plain = true;   // all rows name one block; no row's partly filled one
        int32_t id0 = -1;
#pragma unroll 1
        for (int b0 = 0; b0 < K; b0 += AT_ONCE) {
            int32_t id[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) id[u] = b0 + u < K && c < sh.blocks[b0 + u] ? col[(b0 + u) * a.stride] : -1;
            if (b0 == 0) id0 = id[0];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (b0 + u < K) {
                    v[(b0 + u) * MOVE_THREADS] = id_ok(pool, id[u]) ? id[u] : -1;
                    same = same && id[u] == id0;
                    plain = plain && c != sh.partly[b0 + u];
                }
        }
        same = same && plain && id_ok(pool, id0);
        if (!(same && alive == K)) {
            // counts (the atomics of several rows in flight together)
#pragma unroll 1
            for (int b0 = 0; b0 < K; b0 += AT_ONCE) {
                int32_t left[AT_ONCE];
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u) {
                    const int b = b0 + u;
                    left[u] = -1;
                    if (b < K) {
                        const int32_t id = v[b * MOVE_THREADS];
                        const int children = sh.children[b];
                        const int change = (c == sh.partly[b] ? min(children, 1) : children) - 1;
                        if (id >= 0 && change != 0) left[u] = atomicAdd(&pool.ref[id], change) + change;
                    }
                }
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u)
                    if (left[u] == 0) {
                        const int32_t id = v[(b0 + u) * MOVE_THREADS];
                        atomicOr(&pool.free_bits[id >> 5], 1u << (id & 31));
                        ++freed;
                    }
            }
            // rows
#pragma unroll 1
            for (int j = 0; j < K; ++j) {
                const int p = sh.parent[j];
                int32_t id = p >= 0 ? v[p * MOVE_THREADS] : -1;
                if (p >= 0 && c == sh.partly[p] && j != sh.first[p]) {
                    pool.src[row0 + j] = id;                             // its own block: later
                    id = -1;
                }
                if (id != v[j * MOVE_THREADS]) col[j * a.stride] = id;
            }
        }
    }
    add_freed(pool, freed);
    // ---- the last block to finish
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        is_last = atomicAdd(pool.arrived, 1) == (int)(gridDim.x * gridDim.y) - 1;
        __threadfence();
    }
    __syncthreads();
    if (!is_last) return;
    const uint4 free0 = free_words(pool, (int)threadIdx.x * WORDS_PER_THREAD);
    const int n_rows = a.n_req * K;
    const int n_free = __ldcg(pool.n_free);
    int done = 0;
#pragma unroll 1
    for (int r0 = 0; r0 < n_rows; r0 += MOVE_THREADS * MOVE_ROWS) {
        const int i0 = r0 + (int)threadIdx.x * MOVE_ROWS;
        int32_t src[MOVE_ROWS], len[MOVE_ROWS];
        int mine = 0, total;
#pragma unroll
        for (int u = 0; u < MOVE_ROWS; ++u) {
            src[u] = i0 + u < n_rows ? __ldcg(&pool.src[i0 + u]) : -1;
            len[u] = i0 + u < n_rows ? __ldcg(&pool.new_len[i0 + u]) : 0;
        }
#pragma unroll
        for (int u = 0; u < MOVE_ROWS; ++u) mine += src[u] >= 0;
        int rank = done + block_scan(mine, take.warps, total) - mine;
#pragma unroll
        for (int u = 0; u < MOVE_ROWS; ++u) {
            const int i = i0 + u;
            if (i >= n_rows) break;
            const bool got = src[u] >= 0 && rank < n_free;
            const Blocks n(pool, len[u]);
            if (got) {
                pool.copy[rank] = make_int4(src[u], i, n.rest, n.whole);   // (the row, until its block is known)
            } else if (src[u] >= 0) {
                len[u] -= n.rest;
                if (a.status) a.status[i] = WG_ERR_CAPACITY;
            }
            rank += src[u] >= 0;
            a.len[i] = len[u];
            if (a.copy_src) a.copy_src[i] = got ? src[u] : -1;
            if (a.copy_dst && !got) a.copy_dst[i] = -1;
        }
        done += total;
    }
    const int granted = min(done, n_free);
    __syncthreads();
    take_blocks(pool, take, granted, free0, [&](int k, int id) {
        const int4 copy = pool.copy[k];
        a.table[(int64_t)copy.y * a.stride + copy.w] = id;
        if (a.copy_dst) a.copy_dst[copy.y] = id;
        pool.copy[k].y = id;
    });
    if (threadIdx.x == 0) {
        *pool.n_free = n_free - granted;
        *pool.n_copies = granted;
        *pool.arrived = 0;
    }
}

// Second kernel: the filled tokens of every copied block, in all planes.  The blocks take (copy, plane)
// pairs in turn; there are four times as many as are resident, since pairs differ in length (one block of
// every SM's eight taking two to three pairs: 29.0 -> 27.9 us with the tables; the hardware deals the rest
// out).  Bound by memory: 64 x 8 beams with 16 planes of 2 KB tokens, 87 MB read and written, about 18 us
// (4.8 TB/s) from memory, 13 where the planes lie in L2.  Asking L2 for the sources while the
// first kernel finds places for the copies was slower (29 -> 35 us), 512 threads too (31).
__global__ void __launch_bounds__(COPY_THREADS)
copy_blocks_kernel(PoolDev pool, const wg_kv_plane *planes, int32_t n_planes) {
    kv_enter();
    const int64_t n = (int64_t)*pool.n_copies * n_planes;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int k = (int)(i / n_planes);
        const wg_kv_plane pl = planes[i - (int64_t)k * n_planes];
        const int4 copy = pool.copy[k];
        const int64_t per_block = (int64_t)pool.block.d * pl.token_bytes;
        const char *src = static_cast<const char *>(pl.base) + (int64_t)copy.x * per_block;
        char *dst = static_cast<char *>(pl.base) + (int64_t)copy.y * per_block;
        const int64_t bytes = (int64_t)copy.z * pl.token_bytes;
        if ((((uintptr_t)src | (uintptr_t)dst | (uint64_t)bytes) & 15) == 0) {
            const uint4 *s = reinterpret_cast<const uint4 *>(src);
            uint4 *d = reinterpret_cast<uint4 *>(dst);
            const int64_t m = bytes / 16;
            int64_t at = threadIdx.x;
            for (; at + 3 * COPY_THREADS < m; at += 4 * COPY_THREADS) {
                uint4 x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) x[u] = __ldcs(s + at + u * COPY_THREADS);
#pragma unroll
                for (int u = 0; u < 4; ++u) d[at + u * COPY_THREADS] = x[u];
            }
            for (; at < m; at += COPY_THREADS) d[at] = __ldcs(s + at);
        } else {
            for (int64_t at = threadIdx.x; at < bytes; at += COPY_THREADS) dst[at] = src[at];
        }
    }
}

}  // namespace

struct wg_kv_pool {
    PoolDev dev{};
    int32_t max_seqs = 0;
};

namespace {

bool table_ok(const wg_kv_pool *pool, const int32_t *table, int64_t stride, int32_t max_blocks,
              const int32_t *len, int32_t n_seq) {
    return pool && table && len && n_seq >= 1 && n_seq <= pool->max_seqs && max_blocks >= 1 &&
           stride >= max_blocks;
}

int32_t pool_load(wg_kv_pool *p, const int32_t *refs, cudaStream_t st) {
    WG_CUDA(cudaMemsetAsync(p->dev.n_free, 0, sizeof(int32_t), st));
    pool_load_kernel<<<(p->dev.n_words + 255) / 256, 256, 0, st>>>(p->dev, refs);
    WG_LAUNCHED();
    return WG_OK;
}

}  // namespace

extern "C" {

int32_t wg_kv_pool_create(int32_t n_blocks, int32_t block_size, int32_t max_seqs, wg_kv_pool **out) {
    NvtxRange nvtx_range("wg_kv_pool_create");
    if (!out) return WG_ERR_ARG;
    *out = nullptr;
    if (n_blocks < 1 || n_blocks > (1 << 30) || block_size < 1 || block_size > (1 << 30) || max_seqs < 1 || max_seqs > WG_MAX_ROWS)
        return WG_ERR_ARG;
    wg_kv_pool *p = new (std::nothrow) wg_kv_pool();
    if (!p) return WG_ERR_ARG;
    PoolDev &d = p->dev;
    p->max_seqs = max_seqs;
    d.n_blocks = n_blocks;
    d.block = Divisor::of((uint32_t)block_size);
    d.n_words = (n_blocks + 31) / 32;
    const size_t words = ((size_t)d.n_words + WORDS_PER_THREAD - 1) / WORDS_PER_THREAD * WORDS_PER_THREAD;
    int32_t rc = dev_alloc(&d.ref, (size_t)n_blocks);
    if (rc == WG_OK) rc = dev_alloc(&d.free_bits, words);
    if (rc == WG_OK) rc = dev_alloc(&d.taken, (size_t)n_blocks);
    if (rc == WG_OK) rc = dev_alloc(&d.n_free, 1);
    if (rc == WG_OK) rc = dev_alloc(&d.n_copies, 1);
    if (rc == WG_OK) rc = dev_alloc(&d.arrived, 1);
    if (rc == WG_OK) rc = dev_alloc(&d.copy, (size_t)max_seqs);
    for (int32_t **a : {&d.first, &d.old_len, &d.new_len, &d.src})
        if (rc == WG_OK) rc = dev_alloc(a, (size_t)max_seqs);
    if (rc == WG_OK && (cudaMemset(d.free_bits, 0, words * sizeof(uint32_t)) != cudaSuccess ||
                        cudaMemset(d.arrived, 0, sizeof(int32_t)) != cudaSuccess))
        rc = WG_ERR_CUDA;
    if (rc == WG_OK) rc = pool_load(p, nullptr, cudaStreamLegacy);
    if (rc == WG_OK && cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess) rc = WG_ERR_CUDA;
    if (rc != WG_OK) {
        wg_kv_pool_free(p);
        return rc;
    }
    *out = p;
    return WG_OK;
}

void wg_kv_pool_free(wg_kv_pool *p) {
    if (!p) return;
    const PoolDev &d = p->dev;
    for (void *q : {(void *)d.ref, (void *)d.free_bits, (void *)d.taken, (void *)d.n_free, (void *)d.n_copies,
                    (void *)d.arrived, (void *)d.first, (void *)d.old_len, (void *)d.new_len, (void *)d.src,
                    (void *)d.copy})
        cudaFree(q);
    delete p;
}

const int32_t *wg_kv_pool_refs(const wg_kv_pool *p) { return p ? p->dev.ref : nullptr; }

int32_t wg_kv_pool_load(wg_kv_pool *p, const int32_t *refs, void *stream) {
    NvtxRange nvtx_range("wg_kv_pool_load");
    if (!p || !refs) return WG_ERR_ARG;
    return pool_load(p, refs, static_cast<cudaStream_t>(stream));
}

int32_t wg_kv_pool_n_free(wg_kv_pool *p, int32_t *n_free, void *stream) {
    if (!p || !n_free) return WG_ERR_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    WG_CUDA(cudaMemcpyAsync(n_free, p->dev.n_free, sizeof(int32_t), cudaMemcpyDeviceToHost, st));
    WG_CUDA(cudaStreamSynchronize(st));
    return WG_OK;
}

int32_t wg_kv_extend(wg_kv_pool *p, int32_t *table, int64_t table_stride, int32_t max_blocks, int32_t *len,
                     const int32_t *n_new, int32_t n_seq, int32_t *cu, int64_t *slot, int32_t *pos,
                     int32_t *seq, int32_t n_tokens, int32_t *status, void *stream) {
    NvtxRange nvtx_range("wg_kv_extend");
    if (!table_ok(p, table, table_stride, max_blocks, len, n_seq) || !n_new || !cu || n_tokens < 0 ||
        (n_tokens > 0 && (!slot || !pos || !seq)))
        return WG_ERR_ARG;
    const ExtendArgs a{table, table_stride, max_blocks, len, n_new, n_seq, cu, slot, pos, seq, n_tokens, status};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (n_tokens <= FILL_IN_PLAN && n_seq <= PLAN_THREADS) {
        WG_CUDA(launch_pdl(extend_plan_kernel<true>, dim3(1), dim3(PLAN_THREADS), st, p->dev, a));
        WG_LAUNCHED();
        return WG_OK;
    }
    WG_CUDA(launch_pdl(extend_plan_kernel<false>, dim3(1), dim3(PLAN_THREADS), st, p->dev, a));
    WG_LAUNCHED();
    if (n_tokens == 0) return WG_OK;         // nothing to place
    WG_CUDA(launch_pdl(extend_fill_kernel, dim3(((unsigned)n_tokens + FILL_THREADS - 1) / FILL_THREADS),
                       dim3(FILL_THREADS), st, p->dev, a));
    WG_LAUNCHED();
    return WG_OK;
}

int32_t wg_kv_shrink(wg_kv_pool *p, int32_t *table, int64_t table_stride, int32_t max_blocks, int32_t *len,
                     const int32_t *keep, int32_t n_seq, int32_t *status, void *stream) {
    NvtxRange nvtx_range("wg_kv_shrink");
    if (!table_ok(p, table, table_stride, max_blocks, len, n_seq) || !keep) return WG_ERR_ARG;
    WG_CUDA(launch_pdl(shrink_kernel, dim3((unsigned)n_seq), dim3(SHRINK_THREADS), static_cast<cudaStream_t>(stream),
                       p->dev, table, table_stride, max_blocks, len, keep, status));
    WG_LAUNCHED();
    return WG_OK;
}

int32_t wg_kv_reorder(wg_kv_pool *p, int32_t *table, int64_t table_stride, int32_t max_blocks, int32_t *len,
                      const int32_t *parent, int32_t n_req, int32_t n_beam, const wg_kv_plane *planes,
                      int32_t n_planes, int32_t *copy_src, int32_t *copy_dst, int32_t *status, void *stream) {
    NvtxRange nvtx_range("wg_kv_reorder");
    if (n_req < 1 || n_beam < 1 || n_beam > WG_BEAM_MAX_BEAMS || (int64_t)n_req * n_beam > WG_MAX_ROWS ||
        !table_ok(p, table, table_stride, max_blocks, len, n_req * n_beam) || !parent || n_planes < 0 ||
        (n_planes > 0 && !planes))
        return WG_ERR_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const MoveArgs a{table, table_stride, max_blocks, len, parent, n_req, n_beam, copy_src, copy_dst, status};
    const dim3 grid((unsigned)((max_blocks + MOVE_THREADS - 1) / MOVE_THREADS), (unsigned)n_req);
    WG_CUDA(launch_pdl_smem(move_rows_kernel, grid, dim3(MOVE_THREADS), (size_t)n_beam * MOVE_THREADS * sizeof(int32_t),
                            st, p->dev, a));
    WG_LAUNCHED();
    if (n_planes == 0) return WG_OK;
    const int64_t most = (int64_t)n_req * (n_beam - 1) * n_planes;   // copies cannot be more
    if (most == 0) return WG_OK;
    const int64_t waves = (int64_t)sm_count() * 8 * 4;
    WG_CUDA(launch_pdl(copy_blocks_kernel, dim3((unsigned)(most < waves ? most : waves)), dim3(COPY_THREADS), st,
                       p->dev, planes, n_planes));
    WG_LAUNCHED();
    return WG_OK;
}

}  // extern "C"
