// Acceptance over a tree of drafts: the walk from the root that the target itself would take.
//
// At node c (the root first) the target names a token t: the argmax of c's logits row, or a draw from softmax(row / tau) by inverse CDF with the
// node's uniform.  The child of c that drafted t is accepted and becomes c; if no child did, the walk ends and t is the answer.  Every token
// that leaves is the target's own choice, so the text is the target's whatever the tree held.
//
// A walk needs the rows it passes and no others, and which those are is known one after the other.
//   few rows    one launch scans all rows of all trees in pieces (largest logit, its lowest id, sum of the weights); a workgroup per request then walks
//               in what that left, 1 us a node (greedy) or 8 (sampling: the piece in which the sum passes is gone through once more).
//   many rows   one launch: a workgroup of 16 wavefronts walks for a request and goes through each row by itself, with up to 256 KB asked for at a
//               time: 8 us a row of 128256 values out of L2, 14 out of memory; by sampling 22 us a row of 50257, one CU's float64 exponentials.
// 16 trees of 333 nodes, 128256 values, up to 6 accepted: 38 us; 64 trees of 1946 nodes by sampling, 50257 values, up to 7 accepted: 172 to 217 us by the
// longest walk.  A launch per
// level of the trees took 86 and 288 us: it has to launch for the deepest tree, whose last nodes are hardly ever reached.
// Sums of exponentials are float64 in a fixed order over the row: what rounding leaves between the forms is 1e-14 of the sum.
#include "sled_internal.h"

#include <string.h>

#include <algorithm>
#include <type_traits>

namespace {

constexpr int THREADS = 1024, WAVES = THREADS / 64, ROUND = 16, AHEAD = 4;   // pieces of four values that a thread asks for at a time

struct Piece;
struct walk_args {
    const float* logits;
    const int32_t* tokens;
    const float* u;          // one per row (sampling)
    double inv_tau;
    int V;
    const uint8_t* parent;   // [T] (root: 255), where the shape does not come with the launch
    const int32_t* first;    // [B + 1] first row of a request
    int32_t *accept_len, *path, *out_token;
    Piece* part;      // [T][pieces], where the rows have been scanned already
    int pieces, seg;         // of a row, and their length
};

struct __align__(16) Piece {   // of a row
    double sum;   // weights against its own largest logit (sampling)
    float m;      // largest logit
    int arg;      // its lowest id
};

// The trees' shape comes by value with the launch (so the call needs no copy from host memory and can be captured).
constexpr int PARENTS = 2048;
template <int B, int T>
struct __align__(16) Shape {
    uint8_t n[B];   // nodes - 1
    uint8_t p[T];   // parents (root: 255)
};
typedef Shape<64, 256> Small;
typedef Shape<1024, PARENTS> Large;

struct Best {
    float m;
    int arg;
};
__device__ inline void better(Best& b, float x, int i) {
    if (x > b.m || (x == b.m && i < b.arg)) {
        b.m = x;
        b.arg = i;
    }
}

// four neighbouring values that start anywhere (a row is as aligned as its length)
struct __attribute__((packed, aligned(4))) Four {
    float x[4];
};
// The values at j .. j + 3 of a row of V >= 4, moved down where they would pass its end; returns where they begin
__device__ inline int four_at(const float* __restrict__ row, int V, int j, Four& f) {
    const int at = min(j, V - 4);
    f = *reinterpret_cast<const Four*>(row + at);
    return at;
}

// the same for a row of any length: what a short one lacks has no weight
__device__ inline int four_of(const float* __restrict__ row, int V, int j, Four& f) {
    if (V >= 4) return four_at(row, V, j, f);
#pragma unroll
    for (int e = 0; e < 4; e++) f.x[e] = e < V ? row[min(e, V - 1)] : -INFINITY;
    return 0;
}

// e^y for y <= 0, zero for NaN: y = k ln 2 + r, the Taylor series of e^r up to r^11 (|r| <= ln 2 / 2: the rest is below 9e-15 of it).  Below -746 it is zero in
// float64, and far below (a mask of the type's lowest value) k ln 2 would not be exact and r no longer small.
__device__ inline double exp_below(double y) {
    y = fmax(y, -746.0);
    const double k = rint(y * 1.4426950408889634);
    // ln 2 = 2977044471 / 2^32 + 1.908e-10: the first part times k is exact
    const double r = fma(-k, 1.9082149292705877e-10, fma(-k, 2977044471.0 / 4294967296.0, y));
    double e = 1.0 / 39916800;
    e = fma(e, r, 1.0 / 3628800);
    e = fma(e, r, 1.0 / 362880);
    e = fma(e, r, 1.0 / 40320);
    e = fma(e, r, 1.0 / 5040);
    e = fma(e, r, 1.0 / 720);
    e = fma(e, r, 1.0 / 120);
    e = fma(e, r, 1.0 / 24);
    e = fma(e, r, 1.0 / 6);
    e = fma(e, r, 0.5);
    e = fma(e, r, 1.0);
    e = fma(e, r, 1.0);
    return ldexp(e, (int)k);
}
// weight of a value; one that is not a number, or lies as far above as infinity, has none
__device__ inline double weight(float x, double m, double inv_tau) { return exp_below(((double)x - m) * inv_tau); }

struct walk_shared {
    float m[WAVES];
    int arg[WAVES];
    double sum[WAVES];
    int tok, last;
};

// largest value of a row and its lowest id, in every thread
__device__ __forceinline__ Best row_best(const float* __restrict__ row, int V, walk_shared& sh) {
    const int tid = threadIdx.x;
    Best b{-INFINITY, 0x7fffffff};
    if (V < 4) {
        for (int k = 0; k < V; k++) better(b, row[k], k);
        return b;
    }
    // A thread's pieces ascend, so only a larger value replaces one.  Which of a piece's four it was is found at the end.
    int piece = 0;
    for (int j0 = 0; j0 < V; j0 += ROUND * 4 * THREADS) {
        Four f[ROUND];
        int at[ROUND];
#pragma unroll
        for (int k = 0; k < ROUND; k++)
            if (j0 + k * THREADS * 4 < V) at[k] = four_at(row, V, j0 + (k * THREADS + tid) * 4, f[k]);   // (some values twice, at the row's end)
#pragma unroll
        for (int k = 0; k < ROUND; k++) {
            if (j0 + k * THREADS * 4 >= V) break;
            const float top = fmaxf(fmaxf(f[k].x[0], f[k].x[1]), fmaxf(f[k].x[2], f[k].x[3]));
            if (top > b.m) {
                b.m = top;
                piece = at[k];
            }
        }
    }
    if (b.m > -INFINITY) {
        Four f;
        const int at = four_at(row, V, piece, f);
        b.arg = f.x[0] == b.m ? at : f.x[1] == b.m ? at + 1 : f.x[2] == b.m ? at + 2 : at + 3;
    } else {
        b.arg = min(tid * 4, V - 4);   // nothing larger: the first of this thread's
    }
    for (int off = 32; off > 0; off >>= 1) {
        const float x = __shfl_xor(b.m, off);
        const int i = __shfl_xor(b.arg, off);
        better(b, x, i);
    }
    __syncthreads();
    if ((tid & 63) == 0) {
        sh.m[tid >> 6] = b.m;
        sh.arg[tid >> 6] = b.arg;
    }
    __syncthreads();
    b = Best{sh.m[0], sh.arg[0]};
#pragma unroll
    for (int w = 1; w < WAVES; w++) better(b, sh.m[w], sh.arg[w]);
    return b;
}

__device__ inline double sum_up_to_lane(double c, int lane) {
    for (int off = 1; off < 64; off <<= 1) {
        const double x = __shfl_up(c, off);
        if (lane >= off) c += x;
    }
    return c;
}

// The id of the run of n ids from `from` on at which the cumulative sum, `before` up to there, passes the target; or the run's last id with weight
__device__ __forceinline__ int draw_within(const float* __restrict__ row, int V, int from, int n, double before, double target, double m, double inv_tau, walk_shared& sh) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = (n + 4 * THREADS - 1) / (4 * THREADS) * 4;
    from = min(V, from);
    const int to = min(V, from + n), k0 = min(to, from + tid * per), k1 = min(to, k0 + per);
    double mine = 0.0;
    int last = -1;
    for (int k = k0; k < k1; k += 4) {
        Four f;
        const int at = four_of(row, V, k, f);
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const double w = weight(f.x[e], m, inv_tau);
            if (at + e < k || at + e >= k1 || !(w > 0.0)) continue;
            mine += w;
            last = at + e;
        }
    }
    const double upto = sum_up_to_lane(mine, lane);
    __syncthreads();   // (what the caller has in sh.sum has been read)
    if (tid == 0) {
        sh.tok = 0x7fffffff;
        sh.last = -1;
    }
    if (lane == 63) sh.sum[wave] = upto;
    __syncthreads();
    double base = before;
    for (int w = 0; w < wave; w++) base += sh.sum[w];
    // the first thread that has weight and in whose ids, or before them, the sum passes
    const uint64_t past = __ballot(base + upto > target && last >= 0), any = __ballot(last >= 0);
    if (past && lane == __builtin_ctzll(past)) {
        double at = base + (upto - mine);
        int tok = last;
        for (int k = k0; k < k1 && !(at > target); k += 4) {
            Four f;
            const int j = four_of(row, V, k, f);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                if (j + e < k || j + e >= k1 || at > target) continue;
                at += weight(f.x[e], m, inv_tau);
                if (at > target) tok = j + e;
            }
        }
        atomicMin(&sh.tok, tok);
    }
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&sh.last, last);
    __syncthreads();
    const int tok = sh.tok == 0x7fffffff ? sh.last : sh.tok;
    __syncthreads();
    return tok;
}

// The id at which the cumulative sum of a row's weights passes u of their total.  A wavefront adds up a run of neighbouring ids; the run in which
// the sum passes is then shared out among all threads.
__device__ __forceinline__ int row_draw(const float* __restrict__ row, int V, const Best& b, double u, double inv_tau, walk_shared& sh) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const double m = (double)b.m;
    const int run = (V + WAVES * 256 - 1) / (WAVES * 256) * 256, lo = min(V, wave * run), hi = min(V, lo + run);
    double sum = 0.0;
    if (V >= 4) {
        Four next[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; k++) four_at(row, V, lo + k * 256 + lane * 4, next[k]);
        for (int j0 = lo; j0 < hi; j0 += AHEAD * 256) {
            Four f[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; k++) f[k] = next[k];
#pragma unroll
            for (int k = 0; k < AHEAD; k++) four_at(row, V, j0 + (AHEAD + k) * 256 + lane * 4, next[k]);
#pragma unroll
            for (int k = 0; k < AHEAD; k++) {
                const int j = j0 + k * 256 + lane * 4, at = min(j, V - 4);
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const double w = weight(f[k].x[e], m, inv_tau);
                    sum += j < hi && at + e >= j ? w : 0.0;   // (a piece that was moved down: only what is its own)
                }
            }
        }
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
    } else if (wave == 0) {
        for (int k = 0; k < V; k++) sum += weight(row[k], m, inv_tau);
    }
    if (lane == 0) sh.sum[wave] = sum;
    __syncthreads();
    double total = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; w++) total += sh.sum[w];
    if (!(total > 0.0)) return b.arg;   // nothing weighs anything: a row without a finite value
    const double target = u * total;
    int s = -1, some = 0;
    double before = 0.0, c = 0.0;
#pragma unroll
    for (int w = 0; w < WAVES; w++) {
        const double x = sh.sum[w];
        if (x > 0.0) some = w;
        if (s < 0 && c + x > target) {
            s = w;
            before = c;
        }
        c += x;
    }
    if (s < 0) {   // it never passes (rounding): the last id with weight
        s = some;
        before = target;
    }
    return draw_within(row, V, s * run, run, before, target, m, inv_tau, sh);
}

// Where there are few rows: all of them are scanned in pieces by a launch of its own, and the walk finds its tokens in what that left.
constexpr int SCAN_THREADS = 256;
template <bool SAMPLE>
__global__ __launch_bounds__(SCAN_THREADS) void accept_tree_scan(walk_args a) {
    __shared__ float sh_m[SCAN_THREADS / 64];
    __shared__ int sh_i[SCAN_THREADS / 64];
    __shared__ double sh_d[SCAN_THREADS / 64];
    const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = a.V;
    const size_t t = blockIdx.y;
    const float* row = a.logits + t * V;
    const int lo = s * a.seg, hi = min(V, lo + a.seg);   // (V is no less than 4, and lo less than V)
    Best b{-INFINITY, 0x7fffffff};
    for (int j0 = lo; j0 < hi; j0 += AHEAD * 4 * SCAN_THREADS) {
        Four f[AHEAD];
        int at[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; k++) at[k] = four_at(row, V, j0 + (k * SCAN_THREADS + tid) * 4, f[k]);
#pragma unroll
        for (int k = 0; k < AHEAD; k++)
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (at[k] + e >= lo && at[k] + e < hi) better(b, f[k].x[e], at[k] + e);
    }
    for (int off = 32; off > 0; off >>= 1) {
        const float x = __shfl_xor(b.m, off);
        const int i = __shfl_xor(b.arg, off);
        better(b, x, i);
    }
    if (lane == 0) {
        sh_m[wave] = b.m;
        sh_i[wave] = b.arg;
    }
    __syncthreads();
    b = Best{sh_m[0], sh_i[0]};
#pragma unroll
    for (int w = 1; w < SCAN_THREADS / 64; w++) better(b, sh_m[w], sh_i[w]);
    double sum = 0.0;
    if (SAMPLE) {
        for (int j0 = lo + tid * 4; j0 < hi; j0 += 4 * SCAN_THREADS) {
            Four f;
            const int at = four_at(row, V, j0, f);
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const double w = weight(f.x[e], (double)b.m, a.inv_tau);
                sum += at + e >= j0 && at + e < hi ? w : 0.0;
            }
        }
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        if (lane == 0) sh_d[wave] = sum;
        __syncthreads();
        sum = 0.0;
#pragma unroll
        for (int w = 0; w < SCAN_THREADS / 64; w++) sum += sh_d[w];
    }
    if (tid == 0) a.part[t * a.pieces + s] = Piece{sum, b.m, b.arg};
}

// the token of a row whose pieces are at hand: a lane for each, in every wavefront
template <bool SAMPLE>
__device__ __forceinline__ int row_token(const walk_args& a, size_t t, walk_shared& sh) {
    const int lane = threadIdx.x & 63;
    Piece p{0.0, -INFINITY, 0x7fffffff};
    if (lane < a.pieces) p = a.part[t * a.pieces + lane];
    Best b{p.m, p.arg};
    for (int off = 32; off > 0; off >>= 1) {
        const float x = __shfl_xor(b.m, off);
        const int i = __shfl_xor(b.arg, off);
        better(b, x, i);
    }
    if constexpr (!SAMPLE) return b.arg;
    const double w = p.sum > 0.0 ? p.sum * exp_below(((double)p.m - (double)b.m) * a.inv_tau) : 0.0, c = sum_up_to_lane(w, lane), total = __shfl(c, 63);
    if (!(total > 0.0)) return b.arg;
    double target = (double)a.u[t] * total;
    const uint64_t past = __ballot(c > target), some = __ballot(w > 0.0);
    const int s = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);   // (it never passes: the last with weight)
    double before = __shfl(c, max(s - 1, 0));
    if (s == 0) before = 0.0;
    // against the row's largest logit a piece weighs what it does against its own, times a factor: the sums of its ids are compared in the latter
    const double own = (double)__shfl(p.m, s), scale = exp_below((own - (double)b.m) * a.inv_tau);
    return draw_within(a.logits + t * a.V, a.V, s * a.seg, a.seg, past ? before / scale : 0.0, past ? target / scale : INFINITY, own, a.inv_tau, sh);
}

struct Stored {};   // the shape is in a.first and a.parent

// SCANNED: the rows' pieces are at hand
template <bool SAMPLE, class S, bool SCANNED>
__global__ __launch_bounds__(THREADS) void accept_tree_walk(walk_args a, S shape) {
    __shared__ walk_shared sh;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
    int row0, n;
    if constexpr (!std::is_same_v<S, Stored>) {
        // nodes of the requests before
        constexpr int EACH = sizeof(shape.n) / 64;
        int sum = 0;
#pragma unroll
        for (int k = 0; k < EACH; k++) sum += lane * EACH + k < b ? shape.n[lane * EACH + k] + 1 : 0;
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        row0 = __builtin_amdgcn_readfirstlane(sum);
        n = shape.n[b] + 1;
    } else {
        row0 = a.first[b];
        n = a.first[b + 1] - row0;
    }
    // every wavefront has the whole tree: node `lane`
    const int at = row0 + min(lane, n - 1), token = a.tokens[at];
    int parent;
    if constexpr (!std::is_same_v<S, Stored>) parent = shape.p[at];
    else parent = a.parent[at];
    int cur = 0, way = -1;
    for (int len = 0;; len++) {   // a child's number is larger than its parent's: at most n rounds
        const float* row = a.logits + (size_t)(row0 + cur) * a.V;
        int tok;
        if constexpr (SCANNED) {
            tok = row_token<SAMPLE>(a, row0 + cur, sh);
        } else {
            const Best best = row_best(row, a.V, sh);
            tok = SAMPLE ? row_draw(row, a.V, best, (double)a.u[row0 + cur], a.inv_tau, sh) : best.arg;
        }
        tok = min(max(tok, 0), a.V - 1);
        const uint64_t hits = __ballot(lane > 0 && lane < n && parent == cur && token == tok);   // (the lowest of several)
        if (!hits) {
            if (tid == 0) {
                a.accept_len[b] = len;
                a.out_token[b] = tok;
            }
            break;
        }
        cur = __builtin_ctzll(hits);
        if (tid == len) way = cur;
    }
    if (tid < SLED_TREE_MAX) a.path[(size_t)b * SLED_TREE_MAX + tid] = way;
}

// Trees of more than PARENTS nodes in all: their shape goes to the workspace first.
__global__ __launch_bounds__(256) void accept_tree_parents(Large x, int at, int count, uint8_t* __restrict__ parent) {
    for (int i = threadIdx.x; i < count; i += 256) parent[at + i] = x.p[i];
}
__global__ __launch_bounds__(256) void accept_tree_first(Large x, int B, int32_t* __restrict__ first) {
    __shared__ int sh[256];
    const int tid = threadIdx.x;
    int n[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        n[k] = 4 * tid + k < B ? x.n[4 * tid + k] + 1 : 0;
        sum += n[k];
    }
    sh[tid] = sum;
    __syncthreads();
    for (int off = 1; off < 256; off <<= 1) {
        const int x = tid >= off ? sh[tid - off] : 0;
        __syncthreads();
        sh[tid] += x;
        __syncthreads();
    }
    int at = sh[tid] - sum;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        if (4 * tid + k <= B) first[4 * tid + k] = at;
        at += n[k];
    }
    if (tid == 255 && B == 1024) first[1024] = at;
}

size_t up(size_t x) { return (x + 255) / 256 * 256; }

// Scanning all rows first costs what they hold at the rate of the whole card, walking alone what the longest walk passes at the rate of one CU.  Measured
// with walks of up to 8 nodes, 50257 values, scanned first / alone: 1024 rows 104 / 112 us (sampling 166 / 277), 1536 rows 146 / 127 (216 / 272),
// 1920 rows 168 / 124 (251 / 253).  One tree of 9 rows of 128256 values 19 / 51 (36 / 132), of 1024 values 21 / 33 us.
constexpr int SCAN_ROWS = 1024, SCAN_ROWS_SAMPLE = 1536;
static_assert(PARENTS >= SCAN_ROWS_SAMPLE, "the shape of few rows travels with the launch");
bool scan_first(bool sample, int T, int V) { return V >= 4 && T <= (sample ? SCAN_ROWS_SAMPLE : SCAN_ROWS); }
// pieces of at least 4096 values, and no more than a wavefront has lanes
int seg_of(int V) { return std::max(4096, (V + 63) / 64 + 1023) / 1024 * 1024; }
int pieces_of(int V) { return (V + seg_of(V) - 1) / seg_of(V); }

}  // namespace

// Grows with B and T: a call of more rows than are scanned has no use for their pieces, but a workspace for it also serves the smaller ones that have.
size_t sled_accept_tree_ws_bytes(int B, int T, int vocab) {
    const int scanned = std::min(T, SCAN_ROWS_SAMPLE);
    const size_t part = scan_first(true, scanned, vocab) ? (size_t)scanned * pieces_of(vocab) * sizeof(Piece) : 0;
    return up(part) + up((size_t)(B + 1) * 4) + up(T);
}

int sled_launch_accept_tree(int mode, int B, int T, const int* n_nodes, const int* parent, int vocab, float temperature, const float* logits,
                            const int32_t* tokens, const float* u, int32_t* accept_len, int32_t* path, int32_t* out_token, void* ws, hipStream_t st) {
    const bool sample = mode == SLED_SAMPLE, scan = scan_first(sample, T, vocab);
    char* w = static_cast<char*>(ws);
    int32_t* first = reinterpret_cast<int32_t*>(w);
    w += up((size_t)(B + 1) * 4);
    uint8_t* par = reinterpret_cast<uint8_t*>(w);
    w += up(T);
    const walk_args a{logits, tokens, u, 1.0 / (double)temperature, vocab, par, first, accept_len, path, out_token, reinterpret_cast<Piece*>(w), pieces_of(vocab), seg_of(vocab)};
    if (scan) {
        if (sample) hipLaunchKernelGGL(accept_tree_scan<true>, dim3(a.pieces, T), dim3(SCAN_THREADS), 0, st, a);
        else hipLaunchKernelGGL(accept_tree_scan<false>, dim3(a.pieces, T), dim3(SCAN_THREADS), 0, st, a);
        SLED_LAUNCH_CHECK();
    }
    auto fill = [&](auto& x, int at, int count) {
        memset(&x, 0, sizeof(x));
        for (int i = 0; i < B; i++) x.n[i] = (uint8_t)(n_nodes[i] - 1);
        for (int i = 0; i < count; i++) x.p[i] = parent[at + i] >= 0 ? (uint8_t)parent[at + i] : 255;
    };
    auto walk = [&](auto x) {
        using S = decltype(x);
        auto kernel = sample ? accept_tree_walk<true, S, false> : accept_tree_walk<false, S, false>;
        if constexpr (!std::is_same_v<S, Stored>)   // (there are few rows where they are scanned first)
            if (scan) kernel = sample ? accept_tree_walk<true, S, true> : accept_tree_walk<false, S, true>;
        hipLaunchKernelGGL(kernel, dim3(B), dim3(scan && !sample ? 64 : THREADS), 0, st, a, x);
    };
    // (a launch with 320 bytes of arguments costs the host 4 us less than one with 3 KB: one tree of 9 nodes 9 us instead of 14 in all)
    if (B <= 64 && T <= 256) {
        Small x;
        fill(x, 0, T);
        walk(x);
    } else if (T <= PARENTS) {
        Large x;
        fill(x, 0, T);
        walk(x);
    } else {
        Large x;
        for (int at = 0; at < T; at += PARENTS) {
            const int count = std::min(PARENTS, T - at);
            fill(x, at, count);
            if (at == 0) hipLaunchKernelGGL(accept_tree_first, dim3(1), dim3(256), 0, st, x, B, first);
            SLED_LAUNCH_CHECK();
            hipLaunchKernelGGL(accept_tree_parents, dim3(1), dim3(256), 0, st, x, at, count, par);
            SLED_LAUNCH_CHECK();
        }
        walk(Stored{});
    }
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}
