// Acceptance over a tree of drafts: the walk from the root that the target itself would take.
//
// At node c (the root first) the target names a token t: the argmax of c's logits row, or a draw from softmax(row / tau) by inverse CDF with the
// node's uniform.  The child of c that drafted t is accepted and becomes c; if no child did, the walk ends and t is the answer.  Every token
// that leaves is the target's own choice, so the text is the target's whatever the tree held.
//
// A walk needs the rows it passes and no others, and which those are is known one after the other.  Two forms:
//   step by step   a launch per level of the tree.  Every request's workgroups first settle the level before (the pieces' results of that
//                  row, the token, the child), each for itself, and then scan a piece of the child's row.  Nothing is handed over inside a launch.
//   all rows       one launch that scans all rows of all trees, one that walks: where the rows are few.
// Sums of exponentials are float64 in a fixed order, so a draw does not depend on how the row was cut.
#include "sled_internal.h"

#include <algorithm>

namespace {

constexpr int THREADS = 256, MAX_PIECES = 64;

struct __align__(16) Piece {   // of a row
    double sum;   // of exp((x - m) / tau) (sampling)
    float m;      // largest logit
    int arg;      // its lowest id
};

struct walk_args {
    const float* logits;
    const int32_t* tokens;
    const float* u;          // one per row (sampling)
    double inv_tau;
    int V, pieces, seg, B;   // a row's pieces and their length
    const uint8_t* parent;   // [T] (root: 255)
    const int32_t* first;    // [B + 1] first row of a request
    Piece* part;             // step by step: [2][B][pieces]; all rows: [T][pieces]
    int32_t* cur;            // [2][B] node whose row was scanned last, -1: the walk has ended
    int32_t *accept_len, *path, *out_token;
};

__device__ inline void better(float& m, int& arg, float x, int i) {
    if (x > m || (x == m && i < arg)) {
        m = x;
        arg = i;
    }
}

// largest value and its lowest index over the workgroup, in every thread
__device__ inline void block_max(float& m, int& arg, float* sh_m, int* sh_i) {
    for (int off = 32; off > 0; off >>= 1) {
        const float x = __shfl_xor(m, off);
        const int i = __shfl_xor(arg, off);
        better(m, arg, x, i);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        sh_m[threadIdx.x >> 6] = m;
        sh_i[threadIdx.x >> 6] = arg;
    }
    __syncthreads();
    m = sh_m[0];
    arg = sh_i[0];
    for (int w = 1; w < THREADS / 64; w++) better(m, arg, sh_m[w], sh_i[w]);
}

// piece s of a row -> *out
template <bool SAMPLE>
__device__ void scan_piece(const walk_args& a, const float* __restrict__ row, int s, Piece* out) {
    __shared__ float sh_m[THREADS / 64];
    __shared__ int sh_i[THREADS / 64];
    __shared__ double sh_d[THREADS / 64];
    const int lo = s * a.seg, hi = min(a.V, lo + a.seg), tid = threadIdx.x;
    float m = -INFINITY;
    int arg = 0x7fffffff;
    int i = lo + tid;
    for (; i + 7 * THREADS < hi; i += 8 * THREADS) {   // eight loads in flight
        float x[8];
#pragma unroll
        for (int k = 0; k < 8; k++) x[k] = row[i + k * THREADS];
#pragma unroll
        for (int k = 0; k < 8; k++) better(m, arg, x[k], i + k * THREADS);
    }
    for (; i < hi; i += THREADS) better(m, arg, row[i], i);
    block_max(m, arg, sh_m, sh_i);
    double sum = 0.0;
    if (SAMPLE) {
        for (int k = lo + tid; k < hi; k += THREADS) sum += exp(((double)row[k] - (double)m) * a.inv_tau);
        for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off);
        if ((tid & 63) == 0) sh_d[tid >> 6] = sum;
        __syncthreads();
        sum = 0.0;
        for (int w = 0; w < THREADS / 64; w++) sum += sh_d[w];
    }
    if (tid == 0) *out = Piece{m > -INFINITY ? sum : 0.0, m, arg};
}

// the token that the target names behind a row, from the row's pieces; the whole workgroup takes part and gets it
template <bool SAMPLE>
__device__ int named_token(const walk_args& a, const float* __restrict__ row, const Piece* part, double u) {
    __shared__ int sh_tok, sh_seg;
    __shared__ double sh_rest, sh_wave[THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    __syncthreads();
    Piece p{0.0, -INFINITY, 0x7fffffff};
    if (lane < a.pieces) p = part[lane];
    float m = p.m;
    int arg = p.arg;
    for (int off = 32; off > 0; off >>= 1) {
        const float x = __shfl_xor(m, off);
        const int i = __shfl_xor(arg, off);
        better(m, arg, x, i);
    }
    if (!SAMPLE) return min(max(arg, 0), a.V - 1);
    // the piece in which the cumulative sum passes u of the total
    if (wave == 0) {
        const double w = p.sum > 0.0 ? p.sum * exp(((double)p.m - (double)m) * a.inv_tau) : 0.0;
        double c = w;
        for (int off = 1; off < 64; off <<= 1) {
            const double x = __shfl_up(c, off);
            if (lane >= off) c += x;
        }
        const double target = u * __shfl(c, 63);
        const uint64_t past = __ballot(c > target), some = __ballot(w > 0.0);
        // none (rounding, or a row without a finite value): the last piece that holds anything
        const int s = past ? __builtin_ctzll(past) : some ? 63 - __builtin_clzll(some) : 0;
        const double before = __shfl(c, max(s - 1, 0));
        if (lane == 0) {
            sh_seg = s;
            sh_rest = target - (s > 0 ? before : 0.0);
        }
    }
    __syncthreads();
    // within it, a run of neighbouring ids per thread
    const int lo = sh_seg * a.seg, hi = min(a.V, lo + a.seg), per = (a.seg + THREADS - 1) / THREADS;
    const double rest = sh_rest, md = (double)m;
    const int k0 = min(hi, lo + tid * per), k1 = min(hi, k0 + per);
    double mine = 0.0;
    int last = -1;   // last id with mass
    for (int k = k0; k < k1; k++) {
        const double e = exp(((double)row[k] - md) * a.inv_tau);
        mine += e;
        if (e > 0.0) last = k;
    }
    double c = mine;
    for (int off = 1; off < 64; off <<= 1) {
        const double x = __shfl_up(c, off);
        if (lane >= off) c += x;
    }
    if (lane == 63) sh_wave[wave] = c;
    if (tid == 0) sh_tok = 0x7fffffff;
    __syncthreads();
    double base = 0.0;
    for (int w = 0; w < wave; w++) base += sh_wave[w];
    if (base + c > rest) {   // the sum passes in this thread's run or before it
        double run = base + (c - mine);
        int tok = last;
        for (int k = k0; k < k1; k++) {
            run += exp(((double)row[k] - md) * a.inv_tau);
            if (run > rest) {
                tok = k;
                break;
            }
        }
        if (tok >= 0) atomicMin(&sh_tok, tok);
    }
    __syncthreads();
    int tok = sh_tok;
    if (tok == 0x7fffffff) {   // it never passes: the last id with mass
        __syncthreads();
        if (tid == 0) sh_tok = -1;
        __syncthreads();
        if (last >= 0) atomicMax(&sh_tok, last);
        __syncthreads();
        tok = sh_tok;
    }
    return min(max(tok, 0), a.V - 1);
}

// the child of `cur` (a node of the request whose first row is row0) that drafted `tok`, the lowest if there are several, or -1
__device__ inline int child_of(const walk_args& a, int row0, int n, int cur, int tok) {
    const int lane = threadIdx.x & 63;
    const bool hit = lane > 0 && lane < n && a.parent[row0 + min(lane, n - 1)] == cur && a.tokens[row0 + min(lane, n - 1)] == tok;
    const uint64_t hits = __ballot(hit);
    return hits ? __builtin_ctzll(hits) : -1;
}

// Level `level` of all walks: settle the level before, then scan a piece of the row of the node it led to.
template <bool SAMPLE>
__global__ __launch_bounds__(THREADS) void accept_tree_level(walk_args a, int level, int last_level) {
    const int s = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int row0 = a.first[b], n = a.first[b + 1] - row0;
    int cur = 0;
    if (level > 0) {
        const int before = a.cur[((level - 1) & 1) * a.B + b];
        cur = -1;
        if (before >= 0) {
            const float* row = a.logits + (size_t)(row0 + before) * a.V;
            const int tok = named_token<SAMPLE>(a, row, a.part + ((size_t)((level - 1) & 1) * a.B + b) * a.pieces, SAMPLE ? (double)a.u[row0 + before] : 0.0);
            cur = child_of(a, row0, n, before, tok);
            if (s == 0 && tid == 0) {
                if (cur >= 0) {
                    a.path[(size_t)b * SLED_TREE_MAX + level - 1] = cur;
                } else {
                    a.accept_len[b] = level - 1;
                    a.out_token[b] = tok;
                }
            }
        }
    }
    if (s == 0 && tid == 0) a.cur[(level & 1) * a.B + b] = cur;
    if (cur < 0 || last_level) return;
    scan_piece<SAMPLE>(a, a.logits + (size_t)(row0 + cur) * a.V, s, a.part + ((size_t)(level & 1) * a.B + b) * a.pieces + s);
}

template <bool SAMPLE>
__global__ __launch_bounds__(THREADS) void accept_tree_rows(walk_args a) {
    const int s = blockIdx.x, t = blockIdx.y;
    scan_piece<SAMPLE>(a, a.logits + (size_t)t * a.V, s, a.part + (size_t)t * a.pieces + s);
}

template <bool SAMPLE>
__global__ __launch_bounds__(THREADS) void accept_tree_walk(walk_args a) {
    const int b = blockIdx.x, row0 = a.first[b], n = a.first[b + 1] - row0;
    int cur = 0;
    for (int len = 0;; len++) {   // a child's number is larger than its parent's: at most n rounds
        const size_t t = row0 + cur;
        const int tok = named_token<SAMPLE>(a, a.logits + t * a.V, a.part + t * a.pieces, SAMPLE ? (double)a.u[t] : 0.0);
        const int next = child_of(a, row0, n, cur, tok);
        if (next < 0) {
            if (threadIdx.x == 0) {
                a.accept_len[b] = len;
                a.out_token[b] = tok;
            }
            return;
        }
        if (threadIdx.x == 0) a.path[(size_t)b * SLED_TREE_MAX + len] = next;
        cur = next;
    }
}

// The trees' shape comes by value with the launch (so the call needs no copy from host memory and can be captured): the parents
// in pieces, the sizes with the first.
constexpr int PARENTS = 2048;
struct __align__(16) Sizes {
    uint8_t n[1024];   // nodes - 1
};
struct __align__(16) Parents {
    uint8_t p[PARENTS];
};
__global__ __launch_bounds__(256) void accept_tree_setup(Parents pp, int at, int count, uint8_t* __restrict__ parent) {
    for (int i = threadIdx.x; i < count; i += 256) parent[at + i] = pp.p[i];
}
__global__ __launch_bounds__(256) void accept_tree_first(Sizes sz, int B, int32_t* __restrict__ first, int32_t* __restrict__ path) {
    __shared__ int sh[256];
    const int tid = threadIdx.x;
    int n[4], sum = 0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        n[k] = 4 * tid + k < B ? sz.n[4 * tid + k] + 1 : 0;
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
    for (int i = tid; i < B * SLED_TREE_MAX; i += 256) path[i] = -1;
}

int pick_pieces(int rows, int V) {
    // about 1024 workgroups a launch, none of less than 2048 values
    const int n = std::max(1, std::min(MAX_PIECES, 1024 / std::max(1, rows)));
    return std::max(1, std::min(n, V / 2048));
}
bool all_rows(int B, int T, int depth, int V) {
    (void)B;
    return (int64_t)T * V * 4 <= (int64_t)depth * (8 << 20);
}
size_t up(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

size_t sled_accept_tree_ws_bytes(int B, int T, int vocab) {
    const size_t parts = std::max((size_t)2 * B * pick_pieces(B, vocab), (size_t)T * pick_pieces(T, vocab)) * sizeof(Piece);
    return up(parts) + up((size_t)2 * B * 4) + up((size_t)(B + 1) * 4) + up(T);
}

int sled_launch_accept_tree(int mode, int B, int T, const int* n_nodes, const int* parent, int depth, int vocab, float temperature, const float* logits,
                            const int32_t* tokens, const float* u, int32_t* accept_len, int32_t* path, int32_t* out_token, void* ws, hipStream_t st) {
    walk_args a{};
    a.logits = logits;
    a.tokens = tokens;
    a.u = u;
    a.inv_tau = 1.0 / (double)temperature;
    a.V = vocab;
    a.B = B;
    const bool rows = all_rows(B, T, depth + 1, vocab);
    a.pieces = pick_pieces(rows ? T : B, vocab);
    a.seg = (vocab + a.pieces - 1) / a.pieces;
    char* w = static_cast<char*>(ws);
    a.part = reinterpret_cast<Piece*>(w);
    w += up(std::max((size_t)2 * B * pick_pieces(B, vocab), (size_t)T * pick_pieces(T, vocab)) * sizeof(Piece));
    a.cur = reinterpret_cast<int32_t*>(w);
    w += up((size_t)2 * B * 4);
    int32_t* first = reinterpret_cast<int32_t*>(w);
    w += up((size_t)(B + 1) * 4);
    uint8_t* par = reinterpret_cast<uint8_t*>(w);
    a.first = first;
    a.parent = par;
    a.accept_len = accept_len;
    a.path = path;
    a.out_token = out_token;
    Sizes sz;
    for (int i = 0; i < 1024; i++) sz.n[i] = i < B ? (uint8_t)(n_nodes[i] - 1) : 0;
    hipLaunchKernelGGL(accept_tree_first, dim3(1), dim3(256), 0, st, sz, B, first, path);
    SLED_LAUNCH_CHECK();
    for (int at = 0; at < T; at += PARENTS) {
        Parents pp;
        const int count = std::min(PARENTS, T - at);
        for (int i = 0; i < PARENTS; i++) pp.p[i] = i < count && parent[at + i] >= 0 ? (uint8_t)parent[at + i] : 255;
        hipLaunchKernelGGL(accept_tree_setup, dim3(1), dim3(256), 0, st, pp, at, count, par);
        SLED_LAUNCH_CHECK();
    }
    const bool sample = mode == SLED_SAMPLE;
    if (rows) {
        if (sample) hipLaunchKernelGGL(accept_tree_rows<true>, dim3(a.pieces, T), dim3(THREADS), 0, st, a);
        else hipLaunchKernelGGL(accept_tree_rows<false>, dim3(a.pieces, T), dim3(THREADS), 0, st, a);
        SLED_LAUNCH_CHECK();
        if (sample) hipLaunchKernelGGL(accept_tree_walk<true>, dim3(B), dim3(THREADS), 0, st, a);
        else hipLaunchKernelGGL(accept_tree_walk<false>, dim3(B), dim3(THREADS), 0, st, a);
        SLED_LAUNCH_CHECK();
        return SLED_OK;
    }
    for (int level = 0; level <= depth + 1; level++) {
        const bool last = level == depth + 1;
        const dim3 grid(last ? 1 : a.pieces, B);
        if (sample) hipLaunchKernelGGL(accept_tree_level<true>, grid, dim3(THREADS), 0, st, a, level, (int)last);
        else hipLaunchKernelGGL(accept_tree_level<false>, grid, dim3(THREADS), 0, st, a, level, (int)last);
        SLED_LAUNCH_CHECK();
    }
    return SLED_OK;
}
