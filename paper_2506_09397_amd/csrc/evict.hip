// A request's cache cut down to the tokens that attention uses, and the accepted path of a tree made contiguous.
//
// Eviction, per (layer, kv head) of a request with L tokens: kept are the first `first` and the last `recent` positions and, of those
// between, the keep - first - recent with the largest mass (equal masses: the lower position).  Kept tokens move together in
// ascending order, so token i of the result is the kept token of rank i, with its mass; all layers and heads keep the same number, so
// the request stays one length and one page list while every head keeps its own tokens.
//
//   evict_select_kernel   a workgroup per (layer, kv head) and request.  The smallest mass that is kept is found digit by digit: four passes over
//                         the masses, in registers (beyond 8192 tokens in L2), each counting one byte of the values that agree so far with the bytes already known
//                         in a histogram in LDS.  A last pass in ascending order gives every kept token its rank.
//   evict_move_kernel     a workgroup per (layer, kv head), request and run of 64-token pieces.  A token of rank i moves down or stays (its
//                         position is at least i), so a workgroup that reads a piece's 64 tokens before it writes them may work in place, piece
//                         by piece; into another request's pages pieces are independent and go to several workgroups.
//                         K moves in 16-byte pieces (8 dims of a token); the V pages hold four tokens of a dim together, so every V value is
//                         picked from the 16 bytes that its quad has of two dims, and four tokens are written together.
// What bounds it: memory.  A line of 128 bytes holds pieces of eight tokens (K) or four tokens of 16 dims (V), so with a third of the tokens kept most
// lines are fetched whole: 8 requests of 27803 tokens in all cut to 1111 each, 32 layers of 8 heads of 128: 2.8 of 3.6 GB fetched and 1.1 written in
// 789 us, 5.0 TB/s; the kept tokens alone would be 2.3 GB.  One request of 2048 tokens cut to 1024: 85 us for 0.4 GB (96 with two loads of 2 bytes
// for each value of V in place of one of 16).  Choosing takes 44 and 9 us
// (55 and 12 with each pass over the masses out of L2).  In place, a workgroup a head: 809 and 79 us, choosing 46 and 11.
#include "sled_internal.h"

#include <type_traits>

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int SEL_THREADS = 512, HELD = 16, PIECE = 64;   // masses that a thread holds; tokens of a piece: four pages

// orders like the float, as an unsigned number (+0 and -0 alike)
__device__ inline uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct evict_args {
    const int32_t* meta;   // per request SLED_EVICT_REC ints: source, destination, tokens to keep, first entry of its pages, of the destination's
    const int32_t* pages;
    int32_t *len_dev, *shift_dev;
    float* mass;           // [request][layer][kv head][cap]
    int cap, n_layers, Hkv, D, first, recent;
    int32_t* idx;          // [request][layer][kv head][idx_cap]
    int idx_cap;
    void *k_pool, *v_pool;
    int64_t n_pages;
};

__global__ __launch_bounds__(SEL_THREADS) void evict_select_kernel(evict_args a) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t sh_prefix, sh_want;
    __shared__ int sh_eq[SEL_THREADS / 64], sh_keep[SEL_THREADS / 64];
    const int lh = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int32_t* rec = a.meta + SLED_EVICT_REC * b;
    const int src = rec[0], dst = rec[1], L = a.len_dev[src], keep = min(L, rec[2]);
    const size_t n_lh = (size_t)a.n_layers * a.Hkv;
    const float* m = a.mass + (src * n_lh + lh) * a.cap;
    float* out = a.mass + (dst * n_lh + lh) * a.cap;
    int32_t* idx = a.idx + (b * n_lh + lh) * a.idx_cap;
    if (src != dst && lh == 0 && tid == 0) {   // (nobody reads the destination's length in this call)
        a.shift_dev[dst] = a.shift_dev[src] + L - keep;
        a.len_dev[dst] = keep;
    }
    if (keep == L) {   // everything stays
        if (src == dst) return;
        for (int i = tid; i < L; i += SEL_THREADS) {
            idx[i] = i;
            out[i] = m[i];
        }
        return;
    }
    // up to 8192 tokens: read once, and all at a time
    const bool held = L <= HELD * SEL_THREADS;
    float x[HELD];
    if (held) {
#pragma unroll
        for (int r = 0; r < HELD; r++) {
            if (r * SEL_THREADS >= L) break;
            x[r] = m[min(r * SEL_THREADS + tid, L - 1)];
        }
    }
    const int lo = a.first, hi = L - a.recent;   // the positions to choose from; more of them than are wanted, since keep < L
    const uint32_t want = keep - a.first - a.recent;
    uint32_t prefix = 0, left = want;   // the kept masses' smallest key so far, and how many of the keys that share it are kept
    if (want > 0) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += SEL_THREADS) hist[i] = 0;
            __syncthreads();
            const uint32_t known = shift == 24 ? 0u : ~0u << (shift + 8);
            auto count = [&](float v) {
                const uint32_t k = order_key(v);
                if ((k & known) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            };
            if (held) {
#pragma unroll
                for (int r = 0; r < HELD; r++) {
                    if (r * SEL_THREADS >= hi) break;
                    const int i = r * SEL_THREADS + tid;
                    if (i >= lo && i < hi) count(x[r]);
                }
            } else {
                for (int i = lo + tid; i < hi; i += SEL_THREADS) count(m[i]);
            }
            __syncthreads();
            if (wave == 0) {
                // lane l holds the digits 255 - 4 l .. 252 - 4 l, largest first: how many keys lie above each
                uint32_t c[4], s = 0;
#pragma unroll
                for (int u = 0; u < 4; u++) s += c[u] = hist[255 - 4 * lane - u];
                uint32_t above = s;
                for (int off = 1; off < 64; off <<= 1) {
                    const uint32_t x = __shfl_up(above, off);
                    if (lane >= off) above += x;
                }
                above -= s;
#pragma unroll
                for (int u = 0; u < 4; u++) {
                    if (above < left && above + c[u] >= left) {   // one digit of one lane
                        sh_prefix = prefix | (uint32_t)(255 - 4 * lane - u) << shift;
                        sh_want = left - above;
                    }
                    above += c[u];
                }
            }
            __syncthreads();
            prefix = sh_prefix;
            left = sh_want;
        }
    }
    // ranks, 512 positions at a time: kept are keys above the prefix and the first `left` of those equal to it
    int n_kept = 0, n_eq = 0;
    auto place = [&](int i, float v) {
        asm volatile("" : : "v"(v));   // (it has arrived before the barriers behind which it may be overwritten)
        const bool mid = i >= lo && i < hi;
        const uint32_t k = order_key(v);
        const bool eq = mid && want > 0 && k == prefix;
        const uint64_t eqs = __ballot(eq), below = (1ull << lane) - 1ull;
        if (lane == 0) sh_eq[wave] = __popcll(eqs);
        __syncthreads();
        int rank_eq = n_eq + __popcll(eqs & below), all_eq = 0;
#pragma unroll
        for (int v = 0; v < SEL_THREADS / 64; v++) {
            if (v < wave) rank_eq += sh_eq[v];
            all_eq += sh_eq[v];
        }
        const bool kept = i < L && (!mid || (want > 0 && (k > prefix || (eq && rank_eq < (int)left))));
        const uint64_t keeps = __ballot(kept);
        if (lane == 0) sh_keep[wave] = __popcll(keeps);
        __syncthreads();   // (every mass of these positions has been read: the ones below may be overwritten)
        int rank = n_kept + __popcll(keeps & below), all = 0;
#pragma unroll
        for (int v = 0; v < SEL_THREADS / 64; v++) {
            if (v < wave) rank += sh_keep[v];
            all += sh_keep[v];
        }
        if (kept) {
            idx[rank] = i;
            out[rank] = v;
        }
        n_eq += all_eq;
        n_kept += all;
    };
    if (held) {
#pragma unroll
        for (int r = 0; r < HELD; r++) {
            if (r * SEL_THREADS >= L) break;
            place(r * SEL_THREADS + tid, x[r]);
        }
    } else {
        for (int i0 = 0; i0 < L; i0 += SEL_THREADS) place(i0 + tid, i0 + tid < L ? m[i0 + tid] : 0.f);
    }
    __syncthreads();
    for (int i = keep + tid; i < L; i += SEL_THREADS) out[i] = 0.f;
}

template <int D, bool F32, bool INPLACE>
__global__ __launch_bounds__(256) void evict_move_kernel(evict_args a) {
    using T = std::conditional_t<F32, float, bf16_t>;
    const int lh = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int32_t* rec = a.meta + SLED_EVICT_REC * b;
    const int L = a.len_dev[rec[0]], keep = min(L, rec[2]);
    if (INPLACE && keep == L) return;
    const int32_t *from = a.pages + rec[3], *to = a.pages + rec[4];
    const int32_t* idx = a.idx + ((size_t)b * a.n_layers * a.Hkv + lh) * a.idx_cap;
    const size_t head = (size_t)16 * D, layer_page = (size_t)(lh / a.Hkv) * a.n_pages;
    const int g = lh % a.Hkv;
    auto at = [&](const int32_t* pages, int page) { return ((layer_page + pages[page]) * a.Hkv + g) * head; };
    T *kp = static_cast<T*>(a.k_pool), *vp = static_cast<T*>(a.v_pool);
    __shared__ int sh_slot[PIECE];
    __shared__ size_t sh_at[PIECE];
    auto arrived = [] {   // every thread's share of the piece is in its registers
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    for (int i0 = blockIdx.z * PIECE; i0 < keep; i0 += gridDim.z * PIECE) {
        const int n = min(PIECE, keep - i0);
        if (INPLACE && idx[i0 + n - 1] == i0 + n - 1) continue;   // ranks ascend with positions: none of these moves
        __syncthreads();
        if (tid < PIECE) {
            const int s = idx[i0 + min(tid, n - 1)];   // behind the last token: that token again
            sh_slot[tid] = s & 15;
            sh_at[tid] = at(from, s >> 4);
        }
        __syncthreads();
        if constexpr (!F32) {
            // K: 16 bytes of token e16 of the page; V: four tokens (quad q4) of two dims, each out of the 16 bytes that its own quad has of them
            u32x4 k[4], v[4][4];
            const int c4 = tid >> 6, q4 = (tid >> 4) & 3, e16 = tid & 15;
#pragma unroll
            for (int p = 0; p < 4; p++) {
                if (p * 16 >= n) break;
                k[p] = *reinterpret_cast<const u32x4*>(kp + sh_at[p * 16 + e16] + (c4 * 64 + q4 * 16 + sh_slot[p * 16 + e16]) * 8);
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int t = p * 16 + q4 * 4 + i;
                    v[p][i] = *reinterpret_cast<const u32x4*>(vp + sh_at[t] + (c4 * 64 + (sh_slot[t] >> 2) * 16 + e16) * 8);
                }
            }
            if (INPLACE) arrived();
#pragma unroll
            for (int p = 0; p < 4; p++) {
                if (p * 16 >= n) break;
                const size_t d = at(to, (i0 >> 4) + p) + (size_t)tid * 8;
                *reinterpret_cast<u32x4*>(kp + d) = k[p];
                uint32_t x[4][2];
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const int s = sh_slot[p * 16 + q4 * 4 + i], half = (s & 1) * 16;
                    x[i][0] = (((s & 2) ? v[p][i][1] : v[p][i][0]) >> half) & 0xffffu;
                    x[i][1] = (((s & 2) ? v[p][i][3] : v[p][i][2]) >> half) & 0xffffu;
                }
                *reinterpret_cast<u32x4*>(vp + d) = u32x4{x[0][0] | (x[1][0] << 16), x[2][0] | (x[3][0] << 16), x[0][1] | (x[1][1] << 16), x[2][1] | (x[3][1] << 16)};
            }
        } else {
            constexpr int CH = D / 4, N = PIECE * CH / 256;   // 16-byte pieces of a token; of this thread
            u32x4 k[N], v[N];
#pragma unroll
            for (int u = 0; u < N; u++) {
                const int e = u * 256 + tid, t = e / CH, c = e % CH;
                const size_t x = sh_at[t] + sh_slot[t] * D + c * 4;
                k[u] = *reinterpret_cast<const u32x4*>(kp + x);
                v[u] = *reinterpret_cast<const u32x4*>(vp + x);
            }
            if (INPLACE) arrived();
#pragma unroll
            for (int u = 0; u < N; u++) {
                const int e = u * 256 + tid, t = e / CH, c = e % CH;
                if (t >= n) continue;
                const size_t x = at(to, (i0 + t) >> 4) + ((i0 + t) & 15) * D + c * 4;
                *reinterpret_cast<u32x4*>(kp + x) = k[u];
                *reinterpret_cast<u32x4*>(vp + x) = v[u];
            }
        }
    }
}

// lengths after an eviction in place (the choice sets those of other destinations); the tokens to come keep the positions they would have had
__global__ void evict_len_kernel(evict_args a, int B) {
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b >= B) return;
    const int32_t* rec = a.meta + SLED_EVICT_REC * b;
    const int L = a.len_dev[rec[0]], keep = min(L, rec[2]);
    a.shift_dev[rec[1]] = a.shift_dev[rec[0]] + L - keep;
    a.len_dev[rec[1]] = keep;
}

// How much of a path is one: the leading entries that ascend within 1 .. n-1, at most accept_len of them.  The whole wavefront calls it;
// lane j gets entry j in *node.
__device__ inline int path_length(const int32_t* __restrict__ path, int accept_len, int n, int lane, int* node) {
    const int most = min(min(accept_len, n - 1), SLED_TREE_MAX - 1);
    const int x = lane < most ? path[lane] : -1, before = lane > 0 && lane < most ? path[lane - 1] : 0;
    *node = x;
    const uint64_t wrong = __ballot(lane >= most || x <= before || x >= n);
    return __builtin_ctzll(wrong);   // (lane 63 never holds an entry)
}

struct commit_args {
    const int32_t* meta;    // per request 3 ints: id, nodes staged, first entry of its pages
    const int32_t* pages;
    int32_t* len_dev;
    const int32_t *accept_len, *path;   // [B], [B][SLED_TREE_MAX]
    float* mass;                        // or nullptr
    int32_t* tail;                      // with mass: where nodes have some
    int cap, n_layers, Hkv, D;
    void *k_pool, *v_pool;
    int64_t n_pages;
};

// Tail slot 1 + j of a request takes what node path[j] staged.  A thread owns the same dims of every token, and the path ascends (path[j] is at
// least 1 + j), so nothing is overwritten before it has been read.
template <int D, bool F32>
__global__ __launch_bounds__(256) void tree_commit_kernel(commit_args a) {
    using T = std::conditional_t<F32, float, bf16_t>;
    constexpr int E = 16 / sizeof(T), CH = D / E;   // values of 16 bytes, pieces of a token
    const int layer = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
    const int32_t* rec = a.meta + 3 * b;
    const int n = rec[1], L = a.len_dev[rec[0]];
    const int32_t* pages = a.pages + rec[2];
    int node;
    const int len = path_length(a.path + (size_t)b * SLED_TREE_MAX, a.accept_len[b], n, lane, &node);
    __shared__ int sh_from[SLED_TREE_MAX], sh_page[SLED_TREE_MAX];   // position of a node; physical page of a tail slot
    if (tid < 64) {
        sh_from[lane] = lane < len ? L + node : L + 1 + lane;
        sh_page[lane] = lane < n ? pages[(L + lane) >> 4] : 0;
    }
    __syncthreads();
    const size_t head = (size_t)16 * D, layer_page = (size_t)layer * a.n_pages;
    const int first = __builtin_ctzll(__ballot(lane >= len || node != 1 + lane));   // the entries before stay where they are
    for (int e = tid; e < a.Hkv * 2 * CH; e += 256) {
        const bool isv = e >= a.Hkv * CH;
        const int g = e / CH % a.Hkv, d = e % CH * E;
        T* pool = static_cast<T*>(isv ? a.v_pool : a.k_pool);
        auto page = [&](int pos) { return pool + ((layer_page + sh_page[pos - L]) * a.Hkv + g) * head; };
        for (int j0 = first; j0 < len; j0 += 4) {
            union {
                uint4 u;
                T x[E];
            } r[4];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                if (j0 + u >= len) break;
                const int pos = sh_from[j0 + u];
                const T* p = page(pos);
                if constexpr (F32) {
                    r[u].u = *reinterpret_cast<const uint4*>(p + (pos & 15) * D + d);
                } else if (!isv) {
                    r[u].u = *reinterpret_cast<const uint4*>(p + kpage_offset(pos & 15, d));
                } else {
#pragma unroll
                    for (int i = 0; i < E; i++) r[u].x[i] = p[vpage_offset(pos & 15, d + i)];
                }
            }
#pragma unroll
            for (int u = 0; u < 4; u++) {
                if (j0 + u >= len) break;
                const int pos = L + 1 + j0 + u;
                T* p = page(pos);
                if constexpr (F32) {
                    *reinterpret_cast<uint4*>(p + (pos & 15) * D + d) = r[u].u;
                } else if (!isv) {
                    *reinterpret_cast<uint4*>(p + kpage_offset(pos & 15, d)) = r[u].u;
                } else {
#pragma unroll
                    for (int i = 0; i < E; i++) p[vpage_offset(pos & 15, d + i)] = r[u].x[i];
                }
            }
        }
    }
    if (a.mass) {   // a wavefront per kv head; the rejected nodes' mass goes
        for (int g = tid >> 6; g < a.Hkv; g += 4) {
            float* m = a.mass + (((size_t)rec[0] * a.n_layers + layer) * a.Hkv + g) * a.cap;
            const float x = lane < len ? m[sh_from[lane]] : 0.f;
            if (1 + lane < n) m[L + 1 + lane] = x;
        }
    }
}

__global__ __launch_bounds__(64) void tree_len_kernel(commit_args a) {
    const int b = blockIdx.x, lane = threadIdx.x;
    const int32_t* rec = a.meta + 3 * b;
    int node;
    const int len = path_length(a.path + (size_t)b * SLED_TREE_MAX, a.accept_len[b], rec[1], lane, &node);
    if (lane == 0) a.len_dev[rec[0]] += len + 1;
    if (a.mass && lane < 2) a.tail[2 * rec[0] + lane] = 0;
}

// Once before a step's nodes get mass, or where mass is read: what nodes that were dropped have left behind goes (up to 64 slots of every layer and
// head), and where those of the step lie is noted.  A workgroup per request.
__global__ __launch_bounds__(256) void mass_open_kernel(sled_mass_ids ids, const int32_t* __restrict__ len_dev, int32_t* __restrict__ tail, float* __restrict__ mass,
                                                        int cap, int n_lh) {
    const int r = ids.id[blockIdx.x], nodes = ids.nodes[blockIdx.x], from = tail[2 * r], n = ids.left[blockIdx.x] ? min(tail[2 * r + 1], cap) - from : 0;
    for (int i = threadIdx.x; i < n_lh * n; i += 256) mass[((size_t)r * n_lh + i / n) * cap + from + i % n] = 0.f;
    __syncthreads();
    if (threadIdx.x < 2) tail[2 * r + threadIdx.x] = nodes ? len_dev[r] + threadIdx.x * nodes : 0;
}

template <int D, bool F32>
int launch_move(const evict_args& a, int B, bool in_place, int split, hipStream_t st) {
    const dim3 grid(a.n_layers * a.Hkv, B, split);
    if (in_place) hipLaunchKernelGGL((evict_move_kernel<D, F32, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((evict_move_kernel<D, F32, false>), grid, dim3(256), 0, st, a);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}

}  // namespace

int sled_launch_evict(const sled_model* m, const sled_kvpool* p, const int32_t* meta, const int32_t* pages, int B, int keep_max, int first, int recent, float* mass,
                      int cap, int32_t* idx, int idx_cap, bool in_place, hipStream_t st) {
    const sled_shape& s = m->s;
    evict_args a{meta, pages, p->len_dev, p->shift_dev, mass, cap, s.n_layers, s.n_kv_heads, s.head_dim, first, recent, idx, idx_cap, p->k_pool, p->v_pool, p->n_pages};
    hipLaunchKernelGGL(evict_select_kernel, dim3(s.n_layers * s.n_kv_heads, B), dim3(SEL_THREADS), 0, st, a);
    SLED_LAUNCH_CHECK();
    // several workgroups for a head's pieces where the heads alone are too few for the card
    const int64_t heads = (int64_t)s.n_layers * s.n_kv_heads * B, pieces = (keep_max + PIECE - 1) / PIECE;
    const int split = in_place ? 1 : (int)std::max<int64_t>(1, std::min(pieces, (4096 + heads - 1) / heads));
    int rc;
    if (s.dtype == SLED_BF16) rc = launch_move<128, false>(a, B, in_place, split, st);
    else rc = s.head_dim == 64 ? launch_move<64, true>(a, B, in_place, split, st) : launch_move<128, true>(a, B, in_place, split, st);
    if (rc != SLED_OK) return rc;
    if (in_place) {
        hipLaunchKernelGGL(evict_len_kernel, dim3((B + 63) / 64), dim3(64), 0, st, a, B);
        SLED_LAUNCH_CHECK();
    }
    return SLED_OK;
}

int sled_launch_mass_open(const sled_model* m, const sled_kvpool* p, const sled_mass_ids& ids, int n, float* mass, int cap, hipStream_t st) {
    hipLaunchKernelGGL(mass_open_kernel, dim3(n), dim3(256), 0, st, ids, p->len_dev, p->tail_dev, mass, cap, m->s.n_layers * m->s.n_kv_heads);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}

int sled_launch_tree_commit(const sled_model* m, const sled_kvpool* p, const int32_t* meta, const int32_t* pages, int B, const int32_t* accept_len,
                            const int32_t* path, float* mass, int cap, hipStream_t st) {
    const sled_shape& s = m->s;
    commit_args a{meta, pages, p->len_dev, accept_len, path, mass, p->tail_dev, cap, s.n_layers, s.n_kv_heads, s.head_dim, p->k_pool, p->v_pool, p->n_pages};
    const dim3 grid(s.n_layers, B);
    if (s.dtype == SLED_BF16) hipLaunchKernelGGL((tree_commit_kernel<128, false>), grid, dim3(256), 0, st, a);
    else if (s.head_dim == 64) hipLaunchKernelGGL((tree_commit_kernel<64, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((tree_commit_kernel<128, true>), grid, dim3(256), 0, st, a);
    SLED_LAUNCH_CHECK();
    hipLaunchKernelGGL(tree_len_kernel, dim3(B), dim3(64), 0, st, a);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}
