// Attention for trees of drafted tokens over the paged K/V cache, and the weight that cached tokens get from it.
//
// Request i has L_i context tokens in the pool and a tree of n_i <= 64 nodes: node 0 is the pending token, node j continues node
// parent[j] < j.  A node sees the whole context, its ancestors and itself; which nodes those are is one 64-bit word per node.
// With A(j) the ancestors of j and j itself, for query head h of kv head g = h / G:
//   s_t = q_jh . K_gt / sqrt(D)   (t < L, and the nodes t in A(j))
//   lse = log sum exp(s_t),   out = sum exp(s_t - lse) V_gt
//
// tree_attention_kernel, per work item (request, kv head, group of 16 NT stacked rows, run of context pages):
//   All G heads of all nodes are stacked into tiles of 16 rows (row r = node r / G, head r % G), so that K and V are read once for up to 64
//   rows.  A workgroup is four wavefronts that share nothing while they read: each takes every fourth pair of pages straight
//   from memory into its registers, in the operand order that pages are stored in, PFB pairs ahead, and multiplies
//   it with every row tile.  No barrier and no LDS traffic but the queries' operands stand in the loop.
//     S^T[32 tokens, 16 rows] = K Q^T    v_mfma_f32_16x16x32_bf16, page by page
//     O^T[128 dims, 16 rows] += V^T P^T  the same instruction over both pages at once: a lane holds, of S^T, the four tokens of its
//                                        quad in each page, and these eight are its part of the operand P^T, as the quads of V are of V^T
//   p = 2^(s' - M), s' in log2 units, M a whole number that a row raises when some s' passes it by more than 8; every rescale is then an
//   exact power of two, so neither the order of the pages nor their split over wavefronts changes how p is rounded.  p enters the second product as
//   a bf16 pair (16 bits), which costs 8 of 24 instructions: with a single bf16 the error would be that of the output's own
//   rounding once more.  Sums are float32.
//   The tree's own keys and values come from the caller's k and v through an LDS image in page order, as one or two more steps under the
//   ancestors' bits; the item that reads them also writes them into the request's tail slots, which nobody reads in this launch.
//   The wavefronts' states are added up through LDS; the items of a (request, kv head, row group) store theirs and the last to arrive adds
//   them up in ascending order.
//   fp32 models: the same with v_mfma_f32_16x16x4_f32 and single pages.
// A value that is not finite must not reach the rows that do not see its node (0 * inf is NaN): such values of v are left out of the
// product and added at the end for the rows that do see them.  Slots of the last context page behind L count as zero.
#include "sled_internal.h"

#include <type_traits>

namespace {

constexpr float NEG_BIG = -1.0e30f;
constexpr int WAVES = 4;

// (vectors of the compiler's own: structs of four would not stay in registers where their parts are used)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// sizes of one step of the page loop
template <int D, bool F32>
struct Geo {
    static constexpr int P = F32 ? 1 : 2;        // pages
    static constexpr int TOK = 16 * P;           // tokens
    static constexpr int DT = D / 16;            // tiles of 16 dims of an output
    static constexpr int OWN = DT / WAVES;       // of them, the ones a wavefront adds up at the end
    static constexpr int QC = F32 ? D / 16 : 4;  // operand pieces (16 bytes a lane) of a row tile, per plane
    static constexpr int ELEM = F32 ? 4 : 2;
};

// one step's K and V as the lanes hold them
template <int D, bool F32>
struct KV {
    u32x4 k[2][4];   // [page][32 dims]: token lane % 16, dims (lane / 16) * 8 ..
    u32x4 v[2][4];   // [page][32 dims]: tokens (lane / 16) * 4 .. + 3 of dim lane % 16, then of dim lane % 16 + 16
};
template <int D>
struct KV<D, true> {
    f32x4 k[D / 16];      // token lane % 16, dims 16 c + (lane / 16) * 4 ..
    float v[D / 16][4];   // token (lane / 16) * 4 + i, dim 16 dt + lane % 16
};

template <int D, bool F32>
__device__ __forceinline__ void load_page(KV<D, F32>& kv, int sub, const void* kp, const void* vp, int lane) {
    if constexpr (!F32) {
#pragma unroll
        for (int c = 0; c < 4; c++) kv.k[sub][c] = reinterpret_cast<const u32x4*>(kp)[c * 64 + lane];
#pragma unroll
        for (int c = 0; c < 4; c++) kv.v[sub][c] = reinterpret_cast<const u32x4*>(vp)[c * 64 + lane];
    } else {
        const float* k = static_cast<const float*>(kp) + (lane & 15) * D + (lane >> 4) * 4;
        const float* v = static_cast<const float*>(vp) + (lane >> 4) * 4 * D + (lane & 15);
#pragma unroll
        for (int c = 0; c < D / 16; c++) kv.k[c] = *reinterpret_cast<const f32x4*>(k + 16 * c);
#pragma unroll
        for (int dt = 0; dt < D / 16; dt++)
#pragma unroll
            for (int i = 0; i < 4; i++) kv.v[dt][i] = v[i * D + dt * 16];
    }
}

// values of tokens lim .. of the step become zero
template <int D, bool F32>
__device__ __forceinline__ void cut_values(KV<D, F32>& kv, int lim, int lane) {
    const int t0 = (lane >> 4) * 4;
    if constexpr (!F32) {
#pragma unroll
        for (int p = 0; p < 2; p++) {
            const int t = p * 16 + t0;
            const uint32_t a = (t < lim ? 0xffffu : 0u) | (t + 1 < lim ? 0xffff0000u : 0u), b = (t + 2 < lim ? 0xffffu : 0u) | (t + 3 < lim ? 0xffff0000u : 0u);
#pragma unroll
            for (int c = 0; c < 4; c++) kv.v[p][c] &= u32x4{a, b, a, b};
        }
    } else {
#pragma unroll
        for (int dt = 0; dt < D / 16; dt++)
#pragma unroll
            for (int i = 0; i < 4; i++) kv.v[dt][i] = t0 + i < lim ? kv.v[dt][i] : 0.f;
    }
}

__device__ __forceinline__ float max_over_groups(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_groups(float x) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// S^T of one page (A operand K, B operand Q) or, SWAP, S (A operand Q, B operand K) of a row tile
template <int D, bool F32, int PL, bool SWAP>
__device__ __forceinline__ float4_t page_scores(const KV<D, F32>& kv, int sub, const u32x4* q /* the tile's operand pieces + lane */) {
    float4_t s = {0.f, 0.f, 0.f, 0.f};
    if constexpr (!F32) {
#pragma unroll
        for (int ks = 0; ks < 4; ks++) {
            const bf16x8_t k = __builtin_bit_cast(bf16x8_t, kv.k[sub][ks]);
#pragma unroll
            for (int pl = 0; pl < PL; pl++) {
                const bf16x8_t x = __builtin_bit_cast(bf16x8_t, q[(pl * 4 + ks) * 64]);
                s = SWAP ? __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, k, s, 0, 0, 0) : __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, x, s, 0, 0, 0);
            }
        }
    } else {
#pragma unroll
        for (int c = 0; c < D / 16; c++) {
            const f32x4 kk = kv.k[c], xx = __builtin_bit_cast(f32x4, q[c * 64]);
#pragma unroll
            for (int e = 0; e < 4; e++)
                s = SWAP ? __builtin_amdgcn_mfma_f32_16x16x4f32(xx[e], kk[e], s, 0, 0, 0) : __builtin_amdgcn_mfma_f32_16x16x4f32(kk[e], xx[e], s, 0, 0, 0);
        }
    }
    return s;
}

// where the operand piece of row r (of its tile), 16 bytes number c of the row, sits among a tile's pieces of one plane
template <bool F32>
__device__ __forceinline__ int q_piece(int r, int c) {
    return (c >> 2) * 64 + (c & 3) * 16 + r;
}

struct tree_args {
    sled_tree_plan t;
    const int32_t* len_dev;
    const void* q;             // rows of n_q_heads * D, q_stride elements apart
    size_t q_stride, q_plane;  // PAIR: distance of the low plane
    const void *k, *v;         // rows of n_kv_heads * D, k_stride and v_stride elements apart
    size_t k_stride, v_stride;
    void *k_pool, *v_pool;
    int64_t n_pages;
    int layer, Hq, Hkv;
    float scale_log2;
    void* out;                 // rows of n_q_heads * D; STEP and bf16: operand order of the following projection, two planes
    size_t x_plane;
    float* lse;                // or nullptr
};

// Copies rows r0 .. r0 + n_rows - 1 of a block's stacked rows into LDS, as the operand pieces of their tiles; rows from `rows` on are zero
template <int D, bool F32, int PL>
__device__ __forceinline__ void stage_queries(u32x4* qs, const tree_args& a, int row0, int g, int G, int r0, int n_rows, int rows, int tid, int nt) {
    constexpr int CH = D * Geo<D, F32>::ELEM / 16;   // 16-byte pieces of a row
    for (int e = tid; e < n_rows * PL * CH; e += nt) {
        const int c = e % CH, pl = e / CH % PL, rr = e / (CH * PL);
        u32x4 x = {0u, 0u, 0u, 0u};
        if (r0 + rr < rows) {
            const int j = (r0 + rr) / G, hh = (r0 + rr) - j * G;
            const size_t at = (pl * a.q_plane + (size_t)(row0 + j) * a.q_stride + (size_t)(g * G + hh) * D) * Geo<D, F32>::ELEM + c * 16;
            x = *reinterpret_cast<const u32x4*>(static_cast<const char*>(a.q) + at);
        }
        qs[((rr >> 4) * PL + pl) * CH * 16 + q_piece<F32>(rr & 15, c)] = x;
    }
}

// The running state of a wavefront: row lane % 16 of every tile, dims 16 dt + (lane / 16) * 4 + e
template <int NT, int DT>
struct State {
    float m[NT], l[NT];
    float4_t o[NT][DT];
};

// One step (16 P tokens) against the first n_tiles row tiles.  MASKED: bit t of bits[tile] says whether this lane's row sees token t.
template <int NT, int D, bool F32, int PL, bool MASKED>
__device__ __forceinline__ void tile_steps(const KV<D, F32>& kv, const u32x4* qs, int lane, int n_tiles, float c, const uint32_t* bits, State<NT, D / 16>& st) {
    constexpr int P = Geo<D, F32>::P, DT = Geo<D, F32>::DT, QT = Geo<D, F32>::QC * 64 * PL;
    const int t0 = (lane >> 4) * 4;
    if (NT >= 4) asm volatile("" ::: "memory");   // the queries' operands are read again in every step: there are not registers for all
#pragma unroll
    for (int t = 0; t < NT; t++) {
        if (t >= n_tiles) break;
        float4_t s[P];
#pragma unroll
        for (int p = 0; p < P; p++) s[p] = page_scores<D, F32, PL, false>(kv, p, qs + t * QT + lane);
        if (MASKED) {
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int i = 0; i < 4; i++) s[p][i] = (bits[t] >> (p * 16 + t0 + i)) & 1u ? s[p][i] : -INFINITY;
        }
        float x[P][4], top = -INFINITY;
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int i = 0; i < 4; i++) {
                x[p][i] = fmaf(s[p][i], c, -st.m[t]);
                top = fmaxf(top, x[p][i]);
            }
        if (__builtin_amdgcn_ballot_w64(top > 8.f) != 0ull) {
            // some row's reference is too low: raise it to a whole number (row by row; the four lanes of a row agree)
            float hi = s[0][0];
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int i = 0; i < 4; i++) hi = fmaxf(hi, s[p][i]);
            const float mnew = fmaxf(st.m[t], ceilf(max_over_groups(hi) * c));
            const float alpha = __builtin_amdgcn_exp2f(st.m[t] - mnew);
            st.m[t] = mnew;
            st.l[t] *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; dt++)
#pragma unroll
                for (int e = 0; e < 4; e++) st.o[t][dt][e] *= alpha;
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int i = 0; i < 4; i++) x[p][i] = fmaf(s[p][i], c, -mnew);
        }
        float ps = 0.f;
        if constexpr (!F32) {
            bf16x8_t ph, pl;
#pragma unroll
            for (int p = 0; p < 2; p++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    const float w = __builtin_amdgcn_exp2f(x[p][i]);
                    ps += w;
                    const __bf16 h = (__bf16)w;   // to nearest even
                    ph[p * 4 + i] = h;
                    pl[p * 4 + i] = (__bf16)(w - (float)h);
                }
#pragma unroll
            for (int dt = 0; dt < DT; dt++) {
                const u32x4 a = kv.v[0][dt >> 1], b = kv.v[1][dt >> 1];
                const bf16x8_t va = __builtin_bit_cast(bf16x8_t, (dt & 1) ? __builtin_shufflevector(a, b, 2, 3, 6, 7) : __builtin_shufflevector(a, b, 0, 1, 4, 5));
                st.o[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, ph, st.o[t][dt], 0, 0, 0);
                st.o[t][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, pl, st.o[t][dt], 0, 0, 0);
            }
        } else {
            float w[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                w[i] = __builtin_amdgcn_exp2f(x[0][i]);
                ps += w[i];
            }
#pragma unroll
            for (int dt = 0; dt < DT; dt++)
#pragma unroll
                for (int i = 0; i < 4; i++) st.o[t][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(kv.v[dt][i], w[i], st.o[t][dt], 0, 0, 0);
        }
        st.l[t] += ps;
    }
}

__device__ __forceinline__ bool not_finite(bf16_t x) { return (x & 0x7f80) == 0x7f80; }
__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; }

constexpr int PFB = 2;   // steps whose pages are in registers or on their way

// bytes of LDS: the queries' operands and the image of the tree's keys and values; afterwards the states of up to two row tiles
template <int NT, int D, bool F32, int PL>
constexpr size_t attention_lds() {
    constexpr size_t loop = (size_t)NT * 16 * PL * D * Geo<D, F32>::ELEM + (size_t)2 * SLED_TREE_MAX * D * Geo<D, F32>::ELEM;
    constexpr size_t merge = (size_t)(NT < 2 ? NT : 2) * WAVES * Geo<D, F32>::DT * 256 * sizeof(float);
    return loop > merge ? loop : merge;
}

template <int NT, int D, bool F32, bool STEP>
__global__ __launch_bounds__(64 * WAVES, 1) void tree_attention_kernel(tree_args a) {
    using G_ = Geo<D, F32>;
    using T = std::conditional_t<F32, float, bf16_t>;
    constexpr int P = G_::P, TOK = G_::TOK, DT = G_::DT, OWN = G_::OWN, PL = STEP && !F32 ? 2 : 1, ROWS = NT * 16;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    __shared__ float sh_m[WAVES][ROWS], sh_l[WAVES][ROWS];
    __shared__ uint32_t sh_bad[2];
    __shared__ int sh_last;

    const int w = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int32_t* rec = a.t.items + SLED_TREE_ITEM * w;
    const int req = rec[0], g = rec[1], page0 = rec[2], npg = rec[3], n = rec[4], row0 = rec[5], w0 = rec[7], n_items = rec[8], stride = rec[9], r0 = rec[10];
    const bool last = rec[11] != 0;   // the item that has the tree
    const int32_t* pages = a.t.pages + rec[6];
    const int L = a.len_dev[req];
    const int G = a.Hq / a.Hkv, rows = G * n;
    const int n_tiles = min(NT, (rows - r0 + 15) >> 4);
    const int lr = lane & 15, lg = lane >> 4;

    // this wavefront's pages, in steps of P: the item's, as far as there is context
    const int page_end = min(page0 + npg, (L + 15) >> 4);
    const int n_steps_all = page_end > page0 ? (page_end - page0 + P - 1) / P : 0;
    const int n_steps = n_steps_all > wave ? (n_steps_all - wave + WAVES - 1) / WAVES : 0;
    constexpr int BLK = 64 / P;   // steps whose page numbers the lanes hold
    auto page_ids = [&](int it0) {
        const int i = page0 + ((it0 + lane / P) * WAVES + wave) * P + lane % P;
        return pages[min(i, max(page_end - 1, 0))];
    };
    const size_t head = (size_t)16 * D, layer_page = (size_t)a.layer * a.n_pages;
    int ids = 0, ids_next = 0;
    if (n_steps > 0) ids = page_ids(0);
    if (n_steps > BLK) ids_next = page_ids(BLK);
    KV<D, F32> kv[PFB];
    auto issue = [&](KV<D, F32>& dst, int it) {   // called with it = 0, 1, 2, ..
        if (it != 0 && it % BLK == 0) {
            ids = ids_next;
            if (it + BLK < n_steps) ids_next = page_ids(it + BLK);
        }
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int phys = __builtin_amdgcn_readlane(ids, it % BLK * P + p);
            const size_t at = ((layer_page + phys) * a.Hkv + g) * head;
            load_page<D, F32>(dst, p, static_cast<const T*>(a.k_pool) + at, static_cast<const T*>(a.v_pool) + at, lane);
        }
    };
#pragma unroll
    for (int u = 0; u < PFB; u++)
        if (u < n_steps) issue(kv[u], u);

    // queries, and the tree's keys and values, to LDS
    u32x4* qs = reinterpret_cast<u32x4*>(smem);
    T* kt = reinterpret_cast<T*>(smem + (size_t)ROWS * PL * D * G_::ELEM);
    T* vt = kt + (size_t)SLED_TREE_MAX * D;
    if (tid < 2) sh_bad[tid] = 0u;
    stage_queries<D, F32, PL>(qs, a, row0, g, G, r0, n_tiles * 16, rows, tid, 64 * WAVES);
    __syncthreads();
    if (last) {
        constexpr int E = 16 / G_::ELEM, CH = D / E;   // elements of 16 bytes, pieces of a row
        const int filled = (n + TOK - 1) / TOK * TOK;
        for (int e = tid; e < filled * CH; e += 64 * WAVES) {
            const int j = e / CH, d = e % CH * E;
            union {
                uint4 u;
                T x[E];
            } kk, vv;
            kk.u = vv.u = make_uint4(0u, 0u, 0u, 0u);
            if (j < n) {
                kk.u = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.k) + (size_t)(row0 + j) * a.k_stride + g * D + d);
                vv.u = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.v) + (size_t)(row0 + j) * a.v_stride + g * D + d);
                if (r0 == 0) {   // into the request's tail slots
                    const int pos = L + j;
                    const size_t at = ((layer_page + pages[pos >> 4]) * a.Hkv + g) * head;
                    T *kp = static_cast<T*>(a.k_pool) + at, *vp = static_cast<T*>(a.v_pool) + at;
                    if constexpr (F32) {
                        *reinterpret_cast<uint4*>(kp + (pos & 15) * D + d) = kk.u;
                        *reinterpret_cast<uint4*>(vp + (pos & 15) * D + d) = vv.u;
                    } else {
                        *reinterpret_cast<uint4*>(kp + kpage_offset(pos & 15, d)) = kk.u;
#pragma unroll
                        for (int i = 0; i < E; i++) vp[vpage_offset(pos & 15, d + i)] = vv.x[i];
                    }
                }
                bool bad = false;
#pragma unroll
                for (int i = 0; i < E; i++)
                    if (not_finite(vv.x[i])) {
                        bad = true;
                        vv.x[i] = 0;
                    }
                if (bad) atomicOr(&sh_bad[j >> 5], 1u << (j & 31));
            }
            if constexpr (F32) {
                *reinterpret_cast<uint4*>(kt + j * D + d) = kk.u;
                *reinterpret_cast<uint4*>(vt + j * D + d) = vv.u;
            } else {
                *reinterpret_cast<uint4*>(kt + (j >> 4) * head + kpage_offset(j & 15, d)) = kk.u;
#pragma unroll
                for (int i = 0; i < E; i++) vt[(j >> 4) * head + vpage_offset(j & 15, d + i)] = vv.x[i];
            }
        }
        __syncthreads();
    }

    State<NT, DT> st;
#pragma unroll
    for (int t = 0; t < NT; t++) {
        st.m[t] = NEG_BIG;
        st.l[t] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; dt++) st.o[t][dt] = float4_t{0.f, 0.f, 0.f, 0.f};
    }
    uint32_t bits[NT];
    // whole steps, PFB - 1 of them in flight behind the one at work; only the last one of the request's last item may be cut by L
    const int lim = L - (page0 + ((n_steps - 1) * WAVES + wave) * P) * 16;   // context tokens from the last step's first on
    const int n_whole = n_steps > 0 && lim < TOK ? n_steps - 1 : n_steps;
    for (int it0 = 0; it0 < n_whole; it0 += PFB) {
#pragma unroll
        for (int u = 0; u < PFB; u++) {
            const int it = it0 + u;
            if (it < n_whole) {
                tile_steps<NT, D, F32, PL, false>(kv[u], qs, lane, n_tiles, a.scale_log2, bits, st);
                if (it + PFB < n_steps) issue(kv[u], it + PFB);
            }
        }
    }
    if (n_whole < n_steps) {
        KV<D, F32> cut = kv[0];
#pragma unroll
        for (int u = 1; u < PFB; u++)
            if (n_whole % PFB == u) cut = kv[u];
        cut_values<D, F32>(cut, lim, lane);
#pragma unroll
        for (int t = 0; t < NT; t++) bits[t] = (1u << lim) - 1u;   // (lim is at least 1)
        kv[0] = cut;
    }
    // that step, and the tree's: tokens wave * TOK .. of its nodes
    const bool tree = last && wave * TOK < n;
    for (int more = n_whole < n_steps ? 0 : 1; more < (tree ? 2 : 1); more++) {
        if (more == 1) {
#pragma unroll
            for (int p = 0; p < P; p++) load_page<D, F32>(kv[0], p, kt + (wave * P + p) * head, vt + (wave * P + p) * head, lane);
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const int j = (r0 + t * 16 + lr) / G;
                bits[t] = j < n ? (uint32_t)(a.t.seen[row0 + j] >> (wave * TOK)) : 0u;
            }
        }
        tile_steps<NT, D, F32, PL, true>(kv[0], qs, lane, n_tiles, a.scale_log2, bits, st);
    }
    __syncthreads();   // nobody reads the queries or the image any more

    // The wavefronts' states, added up in ascending order: wavefront w takes over the dims of tiles w * OWN ..
    float4_t own[NT][OWN];
    float m[NT], lsum[NT];
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const float l = sum_over_groups(st.l[t]);
        if (lg == 0) {
            sh_m[wave][t * 16 + lr] = st.m[t];
            sh_l[wave][t * 16 + lr] = l;
        }
    }
    constexpr int TB = NT < 2 ? NT : 2;
    float* park = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int tb = 0; tb < NT; tb += TB) {
        if (tb) __syncthreads();
#pragma unroll
        for (int u = 0; u < TB; u++)
#pragma unroll
            for (int dt = 0; dt < DT; dt++)
                *reinterpret_cast<float4_t*>(park + (((u * WAVES + wave) * DT + dt) * 64 + lane) * 4) = st.o[tb + u][dt];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < TB; u++) {
            const int t = tb + u;
            float f[WAVES];
            m[t] = NEG_BIG;
#pragma unroll
            for (int v = 0; v < WAVES; v++) m[t] = fmaxf(m[t], sh_m[v][t * 16 + lr]);
            lsum[t] = 0.f;
#pragma unroll
            for (int v = 0; v < WAVES; v++) {
                f[v] = exp2f(sh_m[v][t * 16 + lr] - m[t]);
                lsum[t] += sh_l[v][t * 16 + lr] * f[v];
            }
#pragma unroll
            for (int i = 0; i < OWN; i++) {
                own[t][i] = float4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int v = 0; v < WAVES; v++) {
                    const float4_t x = *reinterpret_cast<const float4_t*>(park + (((u * WAVES + v) * DT + wave * OWN + i) * 64 + lane) * 4);
#pragma unroll
                    for (int e = 0; e < 4; e++) own[t][i][e] += x[e] * f[v];
                }
            }
        }
    }

    uint32_t bad[2] = {sh_bad[0], sh_bad[1]};
    if (n_items > 1) {
        // Handing over without a device-wide fence: states are stored and read with device-scope accesses, and the counter is raised only
        // when this workgroup's stores have been acknowledged.
        float* po = a.t.part_o + (size_t)w * (NT * DT * 256) + (wave * OWN) * 256 + lane;
        float* pm = a.t.part_ml + (size_t)w * (2 * ROWS);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            if (wave == 0 && lg == 0) {
                __hip_atomic_store(pm + t * 16 + lr, m[t], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(pm + ROWS + t * 16 + lr, lsum[t], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            if (t >= n_tiles) continue;
#pragma unroll
            for (int i = 0; i < OWN; i++)
#pragma unroll
                for (int e = 0; e < 4; e++)
                    __hip_atomic_store(po + (t * DT + i) * 256 + e * 64, own[t][i][e], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        uint32_t* arrive = reinterpret_cast<uint32_t*>(a.t.arrive + 4 * w0);   // counter, -, the two words of `bad`
        if (last && tid < 2) __hip_atomic_store(arrive + 2 + tid, bad[tid & 1], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (tid == 0) {
            const uint32_t old = __hip_atomic_fetch_add(arrive, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            sh_last = old == (uint32_t)n_items - 1;
            if (sh_last) __hip_atomic_store(arrive, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // for the next layer
        }
        __syncthreads();
        if (!sh_last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        bad[0] = __hip_atomic_load(arrive + 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        bad[1] = __hip_atomic_load(arrive + 3, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int t = 0; t < NT; t++) {
            m[t] = NEG_BIG;
            lsum[t] = 0.f;
#pragma unroll
            for (int i = 0; i < OWN; i++) own[t][i] = float4_t{0.f, 0.f, 0.f, 0.f};
        }
        for (int c = 0; c < n_items; c++) {   // in ascending order, whichever came last
            const int wc = w0 + c * stride;
            const float* qo = a.t.part_o + (size_t)wc * (NT * DT * 256) + (wave * OWN) * 256 + lane;
            const float* qm = a.t.part_ml + (size_t)wc * (2 * ROWS);
            float im[NT], il[NT], io[NT][OWN][4];
#pragma unroll
            for (int t = 0; t < NT; t++) {
                im[t] = __hip_atomic_load(qm + t * 16 + lr, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                il[t] = __hip_atomic_load(qm + ROWS + t * 16 + lr, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (int i = 0; i < OWN; i++)
#pragma unroll
                    for (int e = 0; e < 4; e++)
                        io[t][i][e] = __hip_atomic_load(qo + (min(t, n_tiles - 1) * DT + i) * 256 + e * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
#pragma unroll
            for (int t = 0; t < NT; t++) {
                const float mnew = fmaxf(m[t], im[t]), fo = exp2f(m[t] - mnew), fi = exp2f(im[t] - mnew);
                m[t] = mnew;
                lsum[t] = lsum[t] * fo + il[t] * fi;
#pragma unroll
                for (int i = 0; i < OWN; i++)
#pragma unroll
                    for (int e = 0; e < 4; e++) own[t][i][e] = own[t][i][e] * fo + io[t][i][e] * fi;
            }
        }
    }

    // the output: row lr of tile t, dims (wave * OWN + i) * 16 + lg * 4 ..
#pragma unroll
    for (int t = 0; t < NT; t++) {
        const int r = r0 + t * 16 + lr;
        if (r >= rows) continue;
        const int j = r / G, h = g * G + r - j * G;
        const float inv = 1.0f / lsum[t];
        if (a.lse && wave == 0 && lg == 0) a.lse[(size_t)(row0 + j) * a.Hq + h] = (m[t] + log2f(lsum[t])) * 0.6931471805599453f;
        const uint64_t poison = (bad[0] | bad[1]) ? a.t.seen[row0 + j] & (((uint64_t)bad[1] << 32) | bad[0]) : 0ull;
#pragma unroll
        for (int i = 0; i < OWN; i++) {
            const int d = (wave * OWN + i) * 16 + lg * 4;
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; e++) y[e] = own[t][i][e] * inv;
            for (uint64_t left = poison; left; left &= left - 1) {   // values that are not finite, of nodes that this row sees
                const T* vp = static_cast<const T*>(a.v) + (size_t)(row0 + __builtin_ctzll(left)) * a.v_stride + g * D + d;
#pragma unroll
                for (int e = 0; e < 4; e++)
                    if (not_finite(vp[e])) {
                        if constexpr (F32) y[e] += vp[e];
                        else y[e] += bf16_to_f32(vp[e]);
                    }
            }
            if constexpr (F32) {
                *reinterpret_cast<float4*>(static_cast<float*>(a.out) + ((size_t)(row0 + j) * a.Hq + h) * D + d) = make_float4(y[0], y[1], y[2], y[3]);
            } else if constexpr (STEP) {
                bf16_t* x = static_cast<bf16_t*>(a.out) + frag_offset(row0 + j, h * D + d, a.Hq * D);
                uint32_t hi[2], lo[2];
#pragma unroll
                for (int e = 0; e < 2; e++) {
                    const bf16_t h0 = f32_to_bf16(y[2 * e]), h1 = f32_to_bf16(y[2 * e + 1]);
                    hi[e] = (uint32_t)h0 | ((uint32_t)h1 << 16);
                    lo[e] = (uint32_t)f32_to_bf16(y[2 * e] - bf16_to_f32(h0)) | ((uint32_t)f32_to_bf16(y[2 * e + 1] - bf16_to_f32(h1)) << 16);
                }
                *reinterpret_cast<uint2*>(x) = make_uint2(hi[0], hi[1]);
                *reinterpret_cast<uint2*>(x + a.x_plane) = make_uint2(lo[0], lo[1]);
            } else {
                // the conversion in hardware: to nearest even, infinities and NaN kept
                union {
                    __bf16 b[4];
                    uint2 u;
                } z;
#pragma unroll
                for (int e = 0; e < 4; e++) z.b[e] = (__bf16)y[e];
                *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + ((size_t)(row0 + j) * a.Hq + h) * D + d) = z.u;
            }
        }
    }
}

// mass[token] += sum over the rows of a block and the G heads of a kv head of exp(s - lse), one more pass over K.
// S = Q K^T with the tokens on the lanes (A operand Q, B operand K), so that a lane adds up its token's weights over all rows in one
// register and nothing but the last sum crosses lanes.  A wavefront holds MP pages of K in registers and walks through
// the row tiles, whose operands all wavefronts of the workgroup share in LDS.  A token's sum is made by one
// lane group in a fixed order: no atomics, and the same result every time.
constexpr int MASS_WAVES = 8;
template <bool F32>
__host__ __device__ constexpr int mass_pages() { return F32 ? 2 : 4; }   // pages of a wavefront at a time
__host__ __device__ constexpr int mass_rows(int PL) { return PL == 1 ? 256 : 128; }   // rows in LDS at a time

struct mass_args {
    float* mass;   // [request][layer][kv head][cap]
    int cap, n_layers;
};

template <int D, bool F32, int PL>
__global__ __launch_bounds__(64 * MASS_WAVES) void tree_mass_kernel(tree_args a, mass_args ma) {
    constexpr int MP = mass_pages<F32>(), QT = Geo<D, F32>::QC * 64 * PL, MR = mass_rows(PL);
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int32_t* rec = a.t.mass_items + 8 * blockIdx.x;
    const int req = rec[0], g = rec[1], page0 = rec[2], npg = rec[3], n = rec[4], row0 = rec[5];
    const int32_t* pages = a.t.pages + rec[6];
    const int L = a.len_dev[req], G = a.Hq / a.Hkv, rows = G * n;
    const int page_end = min(page0 + npg, (L + n + 15) >> 4);
    if (page0 >= page_end) return;
    const int lr = lane & 15, lg = lane >> 4;
    u32x4* qs = reinterpret_cast<u32x4*>(smem);
    const int room = min(MR, (rows + 15) & ~15);
    float* lse2 = reinterpret_cast<float*>(smem + (size_t)room * PL * D * Geo<D, F32>::ELEM);   // log2 of a row's denominator
    uint64_t* seen = reinterpret_cast<uint64_t*>(lse2 + room);
    const size_t head = (size_t)16 * D, layer_page = (size_t)a.layer * a.n_pages;
    using T = std::conditional_t<F32, float, bf16_t>;
    for (int r0 = 0; r0 < rows; r0 += MR) {
        const int n_rows = min(MR, (rows - r0 + 15) & ~15);
        if (r0) __syncthreads();
        stage_queries<D, F32, PL>(qs, a, row0, g, G, r0, n_rows, rows, tid, 64 * MASS_WAVES);
        for (int r = tid; r < n_rows; r += 64 * MASS_WAVES) {
            const int j = (r0 + r) / G, h = g * G + (r0 + r) - j * G;
            // a row that does not exist has an infinite denominator: its weights are zero
            lse2[r] = r0 + r < rows ? a.lse[(size_t)(row0 + j) * a.Hq + h] * 1.4426950408889634f : INFINITY;
            seen[r] = r0 + r < rows ? a.t.seen[row0 + j] : 0ull;
        }
        __syncthreads();
        for (int p0 = page0 + wave * MP; p0 < page_end; p0 += MASS_WAVES * MP) {
            KV<D, F32> kv[MP];   // (the values are never loaded)
#pragma unroll
            for (int p = 0; p < MP; p++) {
                const int phys = pages[min(p0 + p, page_end - 1)];
                const T* kp = static_cast<const T*>(a.k_pool) + ((layer_page + phys) * a.Hkv + g) * head;
                if constexpr (!F32) {
#pragma unroll
                    for (int c = 0; c < 4; c++) kv[p].k[0][c] = reinterpret_cast<const u32x4*>(kp)[c * 64 + lane];
                } else {
#pragma unroll
                    for (int c = 0; c < D / 16; c++) kv[p].k[c] = *reinterpret_cast<const f32x4*>(kp + lr * D + lg * 4 + 16 * c);
                }
            }
            float acc[MP];
#pragma unroll
            for (int p = 0; p < MP; p++) acc[p] = 0.f;
            auto walk = [&](auto masked) {
                for (int t = 0; t < n_rows / 16; t++) {
                    const float4 z = *reinterpret_cast<const float4*>(lse2 + t * 16 + lg * 4);   // of the rows this lane has
                    const float zz[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
                    for (int p = 0; p < MP; p++) {
                        const float4_t s = page_scores<D, F32, PL, true>(kv[p], 0, qs + t * QT + lane);
                        float x = 0.f;
#pragma unroll
                        for (int i = 0; i < 4; i++) {
                            float e = __builtin_amdgcn_exp2f(fmaf(s[i], a.scale_log2, -zz[i]));
                            if (decltype(masked)::value) {
                                const int c = (p0 + p) * 16 + lr - L;   // node of this lane's token, if not context
                                const bool on = c < 0 || (c < n && ((seen[t * 16 + lg * 4 + i] >> (c & 63)) & 1ull));
                                e = on ? e : 0.f;
                            }
                            x += e;
                        }
                        acc[p] += x;
                    }
                }
            };
            if ((p0 + MP) * 16 > L) walk(std::true_type{});
            else walk(std::false_type{});
            float* row = ma.mass + (((size_t)req * ma.n_layers + a.layer) * a.Hkv + g) * ma.cap;
#pragma unroll
            for (int p = 0; p < MP; p++) {
                const float x = sum_over_groups(acc[p]);
                const int pos = (p0 + p) * 16 + lr;
                if (lg == 0 && p0 + p < page_end && pos < L + n) {
                    // a node's slot holds no mass of its own yet, but perhaps that of a node that was not accepted
                    if (pos < L || r0) row[pos] += x;
                    else row[pos] = x;
                }
            }
        }
    }
}

// The QKV projection's K slices of row t, added up and rotated: q as a bf16 pair (fp32 models: as it is), k and v in the model's type, all as
// plain rows.  A thread takes four neighbouring rotary pairs of a q or k head or four dims of a v head.
template <bool F32>
__global__ __launch_bounds__(256) void tree_qkv_kernel(const float* __restrict__ partial, int n_split, int T_pad, int Hq, int Hkv, int D, const float2* __restrict__ cs,
                                                       void* __restrict__ Q, size_t q_plane, void* __restrict__ K, void* __restrict__ V) {
    const int t = blockIdx.x, half = D / 2, per_head = half / 4, n_rot = (Hq + Hkv) * per_head, n_qkv = (Hq + 2 * Hkv) * D;
    const int item = blockIdx.y * 256 + threadIdx.x;
    const float* row = partial + (size_t)t * n_qkv;
    const size_t slice = (size_t)T_pad * n_qkv;
    auto add = [&](int col) {
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int s0 = 0; s0 < n_split; s0 += 4) {   // four slices in flight, added in ascending order
            float4 y[4];
#pragma unroll
            for (int s = 0; s < 4; s++) y[s] = s0 + s < n_split ? *reinterpret_cast<const float4*>(row + (s0 + s) * slice + col) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int s = 0; s < 4; s++) {
                x.x += y[s].x;
                x.y += y[s].y;
                x.z += y[s].z;
                x.w += y[s].w;
            }
        }
        return x;
    };
    auto pack = [](const float* y) {
        return make_uint2((uint32_t)f32_to_bf16(y[0]) | ((uint32_t)f32_to_bf16(y[1]) << 16), (uint32_t)f32_to_bf16(y[2]) | ((uint32_t)f32_to_bf16(y[3]) << 16));
    };
    auto put = [&](void* base, size_t at, const float* y) {
        if (F32) *reinterpret_cast<float4*>(static_cast<float*>(base) + at) = make_float4(y[0], y[1], y[2], y[3]);
        else *reinterpret_cast<uint2*>(static_cast<bf16_t*>(base) + at) = pack(y);
    };
    if (item < n_rot) {
        const int h = item / per_head, i = item % per_head * 4;
        const float4 c01 = *reinterpret_cast<const float4*>(cs + (size_t)t * half + i), c23 = *reinterpret_cast<const float4*>(cs + (size_t)t * half + i + 2);
        const float4 x1 = add(h * D + i), x2 = add(h * D + i + half);
        float y1[4], y2[4];
        rope_pair(x1.x, x2.x, c01.x, c01.y, y1[0], y2[0]);
        rope_pair(x1.y, x2.y, c01.z, c01.w, y1[1], y2[1]);
        rope_pair(x1.z, x2.z, c23.x, c23.y, y1[2], y2[2]);
        rope_pair(x1.w, x2.w, c23.z, c23.w, y1[3], y2[3]);
        const bool q = h < Hq;
        void* base = q ? Q : K;
        const size_t at = q ? ((size_t)t * Hq + h) * D + i : ((size_t)t * Hkv + h - Hq) * D + i;
        put(base, at, y1);
        put(base, at + half, y2);
        if (!F32 && q) {
            float l1[4], l2[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                l1[e] = y1[e] - bf16_to_f32(f32_to_bf16(y1[e]));
                l2[e] = y2[e] - bf16_to_f32(f32_to_bf16(y2[e]));
            }
            put(base, at + q_plane, l1);
            put(base, at + q_plane + half, l2);
        }
    } else if (item < n_rot + Hkv * (D / 4)) {
        const int e = item - n_rot;
        const float4 x = add((Hq + Hkv) * D + 4 * e);
        const float y[4] = {x.x, x.y, x.z, x.w};
        put(V, (size_t)t * Hkv * D + 4 * e, y);
    }
}

template <int NT, int D, bool F32, bool STEP>
int launch_attention(const tree_args& a, hipStream_t st) {
    constexpr size_t lds = attention_lds<NT, D, F32, (STEP && !F32 ? 2 : 1)>();
    static_assert(lds <= 150 * 1024, "LDS of a workgroup");
    static bool allowed = false;
    if (!allowed) {
        SLED_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(tree_attention_kernel<NT, D, F32, STEP>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        allowed = true;
    }
    hipLaunchKernelGGL((tree_attention_kernel<NT, D, F32, STEP>), dim3(a.t.n_items), dim3(64 * WAVES), lds, st, a);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}

template <int D, bool F32, bool STEP>
int launch_attention_tiles(const tree_args& a, hipStream_t st) {
    switch (a.t.tiles) {
        case 1: return launch_attention<1, D, F32, STEP>(a, st);
        case 2: return launch_attention<2, D, F32, STEP>(a, st);
        default: return launch_attention<4, D, F32, STEP>(a, st);
    }
}

template <int D, bool F32, int PL>
int launch_mass(const tree_args& a, const mass_args& ma, int max_rows, hipStream_t st) {
    const int room = std::min(mass_rows(PL), (max_rows + 15) & ~15);
    const size_t lds = (size_t)room * (PL * D * Geo<D, F32>::ELEM + sizeof(float) + sizeof(uint64_t));
    static size_t allowed = 0;
    if (lds > allowed) {
        SLED_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(tree_mass_kernel<D, F32, PL>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
        allowed = lds;
    }
    hipLaunchKernelGGL((tree_mass_kernel<D, F32, PL>), dim3(a.t.n_mass_items), dim3(64 * MASS_WAVES), lds, st, a, ma);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}

tree_args common_args(const sled_model* m, const sled_kvpool* p, const sled_tree_plan& t, int layer, const void* q, size_t q_stride, size_t q_plane) {
    tree_args a{};
    a.t = t;
    a.len_dev = p->len_dev;
    a.q = q;
    a.q_stride = q_stride;
    a.q_plane = q_plane;
    a.k_pool = p->k_pool;
    a.v_pool = p->v_pool;
    a.n_pages = p->n_pages;
    a.layer = layer;
    a.Hq = m->s.n_q_heads;
    a.Hkv = m->s.n_kv_heads;
    a.scale_log2 = 1.4426950408889634f / sqrtf((float)m->s.head_dim);
    return a;
}

}  // namespace

int sled_launch_tree_attention(const sled_model* m, const sled_kvpool* p, const sled_tree_plan& t, int layer, const void* q, size_t q_stride, size_t q_plane,
                               const void* k, size_t k_stride, const void* v, size_t v_stride, void* out, size_t x_plane, float* lse, bool step, hipStream_t st) {
    tree_args a = common_args(m, p, t, layer, q, q_stride, q_plane);
    a.k = k;
    a.v = v;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.out = out;
    a.x_plane = x_plane;
    a.lse = lse;
    if (m->s.dtype == SLED_BF16) return step ? launch_attention_tiles<128, false, true>(a, st) : launch_attention_tiles<128, false, false>(a, st);
    return m->s.head_dim == 64 ? launch_attention_tiles<64, true, false>(a, st) : launch_attention_tiles<128, true, false>(a, st);
}

int sled_launch_tree_mass(const sled_model* m, const sled_kvpool* p, const sled_tree_plan& t, int layer, const void* q, size_t q_stride, size_t q_plane,
                          const float* lse, float* mass, int cap, hipStream_t st) {
    tree_args a = common_args(m, p, t, layer, q, q_stride, q_plane);
    a.lse = const_cast<float*>(lse);
    const mass_args ma{mass, cap, m->s.n_layers};
    const int rows = t.max_nodes * (m->s.n_q_heads / m->s.n_kv_heads);
    if (m->s.dtype == SLED_BF16) return q_plane ? launch_mass<128, false, 2>(a, ma, rows, st) : launch_mass<128, false, 1>(a, ma, rows, st);
    return m->s.head_dim == 64 ? launch_mass<64, true, 1>(a, ma, rows, st) : launch_mass<128, true, 1>(a, ma, rows, st);
}

int sled_launch_tree_qkv(const sled_model* m, int T, const float* partial, int n_split, int T_pad, const float* cs, void* Q, size_t q_plane, void* K, void* V,
                         hipStream_t st) {
    const int Hq = m->s.n_q_heads, Hkv = m->s.n_kv_heads, D = m->s.head_dim;
    const dim3 grid(T, ((Hq + Hkv) * (D / 8) + Hkv * (D / 4) + 255) / 256);
    if (m->s.dtype == SLED_BF16)
        hipLaunchKernelGGL(tree_qkv_kernel<false>, grid, dim3(256), 0, st, partial, n_split, T_pad, Hq, Hkv, D, reinterpret_cast<const float2*>(cs), Q, q_plane, K, V);
    else
        hipLaunchKernelGGL(tree_qkv_kernel<true>, grid, dim3(256), 0, st, partial, n_split, T_pad, Hq, Hkv, D, reinterpret_cast<const float2*>(cs), Q, q_plane, K, V);
    SLED_LAUNCH_CHECK();
    return SLED_OK;
}
