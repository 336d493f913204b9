// Lists of tensors next to the flat vectors of the code: norms, clipping, packing into a row of G, updates from a decoded sum.
//
//   N = sqrt(sum_t sum_i g_t[i]^2)  or  max_t,i |g_t[i]|        c = max_norm / N if N > max_norm, else 1
//   clip: g_t <- c g_t       pack: row[off_t + i] = c g_t[i]       update: w_t[i] <- w_t[i] - scale c u[off_t + i],  N = |u|
//
// All of them stream the list once or twice and are bound by HBM; short ones by the latency of one or two launches.
//
// Split.  A list is cut into items of 4 KB (of the tensor's own type), which start on 16-byte boundaries of the tensor's memory, wherever
// the tensor starts, and the items are dealt to the warps of the grid in contiguous ranges of equal length, so that a tensor of any size costs
// what it holds.  The ranges depend on sizes alone and are made once, with the layout; the tensors' addresses come with every call, as
// kernel parameters (a graph captures them, nothing is uploaded), at most kMaxPointers a launch; longer lists take several launches.
// No warp waits for another: block sums are written out and added up, in a fixed order, by whoever needs the norm next.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <stdlib.h>
#include <string.h>

#include <new>
#include <type_traits>

#include "draco_internal.cuh"

namespace draco {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kBlocksPerSm = 4;
constexpr int kItemBytes = 4096;
constexpr int kUnroll = kItemBytes / (32 * 16);   // 16-byte loads per lane and item
constexpr int kMaxPointers = 2000;                // two lists of 8-byte pointers within the 32,764 bytes of kernel parameters

struct TensorInfo {
    int64_t numel;
    int64_t flat;          // offset in the flat vector
    int64_t items;         // 4 KB items, wherever in a 16-byte word the tensor starts
    int32_t type;
    int32_t seg_first;     // partial sums of this tensor alone: one for each warp that has items of it
    int32_t seg_count;
    int32_t pad;
};

struct WarpStart {         // where a warp's items begin; the next entry says where they end
    int64_t item;          // within the tensor
    int64_t index;         // within the launch
    int32_t tensor;
    int32_t pad;
};

struct Part {              // the tensors of one launch
    int first, count;
    int blocks;
    int block0;            // of the partial sums
    int64_t starts;        // into the table of WarpStart
};

template <int N>
struct Pointers {
    void* p[N];
};

__host__ __device__ constexpr int size_of(int type) { return type == DRACO_F32 ? 4 : 2; }

// ---- elements ----

template <int TYPE>
struct Elements;

template <>
struct Elements<DRACO_F32> {
    typedef float type;
    static __device__ float value(float x) { return x; }
    static __device__ float round(float x) { return x; }
};
template <>
struct Elements<DRACO_BF16> {
    typedef __nv_bfloat16 type;
    static __device__ float value(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __nv_bfloat16 round(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct Elements<DRACO_F16> {
    typedef __half type;
    static __device__ float value(__half x) { return __half2float(x); }
    static __device__ __half round(float x) { return __float2half_rn(x); }
};

template <int TYPE, int N>
struct alignas(N * size_of(TYPE)) Vec {
    typename Elements<TYPE>::type e[N];
};

// ---- sums of squares and largest magnitudes, in 64-bit slots ----

// Sums are kept in fp64: products of fp32 values are exact there and neither overflow nor vanish.  Squares of a 16-byte word of 16-bit
// values are added in fp32 first (they have 22 bits at most; eight of them are good to 2^-22) and in fp64 where that sum leaves the
// range in which fp32 loses nothing that counts: one conversion a word instead of eight.
struct SumSquares {
    typedef double Slot;
    static __device__ Slot zero() { return 0.0; }
    static __device__ void add(Slot& a, Slot b) { a += b; }
    template <int TYPE>
    static __device__ void one(Slot& a, typename Elements<TYPE>::type x) {
        const double v = (double)Elements<TYPE>::value(x);
        a = fma(v, v, a);
    }
    template <int TYPE, int N>
    static __device__ void word(Slot& a, const Vec<TYPE, N>& v) {
        if (TYPE == DRACO_F32) {
#pragma unroll
            for (int i = 0; i < N; ++i) one<TYPE>(a, v.e[i]);
        } else {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float x = Elements<TYPE>::value(v.e[i]);
                s = fmaf(x, x, s);
            }
            if (TYPE == DRACO_F16 || (s >= 0x1p-100f && s <= 0x1p120f)) {
                a += (double)s;
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) one<TYPE>(a, v.e[i]);
            }
        }
    }
    static __device__ double norm(Slot a) { return sqrt(a); }
};

// Magnitudes compare like their bit patterns, infinity above all numbers and NaN above infinity.
struct MaxMagnitude {
    typedef unsigned long long Slot;
    static __device__ Slot zero() { return 0; }
    static __device__ void add(Slot& a, Slot b) { a = a > b ? a : b; }
    template <int TYPE>
    static __device__ void one(Slot& a, typename Elements<TYPE>::type x) {
        const unsigned b = __float_as_uint(Elements<TYPE>::value(x)) & 0x7fffffffu;
        a = max((unsigned)a, b);
    }
    template <int TYPE, int N>
    static __device__ void word(Slot& a, const Vec<TYPE, N>& v) {
#pragma unroll
        for (int i = 0; i < N; ++i) one<TYPE>(a, v.e[i]);
    }
    static __device__ double norm(Slot a) { return (double)__uint_as_float((unsigned)a); }
};

template <class K>
__device__ typename K::Slot warp_total(typename K::Slot a) {
#pragma unroll
    for (int m = 16; m; m >>= 1) K::add(a, __shfl_xor_sync(0xffffffffu, a, m));
    return a;
}

// In every thread of the block.
template <class K>
__device__ typename K::Slot block_total(typename K::Slot a, typename K::Slot* shared /*[kWarps]*/) {
    a = warp_total<K>(a);
    if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = a;
    __syncthreads();
    a = shared[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) K::add(a, shared[w]);
    __syncthreads();
    return a;
}

template <class K>
__device__ typename K::Slot total_of(const void* slots, int64_t first, int64_t count, typename K::Slot* shared) {
    const typename K::Slot* s = static_cast<const typename K::Slot*>(slots) + first;
    typename K::Slot a = K::zero();
    for (int64_t i = threadIdx.x; i < count; i += kThreads) K::add(a, s[i]);
    return block_total<K>(a, shared);
}

struct Limit {
    const void* slots;     // block sums, or null: no norm is wanted
    int count;
    int kind;
    float max_norm;
    float* norm;           // may be null
};

struct Factor {
    float c;
    bool finite;
};

__device__ Factor factor_of(double norm, float max_norm) {
    Factor f;
    f.finite = isfinite((float)norm);
    f.c = f.finite && norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
    return f;
}

// The block sums added up and the factor they give, in every thread; the first block writes the norm down.
__device__ Factor block_factor(const Limit& l) {
    __shared__ unsigned long long shared[kWarps];
    if (!l.slots) return Factor{1.0f, true};
    const double n = l.kind == DRACO_NORM_2 ? SumSquares::norm(total_of<SumSquares>(l.slots, 0, l.count, reinterpret_cast<double*>(shared)))
                                            : MaxMagnitude::norm(total_of<MaxMagnitude>(l.slots, 0, l.count, shared));
    if (l.norm && blockIdx.x == 0 && threadIdx.x == 0) *l.norm = (float)n;
    return factor_of(n, l.max_norm);
}

// ---- the walk over a warp's items ----

// f(tensor, info, first item, items) for every tensor that the warp has items of.
template <class F>
__device__ void walk(const TensorInfo* __restrict__ infos, const WarpStart* __restrict__ starts, F f) {
    const int w = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const WarpStart s = starts[w];
    int64_t left = starts[w + 1].index - s.index, item = s.item;
    for (int t = s.tensor; left > 0; ++t, item = 0) {
        const TensorInfo& info = infos[t];
        const int64_t take = min(left, info.items - item);
        if (take > 0) f(t, info, item, take);
        left -= max(take, (int64_t)0);
    }
}

template <class F>
__device__ void by_type(int type, F f) {
    if (type == DRACO_F32) f(std::integral_constant<int, DRACO_F32>());
    else if (type == DRACO_BF16) f(std::integral_constant<int, DRACO_BF16>());
    else f(std::integral_constant<int, DRACO_F16>());
}

template <class K, int TYPE>
__device__ void measure_items(const void* base, int64_t numel, int64_t item, int64_t take, typename K::Slot& acc) {
    constexpr int kVec = 16 / size_of(TYPE), kItem = kItemBytes / size_of(TYPE);
    typedef typename Elements<TYPE>::type T;
    const int lane = threadIdx.x & 31;
    const int shift = (int)((reinterpret_cast<uintptr_t>(base) & 15u) / size_of(TYPE));
    const T* p = static_cast<const T*>(base);
    for (int64_t lo = item * kItem - shift; take > 0; --take, lo += kItem) {
        if (lo >= 0 && lo + kItem <= numel) {
            const Vec<TYPE, kVec>* v = reinterpret_cast<const Vec<TYPE, kVec>*>(p + lo) + lane;
            Vec<TYPE, kVec> x[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) x[u] = v[u * 32];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) K::template word<TYPE, kVec>(acc, x[u]);
        } else {
            for (int u = 0; u < kUnroll; ++u) {
                const int64_t e = lo + (u * 32 + lane) * kVec;
                if (e >= 0 && e + kVec <= numel) {
                    K::template word<TYPE, kVec>(acc, *reinterpret_cast<const Vec<TYPE, kVec>*>(p + e));
                } else {
                    for (int i = 0; i < kVec; ++i)
                        if (e + i >= 0 && e + i < numel) K::template one<TYPE>(acc, p[e + i]);
                }
            }
        }
    }
}

// Block sums to slots[blockIdx.x]; SEGMENTS: the sums of each warp's part of each tensor to segments[warp + tensor], a place of its
// own for every such pair since both only ever grow along the list.  norm: written by the block that finishes last.
template <class K, int N, bool SEGMENTS>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
measure_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const WarpStart* __restrict__ starts,
               typename K::Slot* slots, int block0, typename K::Slot* segments, float* norm, int all_blocks, unsigned* ticket) {
    pdl_begin();
    __shared__ typename K::Slot shared[kWarps];
    __shared__ bool last;
    typename K::Slot acc = K::zero();
    const int w = blockIdx.x * kWarps + (threadIdx.x >> 5);
    walk(infos, starts, [&](int t, const TensorInfo& info, int64_t item, int64_t take) {
        typename K::Slot a = K::zero();
        if (list.p[t])
            by_type(info.type, [&](auto type) { measure_items<K, decltype(type)::value>(list.p[t], info.numel, item, take, SEGMENTS ? a : acc); });
        if (SEGMENTS) {
            a = warp_total<K>(a);
            if ((threadIdx.x & 31) == 0) {
                segments[w + t] = a;
                K::add(acc, a);
            }
        }
    });
    acc = block_total<K>(acc, shared);
    if (threadIdx.x == 0) {
        slots[block0 + blockIdx.x] = acc;
        if (norm) {
            __threadfence();
            last = atomicInc(ticket, all_blocks - 1) == all_blocks - 1;     // back at zero after the last
            __threadfence();
        }
    }
    if (!norm) return;
    __syncthreads();
    if (!last) return;
    typename K::Slot a = K::zero();
    for (int i = threadIdx.x; i < all_blocks; i += kThreads) K::add(a, __ldcg(slots + i));
    a = block_total<K>(a, shared);
    if (threadIdx.x == 0) *norm = (float)K::norm(a);
}

// One block a tensor: its segments added up, its norm and factor; one block more: the norm of all.
template <class K>
__global__ void __launch_bounds__(kThreads)
each_kernel(const TensorInfo* __restrict__ infos, int count, const typename K::Slot* segments, const typename K::Slot* slots, int all_blocks,
            float max_norm, float* norm, float* each, float* factors) {
    pdl_begin();
    __shared__ typename K::Slot shared[kWarps];
    if (blockIdx.x == count) {
        const double n = K::norm(total_of<K>(slots, 0, all_blocks, shared));
        if (norm && threadIdx.x == 0) *norm = (float)n;
        return;
    }
    const TensorInfo& info = infos[blockIdx.x];
    const double n = K::norm(total_of<K>(segments, info.seg_first, info.seg_count, shared));
    if (threadIdx.x == 0) {
        if (each) each[blockIdx.x] = (float)n;
        if (factors) factors[blockIdx.x] = factor_of(n, max_norm).c;
    }
}

template <int TYPE>
__device__ typename Elements<TYPE>::type scaled(typename Elements<TYPE>::type x, float c) {
    return Elements<TYPE>::round(Elements<TYPE>::value(x) * c);
}

template <int TYPE>
__device__ void scale_items(const void* from, void* to, int64_t numel, int64_t item, int64_t take, float c) {
    constexpr int kVec = 16 / size_of(TYPE), kItem = kItemBytes / size_of(TYPE);
    typedef typename Elements<TYPE>::type T;
    const int lane = threadIdx.x & 31;
    const int shift = (int)((reinterpret_cast<uintptr_t>(from) & 15u) / size_of(TYPE));
    const bool together = ((reinterpret_cast<uintptr_t>(from) ^ reinterpret_cast<uintptr_t>(to)) & 15u) == 0;
    const T* p = static_cast<const T*>(from);
    T* q = static_cast<T*>(to);
    for (int64_t lo = item * kItem - shift; take > 0; --take, lo += kItem) {
        if (together && lo >= 0 && lo + kItem <= numel) {
            const Vec<TYPE, kVec>* v = reinterpret_cast<const Vec<TYPE, kVec>*>(p + lo) + lane;
            Vec<TYPE, kVec>* o = reinterpret_cast<Vec<TYPE, kVec>*>(q + lo) + lane;
            Vec<TYPE, kVec> x[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) x[u] = v[u * 32];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) x[u].e[i] = scaled<TYPE>(x[u].e[i], c);
                o[u * 32] = x[u];
            }
        } else {
            for (int64_t e = max(lo, (int64_t)0) + lane; e < min(lo + kItem, numel); e += 32) q[e] = scaled<TYPE>(p[e], c);
        }
    }
}

// to = from * c.  In place nothing is written where c is 1.
template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
scale_kernel(const __grid_constant__ Pointers<N> from, const __grid_constant__ Pointers<N> to, const TensorInfo* __restrict__ infos,
             const WarpStart* __restrict__ starts, Limit limit, const float* factors) {
    pdl_begin();
    const float all = factors ? 1.0f : block_factor(limit).c;
    walk(infos, starts, [&](int t, const TensorInfo& info, int64_t item, int64_t take) {
        const float c = factors ? factors[t] : all;
        if (!from.p[t] || (c == 1.0f && from.p[t] == to.p[t])) return;
        by_type(info.type, [&](auto type) { scale_items<decltype(type)::value>(from.p[t], to.p[t], info.numel, item, take, c); });
    });
}

// ---- a tensor beside its part of a flat fp32 vector: four elements a lane ----

template <int TYPE>
__device__ float4 load4(const typename Elements<TYPE>::type* p, bool aligned) {
    Vec<TYPE, 4> v;
    if (aligned) {
        v = *reinterpret_cast<const Vec<TYPE, 4>*>(p);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v.e[i] = p[i];
    }
    return make_float4(Elements<TYPE>::value(v.e[0]), Elements<TYPE>::value(v.e[1]), Elements<TYPE>::value(v.e[2]), Elements<TYPE>::value(v.e[3]));
}

template <int TYPE>
__device__ void store4(typename Elements<TYPE>::type* p, float4 x, bool aligned) {
    Vec<TYPE, 4> v;
    v.e[0] = Elements<TYPE>::round(x.x);
    v.e[1] = Elements<TYPE>::round(x.y);
    v.e[2] = Elements<TYPE>::round(x.z);
    v.e[3] = Elements<TYPE>::round(x.w);
    if (aligned) {
        *reinterpret_cast<Vec<TYPE, 4>*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = v.e[i];
    }
}

// whole(e): elements e .. e + 3; single(e): one element, at the tensor's ends.  Items start `shift` elements early.
template <int TYPE, class W, class S>
__device__ void by_fours(int shift, int64_t numel, int64_t item, int64_t take, W whole, S single) {
    constexpr int kItem = kItemBytes / size_of(TYPE);
    const int lane = threadIdx.x & 31;
    for (int64_t lo = item * kItem - shift; take > 0; --take, lo += kItem) {
#pragma unroll 4
        for (int u = 0; u < kItem / 128; ++u) {
            const int64_t e = lo + u * 128 + lane * 4;
            if (e >= 0 && e + 4 <= numel) {
                whole(e);
            } else {
                for (int i = 0; i < 4; ++i)
                    if (e + i >= 0 && e + i < numel) single(e + i);
            }
        }
    }
}

template <int TYPE>
__device__ bool fours_at(const typename Elements<TYPE>::type* p, int shift) {
    return ((reinterpret_cast<uintptr_t>(p) - (uintptr_t)shift * size_of(TYPE)) & (4 * size_of(TYPE) - 1)) == 0;
}

// row[flat + i] = c * tensor[i]; zeros for a tensor that is absent.
template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
pack_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const WarpStart* __restrict__ starts, float* row, Limit limit) {
    pdl_begin();
    const float c = block_factor(limit).c;
    walk(infos, starts, [&](int t, const TensorInfo& info, int64_t item, int64_t take) {
        float* out = row + info.flat;
        const int shift = (int)((reinterpret_cast<uintptr_t>(out) >> 2) & 3);
        by_type(info.type, [&](auto type) {
            constexpr int TYPE = decltype(type)::value;
            typedef typename Elements<TYPE>::type T;
            const T* p = static_cast<const T*>(list.p[t]);
            if (!p) {
                by_fours<TYPE>(shift, info.numel, item, take, [&](int64_t e) { store4<DRACO_F32>(out + e, make_float4(0.f, 0.f, 0.f, 0.f), true); },
                               [&](int64_t e) { out[e] = 0.0f; });
                return;
            }
            const bool aligned = fours_at<TYPE>(p, shift);
            by_fours<TYPE>(shift, info.numel, item, take,
                           [&](int64_t e) {
                               const float4 x = load4<TYPE>(p + e, aligned);
                               store4<DRACO_F32>(out + e, make_float4(x.x * c, x.y * c, x.z * c, x.w * c), true);
                           },
                           [&](int64_t e) { out[e] = Elements<TYPE>::value(p[e]) * c; });
        });
    });
}

__device__ float4 step4(float4 w, float4 u, float s) {
    return make_float4(fmaf(-s, u.x, w.x), fmaf(-s, u.y, w.y), fmaf(-s, u.z, w.z), fmaf(-s, u.w, w.w));
}

// w <- w - scale c u; MASTER: the fp32 master copy instead, and w is that, rounded.  Nothing where |u| is not finite.
template <int N, bool MASTER>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
update_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const WarpStart* __restrict__ starts,
              const float* __restrict__ u, float* __restrict__ master, float scale, Limit limit) {
    pdl_begin();
    const Factor f = block_factor(limit);
    if (!f.finite) return;
    const float s = scale * f.c;
    walk(infos, starts, [&](int t, const TensorInfo& info, int64_t item, int64_t take) {
        if (!list.p[t]) return;
        const float* from = u + info.flat;
        float* m = MASTER ? master + info.flat : nullptr;
        by_type(info.type, [&](auto type) {
            constexpr int TYPE = decltype(type)::value;
            typedef typename Elements<TYPE>::type T;
            T* w = static_cast<T*>(list.p[t]);
            // the grid of the side that is both read and written
            const int shift = MASTER ? (int)(info.flat & 3) : (int)((reinterpret_cast<uintptr_t>(w) / size_of(TYPE)) & 3);
            const bool flat_aligned = fours_at<DRACO_F32>(from, shift), w_aligned = fours_at<TYPE>(w, shift);
            by_fours<TYPE>(shift, info.numel, item, take,
                           [&](int64_t e) {
                               const float4 x = load4<DRACO_F32>(from + e, flat_aligned);
                               const float4 old = MASTER ? load4<DRACO_F32>(m + e, true) : load4<TYPE>(w + e, true);
                               const float4 now = step4(old, x, s);
                               if (MASTER) store4<DRACO_F32>(m + e, now, true);
                               store4<TYPE>(w + e, now, w_aligned);
                           },
                           [&](int64_t e) {
                               const float now = fmaf(-s, from[e], MASTER ? m[e] : Elements<TYPE>::value(w[e]));
                               if (MASTER) m[e] = now;
                               w[e] = Elements<TYPE>::round(now);
                           });
        });
    });
}

}  // namespace
}  // namespace draco

using namespace draco;

// The sizes and types of a list, the split of its items over warps, and scratch for the partial sums.
struct draco_layout {
    int count, device;
    int64_t size;
    int64_t* numel;             // [count]
    uint8_t* type;              // [count]
    Part* parts;                // [num_parts], then that of the flat vector
    int num_parts;
    int all_blocks;
    TensorInfo* infos_dev;      // [count], then the flat vector's
    WarpStart* starts_dev;
    void* slots_dev;            // [all_blocks], then [blocks of the flat vector]; 8 bytes each
    void* segments_dev;         // [warps + count]
    float* factors_dev;         // [count]
    unsigned* ticket_dev;
};

namespace {

void free_layout(draco_layout* l) {
    if (!l) return;
    free(l->numel);
    free(l->type);
    free(l->parts);
    if (l->infos_dev) cudaFree(l->infos_dev);
    if (l->starts_dev) cudaFree(l->starts_dev);
    if (l->slots_dev) cudaFree(l->slots_dev);
    if (l->segments_dev) cudaFree(l->segments_dev);
    if (l->factors_dev) cudaFree(l->factors_dev);
    if (l->ticket_dev) cudaFree(l->ticket_dev);
    delete l;
}

int64_t items_of(int64_t numel, int type) {
    const int64_t item = kItemBytes / size_of(type), early = 16 / size_of(type) - 1;
    return numel ? (numel + early + item - 1) / item : 0;
}

// The WarpStarts of a part's tensors (infos[first ..]) and the tensors' segments; returns the number of blocks.
int split(TensorInfo* infos, int first, int count, int sm_count, int seg0, WarpStart* starts) {
    int64_t items = 0;
    for (int t = first; t < first + count; ++t) items += infos[t].items;
    const int64_t wanted = (items + kWarps - 1) / kWarps;
    const int blocks = (int)(wanted < 1 ? 1 : wanted < (int64_t)sm_count * kBlocksPerSm ? wanted : (int64_t)sm_count * kBlocksPerSm);
    const int warps = blocks * kWarps;
    const int used = items < warps ? (int)items : warps;   // the others have none: a tensor's segments are all written
    int t = first;
    int64_t before = 0;                                    // items of the tensors before t
    for (int w = 0; w <= warps; ++w) {
        const int64_t index = w < used ? items / used * w + items % used * w / used : items;
        while (t < first + count - 1 && index >= before + infos[t].items) before += infos[t++].items;
        starts[w].tensor = t - first;
        starts[w].item = index - before;
        starts[w].index = index;
        starts[w].pad = 0;
    }
    int w = 0;
    before = 0;
    for (t = first; t < first + count; ++t) {
        if (!infos[t].items) continue;
        while (starts[w + 1].index <= before) ++w;         // the warp of the tensor's first item
        int v = w;
        while (starts[v + 1].index < before + infos[t].items) ++v;
        infos[t].seg_first = seg0 + w + (t - first);
        infos[t].seg_count = v - w + 1;
        before += infos[t].items;
        w = v;
    }
    return blocks;
}

template <class F>
int with_capacity(int count, F f) {
    if (count <= 64) return f(std::integral_constant<int, 64>());
    if (count <= 512) return f(std::integral_constant<int, 512>());
    return f(std::integral_constant<int, kMaxPointers>());
}

template <int N>
Pointers<N> pointers_of(const void* const* list, const Part& part) {
    Pointers<N> p;
    for (int t = 0; t < part.count; ++t) p.p[t] = const_cast<void*>(list[part.first + t]);
    return p;
}

// The block sums of a list, or of the flat vector u (list null); norm: and the norm itself.
int measure(draco_layout* l, const void* const* list, const float* u, int kind, bool segments, float* norm, cudaStream_t st) {
    const void* flat[1] = {u};
    for (int k = 0; k < (list ? l->num_parts : 1); ++k) {
        const Part& part = l->parts[list ? k : l->num_parts];
        Part given = part;
        if (!list) given.first = 0;
        const int all = list ? l->all_blocks : part.blocks, block0 = list ? part.block0 : 0;
        char* slots = static_cast<char*>(l->slots_dev) + (list ? 0 : (size_t)l->all_blocks * 8);
        char* segs = static_cast<char*>(l->segments_dev) + 8 * ((size_t)part.block0 * kWarps + part.first);
        const int rc = with_capacity(part.count, [&](auto n) -> int {
            constexpr int N = decltype(n)::value;
            const Pointers<N> p = pointers_of<N>(list ? list : flat, given);
            auto go = [&](auto kernel, auto* slot) {
                typedef decltype(slot) S;
                launch_dependent(kernel, dim3(part.blocks), dim3(kThreads), 0, st, p, (const TensorInfo*)l->infos_dev + part.first,
                                 (const WarpStart*)l->starts_dev + part.starts, (S)slots, block0, (S)segs, norm, all, l->ticket_dev);
            };
            if (kind == DRACO_NORM_2) {
                if (segments) go(measure_kernel<SumSquares, N, true>, (double*)nullptr);
                else go(measure_kernel<SumSquares, N, false>, (double*)nullptr);
            } else {
                if (segments) go(measure_kernel<MaxMagnitude, N, true>, (unsigned long long*)nullptr);
                else go(measure_kernel<MaxMagnitude, N, false>, (unsigned long long*)nullptr);
            }
            DRACO_CUDA(cudaGetLastError());
            return DRACO_OK;
        });
        if (rc != DRACO_OK) return rc;
    }
    return DRACO_OK;
}

int finish_each(draco_layout* l, int kind, float max_norm, float* norm, float* each, float* factors, cudaStream_t st) {
    const dim3 grid(l->count + 1), block(kThreads);
    if (kind == DRACO_NORM_2)
        launch_dependent(each_kernel<SumSquares>, grid, block, 0, st, (const TensorInfo*)l->infos_dev, l->count, (const double*)l->segments_dev,
                         (const double*)l->slots_dev, l->all_blocks, max_norm, norm, each, factors);
    else
        launch_dependent(each_kernel<MaxMagnitude>, grid, block, 0, st, (const TensorInfo*)l->infos_dev, l->count,
                         (const unsigned long long*)l->segments_dev, (const unsigned long long*)l->slots_dev, l->all_blocks, max_norm, norm, each, factors);
    DRACO_CUDA(cudaGetLastError());
    return DRACO_OK;
}

bool on_device(const draco_layout* l) {
    int device = -1;
    return cudaGetDevice(&device) == cudaSuccess && device == l->device;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Every address on its element's boundary.
bool addresses_ok(const draco_layout* l, const void* const* list) {
    if (!list) return false;
    for (int t = 0; t < l->count; ++t)
        if (reinterpret_cast<uintptr_t>(list[t]) % size_of(l->type[t])) return false;
    return true;
}

bool apart(const draco_layout* l, const void* const* list, const void* flat, int64_t bytes) {
    const uintptr_t y = reinterpret_cast<uintptr_t>(flat);
    for (int t = 0; t < l->count; ++t) {
        const uintptr_t x = reinterpret_cast<uintptr_t>(list[t]);
        const uintptr_t n = (uintptr_t)l->numel[t] * size_of(l->type[t]);
        if (x && n && x < y + (uintptr_t)bytes && y < x + n) return false;
    }
    return true;
}

// 1: no address of a tensor with elements stands twice in `to`, nor in another place of `from`; 0: one does; negative: a status.
int distinct(const draco_layout* l, const void* const* to, const void* const* from) {
    constexpr int kStack = 2048;
    struct Entry { uintptr_t address; int tensor; };
    Entry stack[kStack], *table = stack;
    int size = 64;
    while (size < 4 * l->count) size *= 2;                 // at most half full with both lists
    if (size > kStack) {
        table = static_cast<Entry*>(malloc(sizeof(Entry) * size));
        if (!table) return DRACO_ENOMEM;
    }
    memset(table, 0, sizeof(Entry) * size);
    int ok = 1;
    for (int pass = 0; pass < (to == from ? 1 : 2) && ok; ++pass) {
        const void* const* list = pass ? from : to;
        for (int t = 0; t < l->count; ++t) {
            const uintptr_t a = reinterpret_cast<uintptr_t>(list[t]);
            if (!a || !l->numel[t]) continue;
            uint32_t h = (uint32_t)((a >> 1) * 0x9E3779B97F4A7C15ull >> 32) & (size - 1);
            while (table[h].address && table[h].address != a) h = (h + 1) & (size - 1);
            if (pass ? table[h].address && table[h].tensor != t : table[h].address != 0) {
                ok = 0;
                break;
            }
            if (!pass) table[h] = {a, t};
        }
    }
    if (table != stack) free(table);
    return ok;
}

bool kind_ok(int kind) { return kind == DRACO_NORM_2 || kind == DRACO_NORM_MAX; }

}  // namespace

extern "C" {

int draco_layout_create(int count, const int64_t* numel, const int* type, draco_layout** out) {
    if (!out) return DRACO_EINVAL;
    *out = nullptr;
    if (count < 1 || !numel || !type) return DRACO_EINVAL;
    if (count > DRACO_MAX_TENSORS) return DRACO_ELIMIT;
    int64_t size = 0;
    for (int t = 0; t < count; ++t) {
        if (numel[t] < 0 || numel[t] > ((int64_t)1 << 48) || size > ((int64_t)1 << 48)) return DRACO_EINVAL;
        if (type[t] != DRACO_F32 && type[t] != DRACO_BF16 && type[t] != DRACO_F16) return DRACO_EINVAL;
        size += numel[t];
    }
    draco_layout* l = new (std::nothrow) draco_layout();
    if (!l) return DRACO_ENOMEM;
    memset(l, 0, sizeof(*l));
    l->count = count;
    l->size = size;
    l->num_parts = (count + kMaxPointers - 1) / kMaxPointers;
    int sm_count = 0;
    cudaError_t err = cudaGetDevice(&l->device);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&sm_count, cudaDevAttrMultiProcessorCount, l->device);
    if (err != cudaSuccess) { free_layout(l); return cuda_fail(err, "cudaGetDevice"); }
    const int64_t most_starts = (int64_t)(l->num_parts + 1) * (sm_count * kBlocksPerSm * kWarps + 1);
    l->numel = static_cast<int64_t*>(malloc(sizeof(int64_t) * count));
    l->type = static_cast<uint8_t*>(malloc(count));
    l->parts = static_cast<Part*>(malloc(sizeof(Part) * (l->num_parts + 1)));
    TensorInfo* infos = static_cast<TensorInfo*>(calloc(count + 1, sizeof(TensorInfo)));
    WarpStart* starts = static_cast<WarpStart*>(malloc(sizeof(WarpStart) * most_starts));
    int rc = DRACO_OK;
    if (!l->numel || !l->type || !l->parts || !infos || !starts) rc = DRACO_ENOMEM;
    int64_t num_starts = 0;
    int flat_blocks = 0;
    if (rc == DRACO_OK) {
        int64_t flat = 0;
        for (int t = 0; t < count; ++t) {
            l->numel[t] = infos[t].numel = numel[t];
            l->type[t] = (uint8_t)(infos[t].type = type[t]);
            infos[t].flat = flat;
            infos[t].items = items_of(numel[t], type[t]);
            flat += numel[t];
        }
        infos[count].numel = size;
        infos[count].type = DRACO_F32;
        infos[count].items = items_of(size, DRACO_F32);
        for (int k = 0; k <= l->num_parts; ++k) {
            Part& p = l->parts[k];
            p.first = k < l->num_parts ? k * kMaxPointers : count;
            p.count = k < l->num_parts ? (count - p.first < kMaxPointers ? count - p.first : kMaxPointers) : 1;
            p.starts = num_starts;
            p.block0 = l->all_blocks;
            p.blocks = split(infos, p.first, p.count, sm_count, l->all_blocks * kWarps + p.first, starts + num_starts);
            num_starts += p.blocks * kWarps + 1;
            if (k < l->num_parts) l->all_blocks += p.blocks;
            else flat_blocks = p.blocks;
        }
    }
#define DRACO_TRY(call)                                                                          \
    do {                                                                                         \
        if (rc == DRACO_OK) {                                                                    \
            cudaError_t e__ = (call);                                                            \
            if (e__ != cudaSuccess) rc = cuda_fail(e__, #call);                                  \
        }                                                                                        \
    } while (0)
    const size_t slots = (size_t)l->all_blocks + flat_blocks;
    DRACO_TRY(cudaMalloc(&l->infos_dev, sizeof(TensorInfo) * (count + 1)));
    DRACO_TRY(cudaMalloc(&l->starts_dev, sizeof(WarpStart) * num_starts));
    DRACO_TRY(cudaMalloc(&l->slots_dev, 8 * slots));
    DRACO_TRY(cudaMalloc(&l->segments_dev, 8 * (slots * kWarps + count + 1)));
    DRACO_TRY(cudaMalloc(&l->factors_dev, sizeof(float) * count));
    DRACO_TRY(cudaMalloc(&l->ticket_dev, sizeof(unsigned)));
    DRACO_TRY(cudaMemset(l->ticket_dev, 0, sizeof(unsigned)));
    DRACO_TRY(cudaMemcpy(l->infos_dev, infos, sizeof(TensorInfo) * (count + 1), cudaMemcpyHostToDevice));
    DRACO_TRY(cudaMemcpy(l->starts_dev, starts, sizeof(WarpStart) * num_starts, cudaMemcpyHostToDevice));
    DRACO_TRY(cudaStreamSynchronize(nullptr));
#undef DRACO_TRY
    free(infos);
    free(starts);
    if (rc != DRACO_OK) { free_layout(l); return rc; }
    *out = l;
    return DRACO_OK;
}

int draco_layout_destroy(draco_layout* layout) {
    free_layout(layout);
    return DRACO_OK;
}

int64_t draco_layout_size(const draco_layout* layout) { return layout ? layout->size : DRACO_EINVAL; }

int draco_norm(draco_layout* layout, const void* const* tensors, int kind, float* norm, float* each, void* stream) {
    if (!layout || !addresses_ok(layout, tensors) || !kind_ok(kind) || !norm || !aligned4(norm) || !aligned4(each) || !on_device(layout)) return DRACO_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    const int rc = measure(layout, tensors, nullptr, kind, each != nullptr, each ? nullptr : norm, st);
    if (rc != DRACO_OK || !each) return rc;
    return finish_each(layout, kind, 0.0f, norm, each, nullptr, st);
}

int draco_clip(draco_layout* layout, const void* const* tensors, void* const* out, int kind, float max_norm, int separately, float* norm, float* each,
               void* stream) {
    if (!layout || !addresses_ok(layout, tensors) || (out && !addresses_ok(layout, out)) || !kind_ok(kind) || !(max_norm >= 0.0f) || !aligned4(norm) ||
        !aligned4(each) || (each && !separately) || !on_device(layout))
        return DRACO_EINVAL;
    const void* const* to = out ? out : tensors;
    if (out)
        for (int t = 0; t < layout->count; ++t)
            if (layout->numel[t] && !out[t] != !tensors[t]) return DRACO_EINVAL;
    const int alone = distinct(layout, to, tensors);
    if (alone <= 0) return alone < 0 ? alone : DRACO_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    int rc = measure(layout, tensors, nullptr, kind, separately != 0, nullptr, st);
    if (rc == DRACO_OK && separately) rc = finish_each(layout, kind, max_norm, norm, each, layout->factors_dev, st);
    for (int k = 0; k < layout->num_parts && rc == DRACO_OK; ++k) {
        const Part& part = layout->parts[k];
        const Limit limit = {layout->slots_dev, layout->all_blocks, kind, max_norm, k == 0 ? norm : nullptr};
        rc = with_capacity(part.count, [&](auto n) -> int {
            constexpr int N = decltype(n)::value;
            launch_dependent(scale_kernel<N>, dim3(part.blocks), dim3(kThreads), 0, st, pointers_of<N>(tensors, part), pointers_of<N>(to, part),
                             (const TensorInfo*)layout->infos_dev + part.first, (const WarpStart*)layout->starts_dev + part.starts, limit,
                             separately ? (const float*)layout->factors_dev + part.first : nullptr);
            DRACO_CUDA(cudaGetLastError());
            return DRACO_OK;
        });
    }
    return rc;
}

int draco_pack(draco_layout* layout, const void* const* tensors, int kind, float max_norm, float* row, float* norm, void* stream) {
    if (!layout || !addresses_ok(layout, tensors) || !kind_ok(kind) || !(max_norm >= 0.0f) || (!row && layout->size) || !aligned4(row) || !aligned4(norm) ||
        !on_device(layout) || !apart(layout, tensors, row, 4 * layout->size))
        return DRACO_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    const bool wanted = norm || !isinf(max_norm);
    int rc = wanted ? measure(layout, tensors, nullptr, kind, false, nullptr, st) : (int)DRACO_OK;
    for (int k = 0; k < layout->num_parts && rc == DRACO_OK; ++k) {
        const Part& part = layout->parts[k];
        const Limit limit = {wanted ? layout->slots_dev : nullptr, layout->all_blocks, kind, max_norm, k == 0 ? norm : nullptr};
        rc = with_capacity(part.count, [&](auto n) -> int {
            constexpr int N = decltype(n)::value;
            launch_dependent(pack_kernel<N>, dim3(part.blocks), dim3(kThreads), 0, st, pointers_of<N>(tensors, part),
                             (const TensorInfo*)layout->infos_dev + part.first, (const WarpStart*)layout->starts_dev + part.starts, row, limit);
            DRACO_CUDA(cudaGetLastError());
            return DRACO_OK;
        });
    }
    return rc;
}

int draco_update(draco_layout* layout, void* const* params, const float* u, float* master, int kind, float max_norm, float scale, float* norm, void* stream) {
    if (!layout || !addresses_ok(layout, params) || !kind_ok(kind) || !(max_norm >= 0.0f) || !(scale == scale) || (!u && layout->size) || !aligned16(u) || !aligned16(master) ||
        !aligned4(norm) || !on_device(layout))
        return DRACO_EINVAL;
    const int64_t bytes = 4 * layout->size;
    const uintptr_t x = reinterpret_cast<uintptr_t>(u), y = reinterpret_cast<uintptr_t>(master);
    if (!apart(layout, params, u, bytes) || (master && (!apart(layout, params, master, bytes) || (x < y + bytes && y < x + bytes)))) return DRACO_EINVAL;
    const int alone = distinct(layout, params, params);
    if (alone <= 0) return alone < 0 ? alone : DRACO_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    const bool wanted = norm || !isinf(max_norm);
    int rc = wanted ? measure(layout, nullptr, u, kind, false, nullptr, st) : (int)DRACO_OK;
    for (int k = 0; k < layout->num_parts && rc == DRACO_OK; ++k) {
        const Part& part = layout->parts[k];
        const Limit limit = {wanted ? static_cast<char*>(layout->slots_dev) + (size_t)layout->all_blocks * 8 : nullptr,
                             layout->parts[layout->num_parts].blocks, kind, max_norm, k == 0 ? norm : nullptr};
        rc = with_capacity(part.count, [&](auto n) -> int {
            constexpr int N = decltype(n)::value;
            auto go = [&](auto kernel) {
                launch_dependent(kernel, dim3(part.blocks), dim3(kThreads), 0, st, pointers_of<N>(params, part),
                                 (const TensorInfo*)layout->infos_dev + part.first, (const WarpStart*)layout->starts_dev + part.starts, u, master, scale, limit);
            };
            if (master) go(update_kernel<N, true>);
            else go(update_kernel<N, false>);
            DRACO_CUDA(cudaGetLastError());
            return DRACO_OK;
        });
    }
    return rc;
}

}  // extern "C"
