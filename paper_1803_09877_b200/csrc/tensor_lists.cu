// Lists of tensors next to the flat vectors of the code: norms, clipping, packing into a row of G, updates from a decoded sum.
//
//   N = sqrt(sum_t sum_i g_t[i]^2)  or  max_t,i |g_t[i]|        c = max_norm / N if N > max_norm, else 1
//   clip: g_t <- c g_t       pack: row[off_t + i] = c g_t[i]       update: w_t[i] <- w_t[i] - scale c u[off_t + i],  N = |u|
//
// Long lists are bound by HBM: the list is read for its norm (up to 7.0 TB/s: 2.1 GB of fp32 in 301 us; 465 bf16 tensors, 120 MB, in 22.4 us, 5.4 TB/s)
// and a second time to be scaled, packed or updated (138 M bf16 packed: 46 + 122 us alone, 179 together, 6.2 TB/s of all that moves).  A pass
// that knew the factor beforehand would read once; the gradients would have to stay on the chip for that.  Short ones are
// bound by latency: one launch of one cluster, 2.5 to 5 us.
//
// Split.  A list is cut into lines of one word a lane, which begin on word boundaries of the tensor's memory, wherever the tensor
// begins (those of a sum, whose bits are not to depend on that, on its first element), and the lines are dealt to warps in contiguous
// chunks of equal cost, so that a tensor of any size takes what it holds.
// The chunks depend on sizes alone and are made once, with the layout; the tensors' addresses come with every call, as kernel
// parameters (a graph captures them, nothing is uploaded), at most kMaxPointers a launch; longer lists take several launches.
// No warp waits for one of another block but at a cluster's hardware barrier: block sums are written out and added up, in a fixed
// order, by whoever needs the norm next.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>
#include <pthread.h>
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
constexpr int kMaxPointers = 2000;                // two lists of 8-byte pointers within the 32,764 bytes of kernel parameters
constexpr int64_t kMostElements = (int64_t)1 << 40; // a warp counts its lines and their elements in 32 bits
constexpr int kBatch = 8;                           // lines that a warp loads at once

// Chunks.  A tensor that a warp comes to costs it as much time as kVisit lines, the wait for its first ones: lists of many small tensors are
// spread over more warps (norm of 300 bf16 tensors, 300 k elements in all: 10.7 us by lines alone, 4.2 with 8; 465 tensors, 60.2 M,
// 25.7 and 23.3).  kMinLines: cost of a chunk before the list gets another warp; 2, 4 and 8 within 5 % of one another, 4 ahead.
constexpr int kVisit = 8, kMinLines = 4;
// Second passes of long lists: several waves of blocks with short chunks.  SMs that are further from memory take longer over the same share, and
// with one wave the last of them holds the others up (138 M bf16 packed: one wave 201 us, chunks of 24 lines 185, of 12 182, of 8 180, of 4 208; with
// a master copy updated, 60.2 M 186, 176, 173, 171, 169).  Below kWaveLines lines a warp one wave is level or faster.  Warps that draw chunks from a
// counter instead wait for it (253 us).
constexpr int kWaveLines = 32, kWavesLines = 8, kWaves = 64;
// In place most calls have nothing to write, and blocks that only find that out cost 1.2 us a thousand: always one wave (1.0e9 bf16 below the limit
// 296 us, chunks of 64 lines 306, of 8 346; above it, which so costs 7 % more, 966, 925, 901).

// A list of up to kSmallTensors tensors that costs at most kSmallLines lines a warp is left to one cluster of up to kSmallBlocks blocks: one launch
// instead of two, 4 us of the caller's time instead of 6.5.  GPU time, two launches / one: clip of 2000 fp32 values 6.6 / 3.5 us, of 100,000 in 20 tensors
// 4.3 / 4.6, of 150,000 4.4 / 5.7: near the line a replayed graph, which has no caller's time, is 0.3 us slower for it.
constexpr int kSmallTensors = 512, kSmallBlocks = 16, kSmallLines = 8;

// Lines: 512 bytes of a tensor's own type (one 16-byte word a lane) where the tensor alone is walked, 128 elements (four a lane) where
// it goes beside its part of a flat vector.
enum { BY_BYTES = 0, BY_ELEMENTS = 1 };

struct TensorInfo {
    int64_t numel;
    int64_t flat;          // offset in the flat vector
    int64_t lines[2];      // wherever between two boundaries the tensor starts
    int32_t type;
    int32_t seg_first;     // partial sums of this tensor alone, one for each chunk that has lines of it
    int32_t seg_count;
    int32_t pad;
};

struct Chunk {             // `left` neighbouring lines: upwards from line `at` of tensor `tensor`, or downwards from the one before it
    int64_t at;
    int64_t numel, flat, lines;    // of that tensor: known as soon as the chunk is
    int32_t left, tensor, type, pad;
};

// A chunk a warp.  MEASURE: upwards, one wave of blocks, which leave few sums to add up.  The second passes go
// back, from the end of the list (and of each chunk), part of which is still in L2 (15 rows of 1,000,003 clipped: 35.2 us upwards, 31.4).
enum { MEASURE = 0, IN_PLACE = 1, BYTES = 2, ELEMENTS = 3, TABLES = 4 };

struct Part {              // the tensors of one launch
    int first, count;
    int block0;            // of the partial sums
    int blocks[TABLES];
    int64_t table[TABLES]; // into the table of chunks
};

struct Result {            // of a measurement
    float c;
    int finite;
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

// N neighbouring elements as they lie in memory.
template <int TYPE, int N>
struct alignas(N * size_of(TYPE)) Vec {
    uint32_t w[N * size_of(TYPE) / 4];
    __device__ typename Elements<TYPE>::type element(int i) const {
        typename Elements<TYPE>::type x;
        if (TYPE == DRACO_F32) {
            memcpy(&x, &w[i], sizeof(x));
        } else {
            const uint16_t half = (uint16_t)(w[i / 2] >> (i & 1) * 16);
            memcpy(&x, &half, sizeof(x));
        }
        return x;
    }
    __device__ float value(int i) const {
        if (TYPE == DRACO_BF16) return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);     // the upper half of an fp32
        return Elements<TYPE>::value(element(i));
    }
    __device__ bool any() const {                          // other than zeros of either sign, 16-bit types
        uint32_t bits = 0;
#pragma unroll
        for (int i = 0; i < N * size_of(TYPE) / 4; ++i) bits |= w[i];
        return (bits & 0x7fff7fffu) != 0;
    }
    __device__ void set(const float (&x)[N]) {
#pragma unroll
        for (int i = 0; i < N; i += 4 / size_of(TYPE)) {
            if (TYPE == DRACO_F32) w[i] = __float_as_uint(x[i]);
            else if (TYPE == DRACO_BF16) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(x[i], x[i + 1]);
                memcpy(&w[i / 2], &h, 4);
            } else {
                const __half2 h = __floats2half2_rn(x[i], x[i + 1]);
                memcpy(&w[i / 2], &h, 4);
            }
        }
    }
};

// ---- sums of squares and largest magnitudes, in 64-bit slots ----

// Sums are kept in fp64: products of fp32 values are exact there and neither overflow nor vanish.  Squares of a 16-byte word of 16-bit
// values are added in fp32 first (they have 22 bits at most; eight of them are off by 8 * 2^-24 at most) and in fp64 where that sum leaves the
// range in which fp32 loses nothing that counts: one conversion a word instead of eight.
struct SumSquares {
    typedef double Slot;
    static constexpr bool kOrdered = true;                 // roundings depend on the order
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
            for (int i = 0; i < N; ++i) one<TYPE>(a, v.element(i));
        } else {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float x = v.value(i);
                s = fmaf(x, x, s);
            }
            if (TYPE == DRACO_F16 || (s >= 0x1p-100f && s <= 0x1p120f)) {
                a += (double)s;
            } else if (v.any()) {
#pragma unroll
                for (int i = 0; i < N; ++i) one<TYPE>(a, v.element(i));
            }
        }
    }
    static __device__ double norm(Slot a) { return sqrt(a); }
};

// Magnitudes compare like their bit patterns, infinity above all numbers and NaN above infinity; 16-bit ones two at a time.
struct MaxMagnitude {
    typedef unsigned long long Slot;
    static constexpr bool kOrdered = false;
    static __device__ Slot zero() { return 0; }
    static __device__ void add(Slot& a, Slot b) { a = a > b ? a : b; }
    template <int TYPE>
    static __device__ void one(Slot& a, typename Elements<TYPE>::type x) {
        const unsigned b = __float_as_uint(Elements<TYPE>::value(x)) & 0x7fffffffu;
        a = max((unsigned)a, b);
    }
    template <int TYPE, int N>
    static __device__ void word(Slot& a, const Vec<TYPE, N>& v) {
        if (TYPE == DRACO_F32) {
#pragma unroll
            for (int i = 0; i < N; ++i) one<TYPE>(a, v.element(i));
        } else {
            unsigned m = 0;
#pragma unroll
            for (int i = 0; i < N / 2; ++i) m = __vmaxu2(m, v.w[i] & 0x7fff7fffu);
            const unsigned short largest = (unsigned short)max(m & 0xffffu, m >> 16);
            typename Elements<TYPE>::type x;
            memcpy(&x, &largest, sizeof(x));
            one<TYPE>(a, x);
        }
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

// Where a kernel gets the factor from: formed already, or to be formed from the sums by every block for itself, which one wave of blocks
// has sooner than the measurement's last block would have it; null both: none is wanted.
struct Limit {
    const Result* result;
    const void* slots;
    int count, kind;
    float max_norm;
    float* norm;           // written by the first block if it forms the norm; may be null
};

__device__ Result result_of(double norm, float max_norm) {
    Result r;
    r.finite = isfinite((float)norm);
    r.c = r.finite && norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
    return r;
}

template <class K>
__device__ double norm_of(const void* slots, int first, int count) {
    __shared__ typename K::Slot shared[kWarps];
    typename K::Slot a = K::zero();
    for (int i = threadIdx.x; i < count; i += kThreads) K::add(a, __ldcg(static_cast<const typename K::Slot*>(slots) + first + i));
    return K::norm(block_total<K>(a, shared));
}

__device__ __forceinline__ Result factor(const Limit& l) {
    if (l.result) return *l.result;
    if (!l.slots) return Result{1.0f, 1};
    const double n = l.kind == DRACO_NORM_2 ? norm_of<SumSquares>(l.slots, 0, l.count) : norm_of<MaxMagnitude>(l.slots, 0, l.count);
    if (l.norm && blockIdx.x == 0 && threadIdx.x == 0) *l.norm = (float)n;
    return result_of(n, l.max_norm);
}

// ---- the walk over a warp's lines ----

// f(index, type, offset in the flat vector, numel, first line, lines) for every tensor that a chunk has lines of.
template <bool DOWN, int BY, class F>
__device__ __forceinline__ void walk(const TensorInfo* infos, const Chunk& chunk, F f) {
    int left = chunk.left, t = chunk.tensor, type = chunk.type;
    int64_t at = chunk.at, numel = chunk.numel, flat = chunk.flat, lines = chunk.lines;
    while (left > 0) {
        const int take = (int)min((int64_t)left, DOWN ? at : lines - at);
        if (take > 0) f(t, type, flat, numel, DOWN ? at - take : at, take);
        left -= take;
        if (left <= 0) break;
        t += DOWN ? -1 : 1;
        const TensorInfo* i = infos + t;
        numel = i->numel;
        flat = i->flat;
        lines = i->lines[BY];
        type = i->type;
        at = DOWN ? lines : 0;
    }
}

template <class F>
__device__ __forceinline__ void by_type(int type, F f) {
    if (type == DRACO_F32) f(std::integral_constant<int, DRACO_F32>());
    else if (type == DRACO_BF16) f(std::integral_constant<int, DRACO_BF16>());
    else f(std::integral_constant<int, DRACO_F16>());
}

template <class F>
__device__ __forceinline__ void by_alignment(bool aligned, F f) {
    if (aligned) f(std::true_type());
    else f(std::false_type());
}

// A part of a tensor: lines of VEC elements a lane, the first of which begins `origin` elements into the tensor (negative at its start,
// where the tensor begins behind a word's boundary).  Elements origin + begin .. origin + end - 1 are the tensor's.
template <int VEC>
struct Range {
    int64_t origin;
    int take, begin, end;
    __device__ Range(int64_t numel, int shift, int64_t line, int take_)
        : origin(line * 32 * VEC - shift), take(take_), begin(origin < 0 ? shift : 0), // the last line may lie behind the tensor
          end((int)max(min(numel - origin, (int64_t)take_ * 32 * VEC), (int64_t)0)) {}

    // batch(at, low, high) for BATCH lines at a time, `at` this lane's place (from origin on) in the first of them: its words u = 0 .. BATCH - 1,
    // at + 32 VEC u, are all the tensor's where low <= u * 32 VEC <= high.
    template <bool DOWN, int BATCH, class F>
    __device__ __forceinline__ void batches(F batch) const {
        const int lane = (threadIdx.x & 31) * VEC;
        const int count = (take + BATCH - 1) / BATCH;
        for (int i = 0; i < count; ++i) {
            const int at = (DOWN ? count - 1 - i : i) * (BATCH * 32 * VEC) + lane;
            batch(at, begin - at, end - VEC - at);
        }
    }

    // single(i) for the elements of a word that reaches over one of the tensor's ends, a lane each.
    template <class F>
    __device__ __forceinline__ void ends(F single) const {
        const int lane = threadIdx.x & 31, tail = end & ~(VEC - 1);
        if (begin > 0 && lane >= begin && lane < min(VEC, end)) single(lane);
        if (tail + lane < end && (tail > 0 || begin == 0)) single(tail + lane);
    }
};

#define DRACO_WHOLE(u) ((u) * 32 * kVec >= low && (u) * 32 * kVec <= high)

template <int TYPE>
__device__ int behind_word(const void* p) { return (int)((reinterpret_cast<uintptr_t>(p) & 15u) / size_of(TYPE)); }

// Zeros where `here` is false.
template <int TYPE, int N, bool ALIGNED>
__device__ __forceinline__ Vec<TYPE, N> load(bool here, const typename Elements<TYPE>::type* p) {
    Vec<TYPE, N> v = {};
    if (!here) return v;
    if (ALIGNED) return *reinterpret_cast<const Vec<TYPE, N>*>(p);
    if (TYPE == DRACO_F32) {
#pragma unroll
        for (int i = 0; i < N; ++i) v.w[i] = reinterpret_cast<const uint32_t*>(p)[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 2) v.w[i / 2] = reinterpret_cast<const uint16_t*>(p)[i] | (uint32_t)reinterpret_cast<const uint16_t*>(p)[i + 1] << 16;
    }
    return v;
}

template <int TYPE, int N, bool ALIGNED>
__device__ __forceinline__ void store(typename Elements<TYPE>::type* p, const Vec<TYPE, N>& v) {
    if (ALIGNED) {
        *reinterpret_cast<Vec<TYPE, N>*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = v.element(i);
    }
}

// A word as it is loaded, by its address: at once (BY = 16); 8 + 8 bytes, on a boundary of 8; 4 + 8 + 4, of 4; else 2 + 8 + 4 + 2 (BY = 2), where the
// second piece is on one of 8, or 2 + 4 + 8 + 2 (BY = 6).
template <int TYPE, int N, int BY>
struct Loaded {
    static constexpr bool kOdd = BY == 2 || BY == 6;
    uint32_t w[kOdd ? 5 : 4];
    template <int BYTES>
    __device__ __forceinline__ void piece(int i, const char* p) {       // from w[i] on
        if (BYTES == 2) {
            w[i] = *reinterpret_cast<const uint16_t*>(p);
        } else if (BYTES == 4) {
            w[i] = *reinterpret_cast<const uint32_t*>(p);
        } else {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            w[i] = v.x, w[i + 1] = v.y;
        }
    }
    __device__ __forceinline__ void load(bool here, const typename Elements<TYPE>::type* q) {
#pragma unroll
        for (int i = 0; i < (kOdd ? 5 : 4); ++i) w[i] = 0;
        if (!here) return;
        const char* p = reinterpret_cast<const char*>(q);
        if (BY == 16) {
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
        } else if (BY == 8) {
            piece<8>(0, p), piece<8>(2, p + 8);
        } else if (BY == 4) {
            piece<4>(0, p), piece<8>(1, p + 4), piece<4>(3, p + 12);
        } else if (BY == 2) {
            piece<2>(0, p), piece<8>(1, p + 2), piece<4>(3, p + 10), piece<2>(kOdd ? 4 : 0, p + 14);
        } else {
            piece<2>(0, p), piece<4>(1, p + 2), piece<8>(2, p + 6), piece<2>(kOdd ? 4 : 0, p + 14);
        }
    }
    __device__ __forceinline__ Vec<TYPE, N> word() const {
        Vec<TYPE, N> v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.w[i] = !kOdd ? w[i] : __funnelshift_l(i ? w[i] : w[0] << 16, w[kOdd ? i + 1 : i], 16);
        return v;
    }
};

// BY = 16: lines begin on a word's boundary, others on the tensor's first element.
template <class K, int TYPE, int BY>
__device__ __forceinline__ void measure_by(const void* base, int shift, int64_t numel, int64_t line, int take, typename K::Slot& acc) {
    constexpr int kVec = 16 / size_of(TYPE);
    typedef typename Elements<TYPE>::type T;
    typedef Loaded<TYPE, kVec, BY> V;
    const Range<kVec> range(numel, BY == 16 ? shift : 0, line, take);
    const T* p = static_cast<const T*>(base) + range.origin;
    // One half of a batch comes while the other is added up.  us, eight lines then their sums / halves of four / of two: 60.2 M bf16 23.3, 22.4, 24.7;
    // 45 rows of 11.7 M fp32 304, 314, 301 (three: 309).  Words loaded in pieces, in halves of three and four: 0.2 and 0.5 us more for 1 M bf16 in 60 tensors.
    constexpr int kHalf = TYPE == DRACO_F32 || BY < 16 ? 2 : 4, kStep = kHalf * 32 * kVec;
    const int lane = (threadIdx.x & 31) * kVec;
    V x[kHalf], y[kHalf];
    auto fetch = [&](V* v, int at) {
        const int low = range.begin - at, high = range.end - kVec - at;
#pragma unroll
        for (int u = 0; u < kHalf; ++u) v[u].load(DRACO_WHOLE(u), p + at + u * 32 * kVec);
    };
    auto add = [&](const V* v) {
#pragma unroll
        for (int u = 0; u < kHalf; ++u) K::template word<TYPE, kVec>(acc, v[u].word());
    };
    fetch(x, lane);
    for (int i = 0; i < take; i += 2 * kHalf) {
        const int at = i * 32 * kVec + lane;
        fetch(y, at + kStep);
        add(x);
        fetch(x, at + 2 * kStep);
        add(y);
    }
    range.ends([&](int i) { K::template one<TYPE>(acc, p[i]); });
}

// Where roundings depend on the order of a sum, that order does not depend on the address: the words that are added up begin with the tensor's first
// element, so that equal gradients have equal norms, to the last bit, and make equal rows.  A tensor that begins elsewhere than on a
// word's boundary has its words loaded in pieces, out of L1 but for the first (us, on the boundary and off it: 60.2 M bf16 in 465 tensors 23.3, 26.0; 45 rows of
// 11.7 M fp32 302, in two pieces 306, in three 331; with pieces of 4 bytes and less 28, 366.  Words joined from two aligned ones, the other by a
// shuffle: 27, 318, and 1 to 2 us for what the two ends of each tensor then need).
template <class K, int TYPE>
__device__ __forceinline__ void measure_lines(const void* base, int64_t numel, int64_t line, int take, typename K::Slot& acc) {
    const int shift = behind_word<TYPE>(base);
    const int bytes = shift * size_of(TYPE) % 8;
    if (!K::kOrdered || shift == 0) measure_by<K, TYPE, 16>(base, shift, numel, line, take, acc);
    else if (bytes == 0) measure_by<K, TYPE, 8>(base, shift, numel, line, take, acc);
    else if (TYPE == DRACO_F32 || bytes == 4) measure_by<K, TYPE, 4>(base, shift, numel, line, take, acc);
    else if (bytes == 6) measure_by<K, TYPE, 2>(base, shift, numel, line, take, acc);
    else measure_by<K, TYPE, 6>(base, shift, numel, line, take, acc);
}

// Block sums to slots[block0 + blockIdx.x]; finish: the norm of all, too, from the block that finishes last (earlier launches of the measurement have
// finished before this one begins, and one launch either runs or does not, so that the ticket is back at zero whatever happens).  SEGMENTS: the
// sums of each warp's part of each tensor to segments[warp + tensor], a place of its own for every such pair, since both only grow along the
// list.
template <class K, int N, bool SEGMENTS>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
measure_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const Chunk* __restrict__ chunks,
               typename K::Slot* slots, int block0, int all_blocks, unsigned* ticket, typename K::Slot* segments, bool finish, float max_norm,
               float* norm, Result* result) {
    const int w = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const Chunk chunk = chunks[w];
    pdl_begin();
    __shared__ typename K::Slot shared[kWarps];
    __shared__ bool last;
    typename K::Slot acc = K::zero();
    walk<false, BY_BYTES>(infos, chunk, [&](int t, int type_, int64_t, int64_t numel, int64_t line, int take) {
        typename K::Slot a = K::zero();
        if (list.p[t]) by_type(type_, [&](auto type) { measure_lines<K, decltype(type)::value>(list.p[t], numel, line, take, SEGMENTS ? a : acc); });
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
        if (finish) {
            __threadfence();
            last = atomicInc(ticket, gridDim.x - 1) == gridDim.x - 1;  // back at zero after the last
            __threadfence();
        }
    }
    if (!finish) return;
    __syncthreads();
    if (!last) return;
    const double n = norm_of<K>(slots, 0, all_blocks);
    if (threadIdx.x == 0) {
        if (norm) *norm = (float)n;
        if (result) *result = result_of(n, max_norm);
    }
}

// One block a tensor: its segments added up, its norm and factor; one block more: the norm of all.
template <class K>
__global__ void __launch_bounds__(kThreads)
each_kernel(const TensorInfo* __restrict__ infos, const typename K::Slot* segments, const typename K::Slot* slots, int all_blocks, float max_norm,
            float* norm, float* each, float* factors) {
    const bool all = blockIdx.x == gridDim.x - 1;
    const int first = all ? 0 : infos[blockIdx.x].seg_first, count = all ? all_blocks : infos[blockIdx.x].seg_count;
    pdl_begin();
    const double n = norm_of<K>(all ? slots : segments, first, count);
    if (threadIdx.x != 0) return;
    if (all) {
        if (norm) *norm = (float)n;
    } else {
        if (each) each[blockIdx.x] = (float)n;
        if (factors) factors[blockIdx.x] = result_of(n, max_norm).c;
    }
}

// The words of what is written; an input that lies otherwise is read element by element, from L1 but for the first of each word (60 M fp32
// scaled 117 us, between addresses that differ 122; packed 71 and 73, bf16 54 and 65; updated 105 and 105, bf16 71 and 73).
template <int TYPE>
__device__ __forceinline__ void scale_lines(const void* from, void* to, int64_t numel, int64_t line, int take, float c) {
    constexpr int kVec = 16 / size_of(TYPE);
    typedef typename Elements<TYPE>::type T;
    typedef Vec<TYPE, kVec> V;
    const int shift = behind_word<TYPE>(to);
    const Range<kVec> range(numel, shift, line, take);
    const T* p = static_cast<const T*>(from) + range.origin;
    T* q = static_cast<T*>(to) + range.origin;
    by_alignment(shift == behind_word<TYPE>(from), [&](auto how) {
        constexpr bool ALIGNED = decltype(how)::value;
        constexpr int kOnce = ALIGNED ? kBatch : kBatch / 2;
        range.template batches<true, kOnce>([&](int at, int low, int high) {
            V x[kOnce];
#pragma unroll
            for (int u = 0; u < kOnce; ++u)
                x[u] = load<TYPE, kVec, ALIGNED>(DRACO_WHOLE(u), p + at + u * 32 * kVec);
#pragma unroll
            for (int u = 0; u < kOnce; ++u) {
                float y[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) y[i] = x[u].value(i) * c;
                x[u].set(y);
                if (DRACO_WHOLE(u)) store<TYPE, kVec, true>(q + at + u * 32 * kVec, x[u]);
            }
        });
    });
    range.ends([&](int i) { q[i] = Elements<TYPE>::round(Elements<TYPE>::value(p[i]) * c); });
}

// to = from * c, c the factor of all or (factors) of each tensor.  In place nothing is written where c is 1.
template <int N>
__device__ __forceinline__ void scale_chunk(const Pointers<N>& from, const Pointers<N>& to, const TensorInfo* infos, const Chunk& chunk, float all,
                                            const float* factors) {
    walk<true, BY_BYTES>(infos, chunk, [&](int t, int type_, int64_t, int64_t numel, int64_t line, int take) {
        const float c = factors ? __ldcg(factors + t) : all;
        if (!from.p[t] || (c == 1.0f && from.p[t] == to.p[t])) return;
        by_type(type_, [&](auto type) { scale_lines<decltype(type)::value>(from.p[t], to.p[t], numel, line, take, c); });
    });
}

__device__ __forceinline__ Chunk chunk_from_the_end(const Chunk* __restrict__ chunks) {
    return chunks[(gridDim.x - 1 - blockIdx.x) * kWarps + (threadIdx.x >> 5)];
}

template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
scale_kernel(const __grid_constant__ Pointers<N> from, const __grid_constant__ Pointers<N> to, const TensorInfo* __restrict__ infos,
             const Chunk* __restrict__ chunks, Limit limit, const float* factors, bool in_place) {
    const Chunk chunk = chunk_from_the_end(chunks);
    pdl_begin();
    const float all = factors ? 1.0f : factor(limit).c;
    if (in_place && !factors && all == 1.0f) return;
    scale_chunk<N>(from, to, infos, chunk, all, factors);
}

// ---- a tensor beside its part of a flat fp32 vector: four elements a lane ----

// Whether groups of four that begin `shift` elements before p are aligned.
template <int TYPE>
__device__ bool fours_at(const void* p, int shift) {
    return ((reinterpret_cast<uintptr_t>(p) - (uintptr_t)shift * size_of(TYPE)) & (4 * size_of(TYPE) - 1)) == 0;
}

// The groups of four are the row's.
template <int TYPE>
__device__ __forceinline__ void pack_lines(const void* base, float* out, int64_t numel, int64_t line, int take, float c) {
    constexpr int kVec = 4;
    typedef typename Elements<TYPE>::type T;
    const int shift = (int)((reinterpret_cast<uintptr_t>(out) >> 2) & 3);
    const Range<kVec> range(numel, shift, line, take);
    const T* p = static_cast<const T*>(base) + range.origin;
    float* q = out + range.origin;
    by_alignment(fours_at<TYPE>(base, shift), [&](auto how) {
        constexpr bool ALIGNED = decltype(how)::value;
        constexpr int kOnce = kBatch;
        range.template batches<true, kOnce>([&](int at, int low, int high) {
            Vec<TYPE, kVec> x[kOnce];
#pragma unroll
            for (int u = 0; u < kOnce; ++u)
                x[u] = load<TYPE, kVec, ALIGNED>(DRACO_WHOLE(u), p + at + u * 32 * kVec);
#pragma unroll
            for (int u = 0; u < kOnce; ++u)
                if (DRACO_WHOLE(u))
                    *reinterpret_cast<float4*>(q + at + u * 32 * kVec) = make_float4(x[u].value(0) * c, x[u].value(1) * c, x[u].value(2) * c, x[u].value(3) * c);
        });
    });
    range.ends([&](int i) { q[i] = Elements<TYPE>::value(p[i]) * c; });
}

// row[flat + i] = c * tensor[i]; zeros for a tensor that is absent.
template <int N>
__device__ __forceinline__ void pack_chunk(const Pointers<N>& list, const TensorInfo* infos, const Chunk& chunk, float* row, float c) {
    walk<true, BY_ELEMENTS>(infos, chunk, [&](int t, int type_, int64_t flat, int64_t numel, int64_t line, int take) {
        if (list.p[t]) {
            by_type(type_, [&](auto type) { pack_lines<decltype(type)::value>(list.p[t], row + flat, numel, line, take, c); });
            return;
        }
        constexpr int kVec = 4;
        const Range<kVec> range(numel, (int)((reinterpret_cast<uintptr_t>(row + flat) >> 2) & 3), line, take);
        float* q = row + flat + range.origin;
        range.template batches<true, kBatch>([&](int at, int low, int high) {
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (DRACO_WHOLE(u)) *reinterpret_cast<float4*>(q + at + u * 32 * kVec) = make_float4(0.f, 0.f, 0.f, 0.f);
        });
        range.ends([&](int i) { q[i] = 0.0f; });
    });
}

template <int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
pack_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const Chunk* __restrict__ chunks, float* row, Limit limit) {
    const Chunk chunk = chunk_from_the_end(chunks);
    pdl_begin();
    pack_chunk<N>(list, infos, chunk, row, factor(limit).c);
}

// The groups of four are those of the side that is both read and written: w, or the master copy of it.
template <int TYPE, bool MASTER>
__device__ __forceinline__ void update_lines(void* base, const float* u, float* master, int64_t flat, int64_t numel, int64_t line, int take, float s) {
    constexpr int kVec = 4, OLD = MASTER ? DRACO_F32 : TYPE;
    typedef typename Elements<TYPE>::type T;
    typedef typename Elements<OLD>::type O;
    const int shift = MASTER ? (int)(flat & 3) : (int)((reinterpret_cast<uintptr_t>(base) / size_of(TYPE)) & 3);
    const Range<kVec> range(numel, shift, line, take);
    T* w = static_cast<T*>(base) + range.origin;
    const float* from = u + flat + range.origin;
    O* o = MASTER ? reinterpret_cast<O*>(master + flat + range.origin) : reinterpret_cast<O*>(w);
    by_alignment(MASTER ? fours_at<TYPE>(base, shift) : ((flat - shift) & 3) == 0, [&](auto how) {
        constexpr bool ALIGNED = decltype(how)::value;     // the other side: u, or w beside its master copy
        constexpr int kOnce = kBatch / 2;                  // two inputs
        range.template batches<true, kOnce>([&](int at, int low, int high) {
            Vec<DRACO_F32, kVec> x[kOnce];
            Vec<OLD, kVec> old[kOnce];
#pragma unroll
            for (int k = 0; k < kOnce; ++k) {
                x[k] = load<DRACO_F32, kVec, MASTER || ALIGNED>(DRACO_WHOLE(k), from + at + k * 32 * kVec);
                old[k] = load<OLD, kVec, true>(DRACO_WHOLE(k), o + at + k * 32 * kVec);
            }
#pragma unroll
            for (int k = 0; k < kOnce; ++k) {
                float now[kVec];
#pragma unroll
                for (int i = 0; i < kVec; ++i) now[i] = fmaf(-s, x[k].value(i), old[k].value(i));
                Vec<TYPE, kVec> y;
                y.set(now);
                if (DRACO_WHOLE(k)) {
                    if (MASTER) *reinterpret_cast<float4*>(o + at + k * 32 * kVec) = make_float4(now[0], now[1], now[2], now[3]);
                    store<TYPE, kVec, !MASTER || ALIGNED>(w + at + k * 32 * kVec, y);
                }
            }
        });
    });
    range.ends([&](int i) {
        const float now = fmaf(-s, from[i], Elements<OLD>::value(o[i]));
        if (MASTER) reinterpret_cast<float*>(o)[i] = now;
        w[i] = Elements<TYPE>::round(now);
    });
}

// w <- w - scale c u; MASTER: the fp32 master copy instead, and w is that, rounded.  Nothing where |u| is not finite.
template <int N, bool MASTER>
__device__ __forceinline__ void update_chunk(const Pointers<N>& list, const TensorInfo* infos, const Chunk& chunk, const float* u, float* master, float scale,
                                             const Result& r) {
    if (!r.finite) return;
    const float s = scale * r.c;
    walk<true, BY_ELEMENTS>(infos, chunk, [&](int t, int type_, int64_t flat, int64_t numel, int64_t line, int take) {
        if (list.p[t]) by_type(type_, [&](auto type) { update_lines<decltype(type)::value, MASTER>(list.p[t], u, master, flat, numel, line, take, s); });
    });
}

template <int N, bool MASTER>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
update_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const Chunk* __restrict__ chunks,
              const float* __restrict__ u, float* __restrict__ master, float scale, Limit limit) {
    const Chunk chunk = chunk_from_the_end(chunks);
    pdl_begin();
    update_chunk<N, MASTER>(list, infos, chunk, u, master, scale, factor(limit));
}

// ---- short lists: measured and worked on by one cluster, in one launch ----

// The blocks of a cluster exchange their sums through shared memory, behind the hardware's barrier; the second pass finds its lines in L1.
struct Small {
    float max_norm;
    float* norm;           // may be null
    float* each;           // may be null
    void* segments;        // null: one factor for all
    float* factors;
};

template <class K>
__device__ __forceinline__ Result cluster_total(typename K::Slot acc, const Small& s) {
    __shared__ typename K::Slot shared[kWarps], mine;
    auto cluster = cooperative_groups::this_cluster();
    acc = block_total<K>(acc, shared);
    if (threadIdx.x == 0) mine = acc;
    cluster.sync();
    typename K::Slot a = K::zero();
    for (int r = 0; r < (int)cluster.num_blocks(); ++r) K::add(a, *cluster.map_shared_rank(&mine, r));
    const double n = K::norm(a);
    if (s.norm && blockIdx.x == 0 && threadIdx.x == 0) *s.norm = (float)n;
    return result_of(n, s.max_norm);
}

// This warp's part of a measurement; with segments the factors of the tensors, too, are in place when it returns.
template <class K, int N>
__device__ __forceinline__ Result measure_small(const Pointers<N>& list, const TensorInfo* infos, const Chunk& chunk, int count, const Small& s) {
    typedef typename K::Slot Slot;
    Slot acc = K::zero();
    const int w = blockIdx.x * kWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
    Slot* segments = static_cast<Slot*>(s.segments);
    walk<false, BY_BYTES>(infos, chunk, [&](int t, int type_, int64_t, int64_t numel, int64_t line, int take) {
        Slot a = K::zero();
        if (list.p[t]) by_type(type_, [&](auto type) { measure_lines<K, decltype(type)::value>(list.p[t], numel, line, take, a); });
        if (segments) {
            const Slot total = warp_total<K>(a);
            if (lane == 0) segments[w + t] = total;
        }
        K::add(acc, a);
    });
    const Result r = cluster_total<K>(acc, s);
    if (!segments) return r;
    for (int t = w; t < count; t += gridDim.x * kWarps) {
        const int first = infos[t].seg_first, n = infos[t].seg_count;
        Slot a = K::zero();
        for (int i = lane; i < n; i += 32) K::add(a, __ldcg(segments + first + i));
        const double norm = K::norm(warp_total<K>(a));
        if (lane == 0) {
            if (s.each) s.each[t] = (float)norm;
            s.factors[t] = result_of(norm, s.max_norm).c;
        }
    }
    cooperative_groups::this_cluster().sync();
    return r;
}

// No block leaves while another may still read its sum.
struct Leave {
    __device__ Leave() { cooperative_groups::this_cluster().barrier_arrive(); }
    __device__ ~Leave() { cooperative_groups::this_cluster().barrier_wait(); }
};

template <class K, int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
small_norm_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const Chunk* __restrict__ chunks, int count, Small s) {
    const Chunk chunk = chunks[blockIdx.x * kWarps + (threadIdx.x >> 5)];
    pdl_begin();
    measure_small<K, N>(list, infos, chunk, count, s);
    const Leave leave;
}

template <class K, int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
small_scale_kernel(const __grid_constant__ Pointers<N> from, const __grid_constant__ Pointers<N> to, const TensorInfo* __restrict__ infos,
                   const Chunk* __restrict__ chunks, const Chunk* __restrict__ second, int count, Small s) {
    const int w = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const Chunk chunk = chunks[w], back = second[w];
    pdl_begin();
    const Result r = measure_small<K, N>(from, infos, chunk, count, s);
    const Leave leave;
    scale_chunk<N>(from, to, infos, back, r.c, s.segments ? s.factors : nullptr);
}

template <class K, int N>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
small_pack_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const Chunk* __restrict__ chunks,
                  const Chunk* __restrict__ second, float* row, Small s) {
    const int w = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const Chunk chunk = chunks[w], back = second[w];
    pdl_begin();
    const Result r = measure_small<K, N>(list, infos, chunk, 0, s);
    const Leave leave;
    pack_chunk<N>(list, infos, back, row, r.c);
}

template <class K, int N, bool MASTER>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm)
small_update_kernel(const __grid_constant__ Pointers<N> list, const TensorInfo* __restrict__ infos, const Chunk* __restrict__ flat,
                    const Chunk* __restrict__ second, const float* __restrict__ u, float* __restrict__ master, float scale, Small s) {
    const int w = blockIdx.x * kWarps + (threadIdx.x >> 5);
    const Chunk chunk = flat[w], back = second[w];
    pdl_begin();
    typename K::Slot acc = K::zero();
    if (chunk.left > 0) measure_lines<K, DRACO_F32>(u, chunk.numel, chunk.at, chunk.left, acc);
    const Result r = cluster_total<K>(acc, s);
    const Leave leave;
    update_chunk<N, MASTER>(list, infos, back, u, master, scale, r);
}

#undef DRACO_WHOLE

}  // namespace
}  // namespace draco

using namespace draco;

// The sizes and types of a list, the split of its lines over warps, and scratch for the partial sums.
struct draco_layout {
    pthread_mutex_t calls;      // held while a call's launches are enqueued: they share the scratch, from the measurement to its last use
    int count, device;
    int64_t size;
    int64_t* numel;             // [count]
    uint8_t* type;              // [count]
    Part* parts;                // [num_parts], then that of the flat vector
    int num_parts;
    int all_blocks;
    int sm_count;
    int small;                  // blocks of the cluster that does all of a call, or 0
    TensorInfo* infos_dev;      // [count], then the flat vector's
    Chunk* chunks_dev;
    void* slots_dev;            // [all_blocks], then [blocks of the flat vector]; 8 bytes each
    void* segments_dev;         // [warps + count]
    float* factors_dev;         // [count]
    Result* result_dev;
    unsigned* ticket_dev;
};

namespace {

struct Calls {
    draco_layout* l;
    explicit Calls(draco_layout* l_) : l(l_) { pthread_mutex_lock(&l->calls); }
    ~Calls() { pthread_mutex_unlock(&l->calls); }
};

void free_layout(draco_layout* l) {
    if (!l) return;
    pthread_mutex_destroy(&l->calls);
    free(l->numel);
    free(l->type);
    free(l->parts);
    if (l->infos_dev) cudaFree(l->infos_dev);
    if (l->chunks_dev) cudaFree(l->chunks_dev);
    if (l->slots_dev) cudaFree(l->slots_dev);
    if (l->segments_dev) cudaFree(l->segments_dev);
    if (l->factors_dev) cudaFree(l->factors_dev);
    if (l->result_dev) cudaFree(l->result_dev);
    if (l->ticket_dev) cudaFree(l->ticket_dev);
    delete l;
}

int64_t lines_of(int64_t numel, int per_lane) {            // the first line begins up to per_lane - 1 elements early
    return numel ? (numel + per_lane - 1 + 32 * per_lane - 1) / (32 * per_lane) : 0;
}

// What a list costs, in lines: a tensor that a warp comes to costs it as much time as kVisit lines, the wait for its first ones.
int64_t cost_of(const TensorInfo* infos, int count, int by) {
    int64_t cost = 0;
    for (int t = 0; t < count; ++t) cost += infos[t].lines[by] ? infos[t].lines[by] + kVisit : 0;
    return cost;
}

// infos[0 .. count - 1] cut into `chunks` chunks of equal cost.
void cut(const TensorInfo* infos, int count, int by, bool down, int chunks, Chunk* table) {
    const int64_t cost = cost_of(infos, count, by);
    const int used = cost < chunks ? (int)cost : chunks;   // the others, the last ones, have none: every chunk between two of a tensor has lines of it
    struct Place {
        int t;
        int64_t before;                                    // cost of the tensors before t
        int64_t line;                                      // in t
    } begin = {0, 0, 0};
    auto next = [&](Place p, int64_t at) {
        auto of = [&](int t) { return infos[t].lines[by] ? infos[t].lines[by] + kVisit : 0; };
        while (p.t < count - 1 && at >= p.before + of(p.t)) p.before += of(p.t++);
        p.line = at - p.before - kVisit;
        if (p.line < 0) p.line = 0;
        if (p.line > infos[p.t].lines[by]) p.line = infos[p.t].lines[by];
        return p;
    };
    begin = next(begin, 0);
    for (int c = 0; c < chunks; ++c) {
        const Place end = next(begin, c + 1 < used ? cost / used * (c + 1) + cost % used * (c + 1) / used : cost);
        int64_t left = end.line - begin.line;
        for (int t = begin.t; t < end.t; ++t) left += infos[t].lines[by];
        Place from = begin;
        if (down) {                                        // the tensor that holds the last line
            from = end;
            while (from.line == 0 && from.t > begin.t) from.line = infos[--from.t].lines[by];
        }
        table[c] = {from.line, infos[from.t].numel, infos[from.t].flat, infos[from.t].lines[by], (int32_t)left, from.t, infos[from.t].type, 0};
        begin = end;
    }
}

// The segments of infos[0 .. count - 1] by the chunks of the measurement: that of chunk w and tensor t is number w + t.
void number_segments(TensorInfo* infos, int count, const Chunk* table, int chunks) {
    for (int w = 0; w < chunks; ++w) {
        int64_t left = table[w].left, at = table[w].at;
        for (int t = table[w].tensor; left > 0; ++t, at = 0) {
            const int64_t take = left < infos[t].lines[BY_BYTES] - at ? left : infos[t].lines[BY_BYTES] - at;
            if (take <= 0) continue;
            if (!infos[t].seg_count++) infos[t].seg_first = w + t;
            left -= take;
        }
    }
}

// Blocks of a list of this cost, a chunk a warp.
int blocks_of(int64_t cost, int what, int sm_count, int small) {
    if (small) return small;
    auto blocks = [&](int64_t per, int64_t most) {
        const int64_t wanted = (cost + kWarps * per - 1) / (kWarps * per);
        return (int)(wanted < 1 ? 1 : wanted < most ? wanted : most);
    };
    const int64_t wave = (int64_t)sm_count * kBlocksPerSm;
    const int64_t a_warp = cost / (wave * kWarps);
    if (what == MEASURE || what == IN_PLACE || a_warp < kWaveLines) return blocks(kMinLines, wave);
    return blocks(kWavesLines, wave * kWaves);
}

template <class F>
int with_capacity(int count, F f) {
    if (count <= 64) return f(std::integral_constant<int, 64>());
    if (count <= 512) return f(std::integral_constant<int, 512>());
    return f(std::integral_constant<int, kMaxPointers>());
}

template <class F>
int with_kind(int kind, F f) {
    return kind == DRACO_NORM_2 ? f(SumSquares()) : f(MaxMagnitude());
}

template <int N>
Pointers<N> pointers_of(const void* const* list, int count) {
    Pointers<N> p;
    for (int t = 0; t < count; ++t) p.p[t] = const_cast<void*>(list[t]);
    return p;
}

// Whether every block of the second pass may form the factor for itself: one wave of them in each launch, and no more sums than one wave leaves.  us, formed
// by all / once: 2000 tensors of 104 bf16 elements and then 60 M packed, most of it by 7300 blocks, 92.8, 85.9; 65,536 tensors of 64, below the limit, clipped in place
// by 33 launches 249, 131.
bool formed_by_all(const draco_layout* l, int what, int sums) {
    const int wave = l->sm_count * kBlocksPerSm;
    for (int k = 0; k < l->num_parts; ++k)
        if (l->parts[k].blocks[what] > wave) return false;
    return sums <= wave;
}

// The sums of a list, or of the flat vector u (list null).  segments: of each tensor too.  limit: null (the norm is all that is wanted), or where
// the second pass, by the table `what`, gets the factor from.
int measure(draco_layout* l, const void* const* list, const float* u, int kind, float max_norm, bool segments, float* norm, Limit* limit, int what,
            cudaStream_t st) {
    const void* flat[1] = {u};
    const int blocks = list ? l->all_blocks : l->parts[l->num_parts].blocks[MEASURE];
    const bool finish = (!limit || !formed_by_all(l, what, blocks)) && !segments;
    if (limit) *limit = {finish ? l->result_dev : nullptr, static_cast<char*>(l->slots_dev) + (list ? 0 : (size_t)l->all_blocks * 8), blocks, kind, max_norm, norm};
    const int launches = list ? l->num_parts : 1;
    for (int k = 0; k < launches; ++k) {
        const Part& part = l->parts[list ? k : l->num_parts];
        const int block0 = list ? part.block0 : 0;
        char* slots = static_cast<char*>(l->slots_dev) + (list ? 0 : (size_t)l->all_blocks * 8);
        char* segs = static_cast<char*>(l->segments_dev) + 8 * ((size_t)part.block0 * kWarps + part.first);
        const int rc = with_capacity(part.count, [&](auto n) -> int {
            constexpr int N = decltype(n)::value;
            const Pointers<N> p = pointers_of<N>(list ? list + part.first : flat, part.count);
            return with_kind(kind, [&](auto how) -> int {
                typedef decltype(how) K;
                typedef typename K::Slot* S;
                const auto kernel = segments ? measure_kernel<K, N, true> : measure_kernel<K, N, false>;
                DRACO_CUDA(launch_dependent(kernel, dim3(part.blocks[MEASURE]), dim3(kThreads), 0, st, p, (const TensorInfo*)l->infos_dev + part.first,
                                            (const Chunk*)l->chunks_dev + part.table[MEASURE], (S)slots, block0, blocks, l->ticket_dev, (S)segs,
                                            finish && k == launches - 1, max_norm, norm, limit ? l->result_dev : nullptr));
                return DRACO_OK;
            });
        });
        if (rc != DRACO_OK) return rc;
    }
    return DRACO_OK;
}

int finish_each(draco_layout* l, int kind, float max_norm, float* norm, float* each, float* factors, cudaStream_t st) {
    return with_kind(kind, [&](auto what) -> int {
        typedef decltype(what) K;
        typedef const typename K::Slot* S;
        DRACO_CUDA(launch_dependent(each_kernel<K>, dim3(l->count + 1), dim3(kThreads), 0, st, (const TensorInfo*)l->infos_dev, (S)l->segments_dev,
                                    (S)l->slots_dev, l->all_blocks, max_norm, norm, each, factors));
        return DRACO_OK;
    });
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
    while (size < 2 * l->count) size *= 2;                 // at most half full: `from` is only looked up
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

template <class F>
int with_small_capacity(int count, F f) {
    if (count <= 64) return f(std::integral_constant<int, 64>());
    return f(std::integral_constant<int, kSmallTensors>());
}

// launch_dependent with all blocks in one cluster.
template <typename... Params, typename... Args>
int launch_small(const draco_layout* l, void (*kernel)(Params...), cudaStream_t st, Args... args) {
    cudaLaunchAttribute attrs[2] = {};
    attrs[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[0].val.programmaticStreamSerializationAllowed = 1;
    attrs[1].id = cudaLaunchAttributeClusterDimension;
    attrs[1].val.clusterDim.x = l->small;
    attrs[1].val.clusterDim.y = attrs[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(l->small);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = st;
    cfg.attrs = attrs;
    cfg.numAttrs = 2;
    DRACO_CUDA(cudaLaunchKernelEx(&cfg, kernel, static_cast<Params>(args)...));
    return DRACO_OK;
}

constexpr int kPortable = 8;                               // blocks of a cluster that every device takes

// Larger clusters have to be allowed, kernel by kernel and device by device.
template <class K, int N>
cudaError_t allow_large_clusters() {
    const void* kernels[] = {(const void*)small_norm_kernel<K, N>, (const void*)small_scale_kernel<K, N>, (const void*)small_pack_kernel<K, N>,
                             (const void*)small_update_kernel<K, N, false>, (const void*)small_update_kernel<K, N, true>};
    for (const void* k : kernels) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

bool large_cluster_fits(int count, int blocks) {
    return with_small_capacity(count, [&](auto n) -> int {
        constexpr int N = decltype(n)::value;
        if (allow_large_clusters<SumSquares, N>() != cudaSuccess || allow_large_clusters<MaxMagnitude, N>() != cudaSuccess) {
            cudaGetLastError();
            return 0;
        }
        cudaLaunchAttribute attr = {};
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = blocks;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(blocks);
        cfg.blockDim = dim3(kThreads);
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        int clusters = 0;
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&clusters, small_scale_kernel<SumSquares, N>, &cfg);
        if (e != cudaSuccess) cudaGetLastError();
        return e == cudaSuccess && clusters > 0;
    });
}

const Chunk* table_of(const draco_layout* l, int what) { return l->chunks_dev + l->parts[0].table[what]; }

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
        if (numel[t] < 0) return DRACO_EINVAL;
        if (type[t] != DRACO_F32 && type[t] != DRACO_BF16 && type[t] != DRACO_F16) return DRACO_EINVAL;
        if (numel[t] > kMostElements - size) return DRACO_ELIMIT;
        size += numel[t];
    }
    draco_layout* l = new (std::nothrow) draco_layout();
    if (!l) return DRACO_ENOMEM;
    memset(l, 0, sizeof(*l));
    pthread_mutex_init(&l->calls, nullptr);
    l->count = count;
    l->size = size;
    l->num_parts = (count + kMaxPointers - 1) / kMaxPointers;
    cudaError_t err = cudaGetDevice(&l->device);
    if (err == cudaSuccess) err = cudaDeviceGetAttribute(&l->sm_count, cudaDevAttrMultiProcessorCount, l->device);
    if (err != cudaSuccess) { free_layout(l); return cuda_fail(err, "cudaGetDevice"); }
    l->numel = static_cast<int64_t*>(malloc(sizeof(int64_t) * count));
    l->type = static_cast<uint8_t*>(malloc(count));
    l->parts = static_cast<Part*>(calloc(l->num_parts + 1, sizeof(Part)));
    TensorInfo* infos = static_cast<TensorInfo*>(calloc(count + 1, sizeof(TensorInfo)));
    Chunk* chunks = nullptr;
    int64_t num_chunks = 0;
    int rc = DRACO_OK;
    if (!l->numel || !l->type || !l->parts || !infos) rc = DRACO_ENOMEM;
    if (rc == DRACO_OK) {
        int64_t flat = 0;
        for (int t = 0; t <= count; ++t) {                 // the last: the flat vector
            TensorInfo& i = infos[t];
            i.numel = t < count ? numel[t] : size;
            i.type = t < count ? type[t] : DRACO_F32;
            i.flat = t < count ? flat : 0;
            i.lines[BY_BYTES] = lines_of(i.numel, 16 / size_of(i.type));
            i.lines[BY_ELEMENTS] = lines_of(i.numel, 4);
            if (t == count) break;
            l->numel[t] = i.numel;
            l->type[t] = (uint8_t)i.type;
            flat += i.numel;
        }
        const int64_t alone = cost_of(infos, count, BY_BYTES), beside = cost_of(infos, count, BY_ELEMENTS), most = alone > beside ? alone : beside;
        if (count <= kSmallTensors && most <= kSmallBlocks * kWarps * kSmallLines) {
            const int64_t wanted = (most + kWarps * kMinLines - 1) / (kWarps * kMinLines);
            l->small = (int)(wanted < 1 ? 1 : wanted < kSmallBlocks ? wanted : kSmallBlocks);
            if (l->small > kPortable && !large_cluster_fits(count, l->small)) l->small = kPortable;
        }
        for (int k = 0; k <= l->num_parts; ++k) {
            Part& p = l->parts[k];
            const bool list = k < l->num_parts;
            p.first = list ? k * kMaxPointers : count;
            p.count = list ? (count - p.first < kMaxPointers ? count - p.first : kMaxPointers) : 1;
            p.block0 = l->all_blocks;
            for (int what = MEASURE; what <= (list ? ELEMENTS : MEASURE); ++what) {
                p.blocks[what] = blocks_of(cost_of(infos + p.first, p.count, what == ELEMENTS ? BY_ELEMENTS : BY_BYTES), what, l->sm_count, l->small);
                p.table[what] = num_chunks;
                num_chunks += p.blocks[what] * kWarps;
            }
            if (list) l->all_blocks += p.blocks[MEASURE];
        }
        chunks = static_cast<Chunk*>(malloc(sizeof(Chunk) * num_chunks));
        if (!chunks) rc = DRACO_ENOMEM;
    }
    for (int k = 0; k <= l->num_parts && rc == DRACO_OK; ++k) {
        const Part& p = l->parts[k];
        TensorInfo* mine = infos + p.first;
        for (int what = MEASURE; what <= (k < l->num_parts ? ELEMENTS : MEASURE); ++what)
            cut(mine, p.count, what == ELEMENTS ? BY_ELEMENTS : BY_BYTES, what != MEASURE, p.blocks[what] * kWarps, chunks + p.table[what]);
        if (k == l->num_parts) break;
        number_segments(mine, p.count, chunks + p.table[MEASURE], p.blocks[MEASURE] * kWarps);
        for (int t = 0; t < p.count; ++t) mine[t].seg_first += p.block0 * kWarps + p.first;
    }
#define DRACO_TRY(call)                                                                          \
    do {                                                                                         \
        if (rc == DRACO_OK) {                                                                    \
            cudaError_t e__ = (call);                                                            \
            if (e__ != cudaSuccess) rc = cuda_fail(e__, #call);                                  \
        }                                                                                        \
    } while (0)
    const size_t slots = rc == DRACO_OK ? (size_t)l->all_blocks + l->parts[l->num_parts].blocks[MEASURE] : 0;
    DRACO_TRY(cudaMalloc(&l->infos_dev, sizeof(TensorInfo) * (count + 1)));
    DRACO_TRY(cudaMalloc(&l->chunks_dev, sizeof(Chunk) * num_chunks));
    DRACO_TRY(cudaMalloc(&l->slots_dev, 8 * slots));
    DRACO_TRY(cudaMalloc(&l->segments_dev, 8 * (slots * kWarps + count + 1)));
    DRACO_TRY(cudaMalloc(&l->factors_dev, sizeof(float) * count));
    DRACO_TRY(cudaMalloc(&l->result_dev, sizeof(Result)));
    DRACO_TRY(cudaMalloc(&l->ticket_dev, sizeof(unsigned)));
    DRACO_TRY(cudaMemset(l->ticket_dev, 0, sizeof(unsigned)));
    DRACO_TRY(cudaMemcpy(l->infos_dev, infos, sizeof(TensorInfo) * (count + 1), cudaMemcpyHostToDevice));
    DRACO_TRY(cudaMemcpy(l->chunks_dev, chunks, sizeof(Chunk) * num_chunks, cudaMemcpyHostToDevice));
    DRACO_TRY(cudaStreamSynchronize(nullptr));
#undef DRACO_TRY
    free(infos);
    free(chunks);
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
    const Calls one_at_a_time(layout);
    if (layout->small)
        return with_small_capacity(layout->count, [&](auto n) {
            return with_kind(kind, [&](auto k) {
                constexpr int N = decltype(n)::value;
                const Small s = {INFINITY, norm, each, each ? layout->segments_dev : nullptr, layout->factors_dev};
                return launch_small(layout, small_norm_kernel<decltype(k), N>, st, pointers_of<N>(tensors, layout->count), layout->infos_dev,
                                    table_of(layout, MEASURE), layout->count, s);
            });
        });
    const int rc = measure(layout, tensors, nullptr, kind, INFINITY, each != nullptr, norm, nullptr, 0, st);
    if (rc != DRACO_OK || !each) return rc;
    return finish_each(layout, kind, INFINITY, norm, each, nullptr, st);
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
    const Calls one_at_a_time(layout);
    const int table = out ? BYTES : IN_PLACE;
    if (layout->small)
        return with_small_capacity(layout->count, [&](auto n) {
            return with_kind(kind, [&](auto k) {
                constexpr int N = decltype(n)::value;
                const Small s = {max_norm, norm, each, separately ? layout->segments_dev : nullptr, layout->factors_dev};
                return launch_small(layout, small_scale_kernel<decltype(k), N>, st, pointers_of<N>(tensors, layout->count),
                                    pointers_of<N>(to, layout->count), layout->infos_dev, table_of(layout, MEASURE), table_of(layout, table), layout->count, s);
            });
        });
    Limit limit = {};
    int rc = measure(layout, tensors, nullptr, kind, max_norm, separately != 0, norm, &limit, table, st);
    if (rc == DRACO_OK && separately) rc = finish_each(layout, kind, max_norm, norm, each, layout->factors_dev, st);
    for (int k = 0; k < layout->num_parts && rc == DRACO_OK; ++k) {
        const Part& part = layout->parts[k];
        rc = with_capacity(part.count, [&](auto n) -> int {
            constexpr int N = decltype(n)::value;
            DRACO_CUDA(launch_dependent(scale_kernel<N>, dim3(part.blocks[table]), dim3(kThreads), 0, st,
                                        pointers_of<N>(tensors + part.first, part.count), pointers_of<N>(to + part.first, part.count),
                                        (const TensorInfo*)layout->infos_dev + part.first, (const Chunk*)layout->chunks_dev + part.table[table], limit,
                                        separately ? (const float*)layout->factors_dev + part.first : nullptr, !out));
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
    const Calls one_at_a_time(layout);
    const bool wanted = norm || !isinf(max_norm);
    if (layout->small && wanted)
        return with_small_capacity(layout->count, [&](auto n) {
            return with_kind(kind, [&](auto k) {
                constexpr int N = decltype(n)::value;
                return launch_small(layout, small_pack_kernel<decltype(k), N>, st, pointers_of<N>(tensors, layout->count), layout->infos_dev,
                                    table_of(layout, MEASURE), table_of(layout, ELEMENTS), row, Small{max_norm, norm, nullptr, nullptr, nullptr});
            });
        });
    Limit limit = {};
    int rc = wanted ? measure(layout, tensors, nullptr, kind, max_norm, false, norm, &limit, ELEMENTS, st) : (int)DRACO_OK;
    for (int k = 0; k < layout->num_parts && rc == DRACO_OK; ++k) {
        const Part& part = layout->parts[k];
        rc = with_capacity(part.count, [&](auto n) -> int {
            constexpr int N = decltype(n)::value;
            DRACO_CUDA(launch_dependent(pack_kernel<N>, dim3(part.blocks[ELEMENTS]), dim3(kThreads), 0, st, pointers_of<N>(tensors + part.first, part.count),
                                        (const TensorInfo*)layout->infos_dev + part.first, (const Chunk*)layout->chunks_dev + part.table[ELEMENTS], row,
                                        limit));
            return DRACO_OK;
        });
    }
    return rc;
}

int draco_update(draco_layout* layout, void* const* params, const float* u, float* master, int kind, float max_norm, float scale, float* norm, void* stream) {
    if (!layout || !addresses_ok(layout, params) || !kind_ok(kind) || !(max_norm >= 0.0f) || !(scale == scale) || (!u && layout->size) ||
        !aligned16(u) || !aligned16(master) || !aligned4(norm) || !on_device(layout))
        return DRACO_EINVAL;
    const int64_t bytes = 4 * layout->size;
    const uintptr_t x = reinterpret_cast<uintptr_t>(u), y = reinterpret_cast<uintptr_t>(master);
    if (!apart(layout, params, u, bytes) || (master && (!apart(layout, params, master, bytes) || (x < y + bytes && y < x + bytes)))) return DRACO_EINVAL;
    const int alone = distinct(layout, params, params);
    if (alone <= 0) return alone < 0 ? alone : DRACO_EINVAL;
    cudaStream_t st = (cudaStream_t)stream;
    const Calls one_at_a_time(layout);
    const bool wanted = norm || !isinf(max_norm);
    if (layout->small && wanted)
        return with_small_capacity(layout->count, [&](auto n) {
            return with_kind(kind, [&](auto k) -> int {
                constexpr int N = decltype(n)::value;
                auto go = [&](auto kernel) {
                    return launch_small(layout, kernel, st, pointers_of<N>(params, layout->count), layout->infos_dev,
                                        layout->chunks_dev + layout->parts[layout->num_parts].table[MEASURE], table_of(layout, ELEMENTS), u, master, scale,
                                        Small{max_norm, norm, nullptr, nullptr, nullptr});
                };
                return master ? go(small_update_kernel<decltype(k), N, true>) : go(small_update_kernel<decltype(k), N, false>);
            });
        });
    Limit limit = {};
    int rc = wanted ? measure(layout, nullptr, u, kind, max_norm, false, norm, &limit, ELEMENTS, st) : (int)DRACO_OK;
    for (int k = 0; k < layout->num_parts && rc == DRACO_OK; ++k) {
        const Part& part = layout->parts[k];
        rc = with_capacity(part.count, [&](auto n) -> int {
            constexpr int N = decltype(n)::value;
            auto go = [&](auto kernel) -> int {
                DRACO_CUDA(launch_dependent(kernel, dim3(part.blocks[ELEMENTS]), dim3(kThreads), 0, st, pointers_of<N>(params + part.first, part.count),
                                            (const TensorInfo*)layout->infos_dev + part.first, (const Chunk*)layout->chunks_dev + part.table[ELEMENTS], u,
                                            master, scale, limit));
                return DRACO_OK;
            };
            return master ? go(update_kernel<N, true>) : go(update_kernel<N, false>);
        });
    }
    return rc;
}

}  // extern "C"
