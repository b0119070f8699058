// Routing to experts: a token's scores, the experts it is sent to and their weights; the order in which the experts' products
// take the rows; the gradient of the weights with respect to the logits; and the weighted sum of the experts' results.
//
//   s_e = softmax(z)_e or 1 / (1 + e^-z_e)         over the experts that are open to the token (z neither -inf nor NaN)
//   key = z_e, or fl32(s_e + b_e) with a balance bias b      (both scores grow with z)
//   groups of neighbouring experts: those with the best keys (or sums of the two best scores) stay
//   the k largest keys, ties to the lower expert;  w_j = scale s_j [/ sum of the chosen scores]
//
// A group of LPT lanes owns a token, expert e in lane e % LPT, so that a wave of 16-lane groups chooses for four tokens at once.
// Keys are compared as integers that order like the floats; 0 is "closed" or "already taken".  Each of the k rounds is a scan of the
// lane's own keys and two reductions over the group (largest key, lowest expert that has it) in DPP steps.
// Long batches are bound by the vector ALU: 16384 tokens, 256 experts, sigmoid and bias, 8 of 4 groups of 8: 17.8 us (5 more with the keys of
// all groups in every round and the groups read in step, from the same banks), half the time with k = 1; 17 MB would take 3.3.  Short ones
// by latency: 331 tokens 7.1 us.  The order of the rows is a second launch (5 to 9 us), whose blocks each need the counts of all.
#include "ssg_device.h"
#include "ssg_internal.h"

namespace ssg {

namespace {

constexpr int kOneLaunch = 16;                            // tokens that one block chooses for and sorts
constexpr int kBlock = 1024;                              // threads of a block that sorts, and the most of one that chooses
constexpr int kLeast = 256;                               // the fewest of one that chooses
constexpr int kWaves = kBlock / 64;

// float -> integer in the same order; -0 counts as +0
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t u = __float_as_uint(v + 0.0f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t u) { return __uint_as_float(u ^ ((u >> 31) ? 0x80000000u : 0xffffffffu)); }

// Lane exchanges inside groups of 16: neighbours, pairs, then mirrored halves (which are uniform by then).
template <int STEP> __device__ __forceinline__ uint32_t exchange(uint32_t v) {
    constexpr int ctrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, ctrl, 0xf, 0xf, false);
}
// Every lane of the group gets op over the group, in the same order of operations in every lane's value.
template <int LPT, class Op> __device__ __forceinline__ uint32_t reduce(uint32_t v, Op op) {
    v = op(v, exchange<0>(v));
    v = op(v, exchange<1>(v));
    v = op(v, exchange<2>(v));
    v = op(v, exchange<3>(v));
    if (LPT == 64) {
        // both operands the same: the even rows (the lower half) in one result and the odd ones (the upper half) in the other
        const auto rows = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = op(rows[0], rows[1]);
        const auto halves = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = op(halves[0], halves[1]);
    }
    return v;
}
template <int LPT> __device__ __forceinline__ uint32_t reduce_max(uint32_t v) {
    return reduce<LPT>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
template <int LPT> __device__ __forceinline__ uint32_t reduce_min(uint32_t v) {
    return reduce<LPT>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
template <int LPT> __device__ __forceinline__ float reduce_sum(float v) {
    return __uint_as_float(reduce<LPT>(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

template <bool BF16> __device__ __forceinline__ float load_logit(const void *p, int64_t at) {
    return BF16 ? bf16_bits_to_f32(static_cast<const uint16_t *>(p)[at]) : static_cast<const float *>(p)[at];
}
__device__ __forceinline__ bool is_open(float z) { return z > -INFINITY; }            // false for NaN
__device__ __forceinline__ float held(float z) { return fminf(z, 3.402823466e+38f); } // +inf: the largest finite number

// The sigmoid of every logit: sigmoid_f32 stays at e^-88 below -88; where 1 + e^z is 1 to 35 digits this is e^z itself, down to the smallest number.
__device__ __forceinline__ float score_sigmoid(float z) {
    float s = sigmoid_f32(z);
    if (__builtin_expect(z < -80.0f, 0)) s = expf(z);
    return s;
}

constexpr float kTiny = 1e-38f;                           // what a sum of scores is held above where it divides (without any it is 0)

// Renormalised weights need the chosen scores up to a common factor, which is taken so that their sum neither underflows nor loses bits:
// softmax scores beside the largest chosen logit, and so sigmoids where that is below this, which are e^z to 2e-9.
constexpr float kLowSigmoid = -20.0f;

// The k largest keys of the group's lanes, key i of lane l in slot l + i LPT: lane j returns the slot of the j-th, -1 if there is none.
template <int LPT, int VPL> __device__ __forceinline__ int pick(uint32_t (&key)[VPL], int k) {
    const int g0 = threadIdx.x & (LPT - 1);
    int slot = -1;
    for (int j = 0; j < k; ++j) {
        uint32_t best = 0, e = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (key[i] > best) { best = key[i]; e = (uint32_t)(g0 + i * LPT); }
        const uint32_t all = reduce_max<LPT>(best);
        e = reduce_min<LPT>(best == all ? e : 0xffffffffu);
        if (all == 0) e = 0xffffffffu;
        if (g0 == j) slot = (int)e;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
            if (e == (uint32_t)(g0 + i * LPT)) key[i] = 0;
    }
    return slot;
}

// The experts of token t: lane j of the group returns the j-th (or -1) in id, its weight in w.  `keys`: a.key_stride words of LDS of the
// group's own (used with groups only).  All lanes of a wave come here together; `live` says whether the group has a token.
template <int LPT, int VPL, bool BF16>
__device__ __forceinline__ void choose(const RouteArgs &a, int64_t t, bool live, uint32_t *keys, int &id, float &w) {
    const int g0 = threadIdx.x & (LPT - 1);
    const bool softmax = a.score == 0, biased = a.bias != nullptr, grouped = a.top_groups < a.groups;
    float z[VPL];
    uint32_t key[VPL];
    const int64_t row = t * a.ld;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = g0 + i * LPT;
        z[i] = live && e < a.E ? load_logit<BF16>(a.logits, row + e) : -INFINITY;
    }
    // softmax: largest logit and sum of exponentials over the open experts
    float top = 0.0f, sum = 0.0f;
    if (softmax) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const uint32_t u = is_open(z[i]) ? ordered(held(z[i])) : 0u;
            m = m > u ? m : u;
        }
        m = reduce_max<LPT>(m);
        top = m ? from_ordered(m) : 0.0f;
        if (biased || !a.renorm || (grouped && a.group_top == 2)) {
#pragma unroll
            for (int i = 0; i < VPL; ++i) sum += is_open(z[i]) ? expf(held(z[i]) - top) : 0.0f;
            sum = fmaxf(reduce_sum<LPT>(sum), kTiny);
        }
    }
    auto score = [&](float v) { return softmax ? expf(held(v) - top) / sum : score_sigmoid(held(v)); };
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
        const int e = g0 + i * LPT;
        float v = z[i];
        if (biased && is_open(v)) v = score(v) + a.bias[e];
        key[i] = is_open(v) ? ordered(held(v)) : 0u;
    }
    if (grouped) {
        // L lanes to a group of experts; the two best of each, then the group's rank among the others
        const int size = a.E / a.groups;
        int L = 1;
        while (2 * L * a.groups <= LPT) L *= 2;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int e = g0 + i * LPT;
            if (e < a.E) keys[e] = a.group_top == 2 && !biased && key[i] ? ordered(score(z[i])) : key[i];
        }
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
        const int group = g0 / L, sub = g0 % L, count = (size + L - 1) / L;
        uint32_t first = 0, second = 0;
        if (group < a.groups) {
            // (each group from another place on, since those of the same size begin in the same bank)
            int n = group % count;
#pragma unroll 4
            for (int i = 0; i < count; ++i) {
                const int x = sub + n * L;
                const uint32_t u = x < size ? keys[group * size + x] : 0;
                second = u > first ? first : (u > second ? u : second);
                first = u > first ? u : first;
                n = n + 1 == count ? 0 : n + 1;
            }
        }
        for (int step = 1; step < L; step *= 2) {
            const uint32_t f = (uint32_t)__shfl_xor((int)first, step, 64), s = (uint32_t)__shfl_xor((int)second, step, 64);
            const uint32_t low = f > first ? first : f;
            first = f > first ? f : first;
            second = second > s ? second : s;
            second = second > low ? second : low;
        }
        uint32_t mine = first;
        if (a.group_top == 2 && first && second) mine = ordered(from_ordered(first) + from_ordered(second));
        int ahead = 0;
        const int lane0 = (threadIdx.x & 63) - g0;
#pragma unroll 4
        for (int g = 0; g < a.groups; ++g) {
            const uint32_t other = (uint32_t)__shfl((int)mine, lane0 + g * L, 64);
            ahead += other > mine || (other == mine && g < group);
        }
        // The experts of the groups that stay, in their order, are what is chosen from: slot s is number s % size of the group that
        // is number s / size among them.
        const bool stays = group < a.groups && sub == 0 && ahead < a.top_groups;
        const uint64_t kept = __ballot(stays) >> lane0;
        uint32_t *starts = keys + a.E;
        if (stays) starts[__popcll(kept & ((1ull << g0) - 1))] = (uint32_t)(group * size);
        if (a.group_top == 2 && !biased) {                 // (by their scores until now)
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (g0 + i * LPT < a.E) keys[g0 + i * LPT] = key[i];
        }
        __builtin_amdgcn_wave_barrier();
        __threadfence_block();
        const int slots = a.top_groups * size;
        const uint32_t inv = ((1u << 20) + size - 1) / size;          // s * inv >> 20 = s / size for s, size up to 1024
        auto expert = [&](int s) {
            const uint32_t nth = (uint32_t)s * inv >> 20;
            return starts[nth] + (uint32_t)s - nth * size;
        };
        auto pick_kept = [&](auto values) {
            uint32_t k2[decltype(values)::value];
#pragma unroll
            for (int i = 0; i < decltype(values)::value; ++i) {
                const int s = g0 + i * LPT;
                k2[i] = live && s < slots ? keys[expert(s)] : 0u;
            }
            return pick<LPT>(k2, a.k);
        };
        constexpr int kHalf = VPL > 1 ? VPL / 2 : 1;
        id = slots <= kHalf * LPT ? pick_kept(std::integral_constant<int, kHalf>{}) : pick_kept(std::integral_constant<int, VPL>{});
        if (id >= 0) id = (int)expert(id);
        __builtin_amdgcn_wave_barrier();
    } else {
        id = pick<LPT>(key, a.k);
    }
    w = 0.0f;
    const float v = id >= 0 ? held(load_logit<BF16>(a.logits, row + id)) : 0.0f;
    bool beside_best = false;
    if (a.renorm) {
        const uint32_t m = reduce_max<LPT>(id >= 0 ? ordered(v) : 0u);
        if (m) top = from_ordered(m);
        beside_best = softmax || (m && top < kLowSigmoid);
    }
    if (id >= 0) {
        if (beside_best) w = expf(v - top);
        else w = softmax ? expf(v - top) / sum : score_sigmoid(v);
    }
    if (a.renorm) w = w / fmaxf(reduce_sum<LPT>(w), kTiny);
    w = w * a.scale;
}

// What a block of the sort needs in LDS: the experts' totals, rows before this block's, offsets, and the running counts.
struct SortLds {
    uint32_t *total, *before, *offset, *wave_count;       // E, E, E + 1, kWaves * E words
};

// Exclusive prefix over up to 1024 experts of their rows, rounded up to the alignment; offset[E] = all rows.
__device__ __forceinline__ void scan_offsets(const RouteArgs &a, const SortLds &s, uint32_t *wave_sum) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    uint32_t v = 0;
    if (tid < a.E) v = (s.total[tid] + a.align - 1) / a.align * a.align;
    uint32_t inc = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = (uint32_t)__shfl_up((int)inc, d, 64);
        if (lane >= d) inc += o;
    }
    if (lane == 63) wave_sum[wv] = inc;
    __syncthreads();
    uint32_t base = 0;
    for (int i = 0; i < wv; ++i) base += wave_sum[i];
    if (tid < a.E) {
        s.offset[tid] = base + inc - v;
        if (tid == a.E - 1) s.offset[a.E] = base + inc;
    }
    __syncthreads();
}

// The rows of assignments [first, last), in their order, behind `before` others of the same expert; and this block's share of
// what no assignment fills.
__device__ __forceinline__ void scatter(const RouteArgs &a, const SortLds &s, int64_t first, int64_t last, int block, int blocks) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    int bits = 0;
    while ((1 << bits) < a.E) ++bits;
    for (int64_t base = first; base < last; base += kBlock) {
        for (int i = tid; i < kWaves * a.E; i += kBlock) s.wave_count[i] = 0;
        __syncthreads();
        const int64_t at = base + tid;
        const int e = at < last ? a.ids[at] : -1;
        // lanes of this wave with the same expert
        uint64_t same = __ballot(e >= 0);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((e >> b) & 1);
            same &= (e >> b) & 1 ? set : ~set;
        }
        const int rank = __popcll(same & ((1ull << lane) - 1));
        if (e >= 0 && rank == 0) s.wave_count[wv * a.E + e] = (uint32_t)__popcll(same);
        __syncthreads();
        if (e >= 0) {
            uint32_t row = s.offset[e] + s.before[e] + rank;
            for (int i = 0; i < wv; ++i) row += s.wave_count[i * a.E + e];
            a.place[at] = (int)row;
            a.source[row] = (int)at;
        } else if (at < last) {
            a.place[at] = -1;
        }
        if (base + kBlock >= last) break;
        __syncthreads();
        for (int x = tid; x < a.E; x += kBlock) {
            uint32_t n = 0;
            for (int i = 0; i < kWaves; ++i) n += s.wave_count[i * a.E + x];
            s.before[x] += n;
        }
        __syncthreads();
    }
    // rows that fill up an expert's last set (fewer than the alignment; all experts' side by side, since one after the other 256 of them
    // took 23 us), and those beyond all experts
    for (int i = block * kBlock + tid; i < a.E * a.align; i += blocks * kBlock) {
        const int e = i / a.align;
        const uint32_t r = s.offset[e] + s.total[e] + (uint32_t)(i % a.align);
        if (r < s.offset[e + 1]) a.source[r] = -1;
    }
    for (int64_t r = s.offset[a.E] + (int64_t)block * kBlock + tid; r < a.rows; r += (int64_t)blocks * kBlock) a.source[r] = -1;
    if (block == 0)
        for (int e = tid; e <= a.E; e += kBlock) {
            a.offsets[e] = (int)s.offset[e];
            if (e < a.E) a.counts[e] = (int)s.total[e];
        }
}

__device__ __forceinline__ SortLds sort_lds(uint32_t *lds, int E) { return SortLds{lds, lds + E, lds + 2 * E, lds + 3 * E + 1}; }

// Counts of a block: at most its tokens, since a token takes an expert once; 16 bits each, rows of 16 bytes.
__host__ __device__ constexpr int hist_stride(int E) { return (E + 7) & ~7; }

// One block per a.block_tokens tokens.  With one block in all it sorts too (and has kBlock threads); otherwise it leaves its experts' counts.
template <int LPT, int VPL, bool BF16> __global__ __launch_bounds__(kBlock) void route_kernel(RouteArgs a) {
    extern __shared__ uint32_t lds[];
    __shared__ uint32_t wave_sum[kWaves];
    const int tid = threadIdx.x, threads = blockDim.x;
    uint32_t *hist = lds;                                  // = the totals of the sort
    if (a.place)
        for (int e = tid; e < a.E; e += threads) hist[e] = 0;
    __syncthreads();
    uint32_t *keys = lds + a.lds_keys + (size_t)(tid / LPT) * a.key_stride;
    const int64_t t0 = (int64_t)blockIdx.x * a.block_tokens;
    const int64_t t1 = t0 + a.block_tokens < a.T ? t0 + a.block_tokens : a.T;
    for (int64_t t = t0 + tid / LPT; t - tid / LPT < t1; t += threads / LPT) {
        const int64_t wave_first = t - (tid & 63) / LPT;
        if (wave_first >= t1) continue;                    // the whole wave is beyond
        int id;
        float w;
        choose<LPT, VPL, BF16>(a, t, t < t1, keys, id, w);
        const int j = tid & (LPT - 1);
        if (t < t1 && j < a.k) {
            a.ids[t * a.k + j] = id;
            a.weights[t * a.k + j] = w;
            if (a.place && id >= 0) atomicAdd(&hist[id], 1u);
        }
    }
    if (!a.place) return;
    __syncthreads();                                       // (also: this block's ids are visible to it)
    if (gridDim.x > 1) {
        const int stride = hist_stride(a.E);
        for (int e = tid; e < stride; e += threads) a.hist[(size_t)blockIdx.x * stride + e] = (uint16_t)(e < a.E ? hist[e] : 0);
        return;
    }
    const SortLds s = sort_lds(lds, a.E);
    for (int e = tid; e < a.E; e += kBlock) s.before[e] = 0;
    scan_offsets(a, s, wave_sum);
    scatter(a, s, 0, a.T * a.k, 0, 1);
}

// Second launch where there are several blocks: every block sums up all blocks' counts (up to 128 KB, out of the L2) for the
// experts' totals and for what lies before its own tokens.
__global__ __launch_bounds__(kBlock) void dispatch_kernel(RouteArgs a, int blocks) {
    extern __shared__ uint32_t lds[];
    __shared__ uint32_t wave_sum[kWaves];
    const SortLds s = sort_lds(lds, a.E);
    const int tid = threadIdx.x, block = blockIdx.x;
    // sums of expert 8 q + i lie at i * eights + q meanwhile, so that neighbouring lanes are in neighbouring banks
    // (few parts where there are few experts: their sums meet in the same words)
    const int eights = hist_stride(a.E) / 8, parts = min(kBlock / eights, min(blocks, 64));          // E <= 1024: eight threads to eight experts
    uint32_t *total = s.wave_count, *before = total + 8 * eights;
    for (int i = tid; i < 16 * eights; i += kBlock) total[i] = 0;
    __syncthreads();
    const int q = tid % eights, part = tid / eights;
    if (part < parts) {
        uint32_t all[8] = {}, mine[8] = {};
#pragma unroll 4
        for (int b = part; b < blocks; b += parts) {
            const uint4 v = reinterpret_cast<const uint4 *>(a.hist)[(size_t)b * eights + q];
            const uint32_t n[4] = {v.x, v.y, v.z, v.w};
            const uint32_t mask = b < block ? 0xffffffffu : 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                all[2 * i] += n[i] & 0xffff;
                all[2 * i + 1] += n[i] >> 16;
                mine[2 * i] += n[i] & mask & 0xffff;
                mine[2 * i + 1] += (n[i] & mask) >> 16;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            atomicAdd(&total[i * eights + q], all[i]);
            atomicAdd(&before[i * eights + q], mine[i]);
        }
    }
    __syncthreads();
    for (int e = tid; e < a.E; e += kBlock) {
        s.total[e] = total[e % 8 * eights + e / 8];
        s.before[e] = before[e % 8 * eights + e / 8];
    }
    __syncthreads();
    scan_offsets(a, s, wave_sum);
    const int64_t first = (int64_t)block * a.block_tokens * a.k, end = first + (int64_t)a.block_tokens * a.k;
    scatter(a, s, first, end < a.T * a.k ? end : a.T * a.k, block, blocks);
}

// ---- gradient ----------------------------------------------------------------------------------------------
// With q_j = ds/dw of the chosen: (scale dw_j - sum_i w_i dw_i) / S where renormalised (S the sum of the chosen scores), else scale dw_j;
//   sigmoid: dz_j = q_j s_j (1 - s_j)        softmax: dz_e = s_e ([e chosen] q_e - sum_j q_j s_j)
// and with renormalised softmax weights the last sum is zero and s_j / S = w_j / scale: only the chosen experts' logits have one.
// A sum over shares of which one is nearly 1 is nearly that one's own term, and its difference from it would have no bits left.  So the dw
// and q above are counted from those of the expert with the largest share (not renormalised: where that is above one half; the
// experts that were not chosen, whose q is 0, then have minus that): its own term is zero, and what remains is the others'.
// A block forms the rows of its tokens in LDS, 16 lanes to a token, and streams them out: 16384 x 256 fp32 (17 MB written, 1.5 read)
// 7.9 us, which is the writes and a launch.  Without renormalisation the row's logits are read too (4099 x 64 bf16 5.1 us).
constexpr int kBwdThreads = 256, kBwdTokens = kBwdThreads / 16;
template <bool BF16> __global__ __launch_bounds__(kBwdThreads) void route_bwd_kernel(RouteBwdArgs a) {
    extern __shared__ float rows[];
    const int tid = threadIdx.x, g0 = tid & 15;
    const int64_t t0 = (int64_t)blockIdx.x * kBwdTokens, t = t0 + tid / 16;
    const bool live = t < a.T, softmax = a.score == 0, dense = softmax && !a.renorm;
    float *mine = rows + (tid / 16) * a.E;
    // k up to 32: two assignments to a lane
    int id[2];
    float w[2], dw[2], z[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int j = g0 + 16 * i;
        const bool ok = live && j < a.k;
        id[i] = ok ? a.ids[t * a.k + j] : -1;
        if (id[i] >= a.E) id[i] = -1;
        w[i] = ok ? a.weights[t * a.k + j] : 0.0f;
        dw[i] = ok && id[i] >= 0 ? a.dweights[t * a.k + j] : 0.0f;
        z[i] = id[i] >= 0 ? held(load_logit<BF16>(a.logits, t * a.ld + id[i])) : 0.0f;
    }
    float top = 0.0f, sum = 1.0f;
    if (softmax || a.renorm) {
        uint32_t m = 0;
        if (dense) {
            for (int e = g0; e < a.E; e += 16) {
                const float v = live ? load_logit<BF16>(a.logits, t * a.ld + e) : -INFINITY;
                mine[e] = v;
                const uint32_t u = is_open(v) ? ordered(held(v)) : 0u;
                m = m > u ? m : u;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t u = id[i] >= 0 && is_open(z[i]) ? ordered(z[i]) : 0u;
                m = m > u ? m : u;
            }
        }
        m = reduce_max<16>(m);
        top = m ? from_ordered(m) : 0.0f;
        if (dense) {
            sum = 0.0f;
            for (int e = g0; e < a.E; e += 16) {
                const float p = is_open(mine[e]) ? expf(held(mine[e]) - top) : 0.0f;
                mine[e] = p;
                sum += p;
            }
            sum = fmaxf(reduce_sum<16>(sum), kTiny);
        }
    }
    float s[2], part = 0.0f, chosen = 0.0f;
    uint32_t most = 0, star = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        s[i] = 0.0f;
        if (id[i] >= 0) s[i] = softmax || (a.renorm && top < kLowSigmoid) ? expf(z[i] - top) / sum : score_sigmoid(z[i]);
        const uint32_t u = __float_as_uint(s[i]);
        most = most > u ? most : u;
        chosen += s[i];
    }
    most = reduce_max<16>(most);
    float from = 0.0f;                                     // what the dw are counted from
    if (a.renorm || (dense && __uint_as_float(most) > 0.5f)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t u = id[i] >= 0 && __float_as_uint(s[i]) == most ? ordered(dw[i]) : 0u;
            star = star > u ? star : u;
        }
        star = reduce_max<16>(star);
        if (star) from = from_ordered(star);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (id[i] >= 0) dw[i] -= from;
        part += w[i] * dw[i];
    }
    if (a.renorm) {
        part = reduce_sum<16>(part);
        chosen = fmaxf(reduce_sum<16>(chosen), kTiny);
    }
    float q[2], mean = 0.0f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        q[i] = a.renorm ? (a.scale * dw[i] - part) / chosen : a.scale * dw[i];
        if (id[i] < 0) q[i] = 0.0f;
        mean += q[i] * s[i];
    }
    if (dense) {
        mean = reduce_sum<16>(mean);
        const float none = -a.scale * from;                // q of the experts that were not chosen
        if (__any(from != 0.0f)) {
            // their share, summed without the chosen ones
            __builtin_amdgcn_wave_barrier();
            __threadfence_block();
            float rest = 0.0f;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (id[i] >= 0) mine[id[i]] = 0.0f;
            __builtin_amdgcn_wave_barrier();
            __threadfence_block();
            for (int e = g0; e < a.E; e += 16) rest += mine[e];
            mean += none * (reduce_sum<16>(rest) / sum);
        }
        const float by = (none - mean) / sum;
        for (int e = g0; e < a.E; e += 16) mine[e] = mine[e] * by;
    } else {
        for (int e = g0; e < a.E; e += 16) mine[e] = 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (id[i] >= 0) {
            // (1 - s from the logit: as a difference it has no bits left where s is close to 1, a quarter of the value at z = 16)
            if (dense) mine[id[i]] = s[i] * (q[i] - mean);
            else mine[id[i]] = softmax ? q[i] * s[i] : q[i] * s[i] * score_sigmoid(-z[i]);
        }
    __syncthreads();
    // the block's rows are one run of memory that starts on 16 bytes (kBwdTokens rows are a multiple of it)
    const int n = (int)((a.T - t0 < kBwdTokens ? a.T - t0 : kBwdTokens) * a.E);
    constexpr int kVec = BF16 ? 8 : 4;
    uint8_t *out = static_cast<uint8_t *>(a.dlogits) + t0 * a.E * (BF16 ? 2 : 4);
    for (int i = tid * kVec; i < n; i += kBwdThreads * kVec) {
        if (i + kVec <= n) {
            uint4 v;
            if (BF16) v = make_uint4(pack_bf16x2(rows[i], rows[i + 1]), pack_bf16x2(rows[i + 2], rows[i + 3]),
                                     pack_bf16x2(rows[i + 4], rows[i + 5]), pack_bf16x2(rows[i + 6], rows[i + 7]));
            else v = make_uint4(__float_as_uint(rows[i]), __float_as_uint(rows[i + 1]), __float_as_uint(rows[i + 2]), __float_as_uint(rows[i + 3]));
            *reinterpret_cast<uint4 *>(out + (size_t)i * (BF16 ? 2 : 4)) = v;
        } else {
            for (int x = i; x < n; ++x) {
                if (BF16) reinterpret_cast<uint16_t *>(out)[x] = (uint16_t)f32_to_bf16_bits(rows[x]);
                else reinterpret_cast<float *>(out)[x] = rows[x];
            }
        }
    }
}

// ---- the weighted sum of the experts' rows -------------------------------------------------------------------
// y[t] = sum_j w[t,j] o[place[t,j]], in the order of j, in fp32.  A thread owns 8 columns of a token.  At the rate of a copy: 4096
// tokens of 8 rows of 2048 bf16 (151 MB) 23.8 us, 6.3 TB/s, part of them still in the memory-side cache; rows in fp32 (285 MB) 51.6, 5.5 TB/s.
// F32: the rows' type, Y_F32: y's.
template <bool F32, bool Y_F32, int AT_ONCE> __global__ __launch_bounds__(256) void combine_kernel(CombineArgs a) {
    const int per_row = (int)(a.d / 8);
    const int64_t i = block_of_many() * 256 + threadIdx.x;
    if (i >= a.T * per_row) return;
    const int64_t t = i / per_row;
    const int64_t c = (i - t * per_row) * 8;
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    // AT_ONCE rows are on their way together; one that there is not is the first row, and left out of the sum
    for (int j0 = 0; j0 < a.k; j0 += AT_ONCE) {
        int row[AT_ONCE];
        float w[AT_ONCE];
        uint4 x[AT_ONCE][F32 ? 2 : 1];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const int j = j0 + u < a.k ? j0 + u : a.k - 1;
            row[u] = a.place[t * a.k + j];
            w[u] = a.weights[t * a.k + j];
            if (j0 + u >= a.k) row[u] = -1;
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(a.o) + ((int64_t)(row[u] < 0 ? 0 : row[u]) * a.d + c) * (F32 ? 4 : 2));
#pragma unroll
            for (int b = 0; b < (F32 ? 2 : 1); ++b) x[u][b] = p[b];
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            float v[8];
#pragma unroll
            for (int b = 0; b < (F32 ? 2 : 1); ++b) {
                const uint32_t words[4] = {x[u][b].x, x[u][b].y, x[u][b].z, x[u][b].w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if (F32) v[4 * b + q] = __uint_as_float(words[q]);
                    else { v[2 * q] = __uint_as_float(words[q] << 16); v[2 * q + 1] = __uint_as_float(words[q] & 0xffff0000u); }
                }
            }
#pragma unroll
            for (int b = 0; b < 8; ++b) acc[b] = row[u] < 0 ? acc[b] : __fmaf_rn(w[u], v[b], acc[b]);
        }
    }
    if (Y_F32) {
        float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(a.y) + t * a.d + c);
        p[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        p[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    } else {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(a.y) + t * a.d + c) =
            make_uint4(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]), pack_bf16x2(acc[4], acc[5]), pack_bf16x2(acc[6], acc[7]));
    }
}

// Tokens to a block, so that there are at most 256 blocks and 64 K counts (which every block of the second launch reads).
int most_blocks(int E) { return std::min(256, 65536 / E); }
struct RoutePlan { int lpt, vpl, block_tokens, blocks, threads; };
RoutePlan route_plan(const RouteArgs &a) {
    RoutePlan p;
    // 16 lanes to a token choose for four tokens in one wave, which bounds long batches; 64 where the experts, their groups or k need
    // them, and up to 4096 tokens, which 256 blocks take at once and where a token's own time counts
    p.lpt = a.E > 256 || a.k > 16 || a.groups > 16 || a.T <= 4096 ? 64 : 16;
    p.vpl = 1;
    while (p.vpl * p.lpt < a.E) p.vpl *= 2;
    // One block chooses and sorts what it can take at once (64 tokens in four passes took 26 us, in two launches 17 with the events around
    // them).  Otherwise as many blocks as there may be, so that a compute unit has few waves that choose.
    const bool one = a.place && a.T <= kOneLaunch;
    const int64_t tokens = one ? a.T : (a.T + most_blocks(a.E) - 1) / most_blocks(a.E);
    const int64_t least = kLeast / p.lpt, most = kBlock / p.lpt;
    if (one) p.threads = kBlock;
    else p.threads = (int)std::min(std::max(tokens, least), most) * p.lpt;
    p.threads = (p.threads + 63) / 64 * 64;
    const int64_t pass = p.threads / p.lpt;
    p.block_tokens = (int)((tokens + pass - 1) / pass * pass);
    p.blocks = (int)((a.T + p.block_tokens - 1) / p.block_tokens);
    return p;
}

template <int LPT, int VPL> void launch_route_as(const RouteArgs &a, const RoutePlan &p, size_t lds, hipStream_t st) {
    if (a.bf16) hipLaunchKernelGGL((route_kernel<LPT, VPL, true>), dim3(p.blocks), dim3(p.threads), lds, st, a);
    else hipLaunchKernelGGL((route_kernel<LPT, VPL, false>), dim3(p.blocks), dim3(p.threads), lds, st, a);
}

// T = 0: no expert has a row
__global__ void no_rows_kernel(int *counts, int *offsets, int E) {
    for (int e = threadIdx.x; e <= E; e += blockDim.x) {
        offsets[e] = 0;
        if (e < E) counts[e] = 0;
    }
}

}  // namespace

size_t route_hist_bytes(const RouteArgs &a) {
    // (of the most blocks, so that it does not fall as T grows)
    return a.T > kOneLaunch ? (size_t)most_blocks(a.E) * hist_stride(a.E) * sizeof(uint16_t) : 0;
}

void launch_route(RouteArgs a, hipStream_t st) {
    if (a.T == 0) {
        if (a.offsets) hipLaunchKernelGGL(no_rows_kernel, dim3(1), dim3(256), 0, st, a.counts, a.offsets, a.E);
        return;
    }
    const RoutePlan p = route_plan(a);
    a.block_tokens = p.block_tokens;
    const bool grouped = a.top_groups < a.groups;
    const size_t sort_words = 3 * (size_t)a.E + 1 + (size_t)kWaves * hist_stride(a.E);
    // the keys of all tokens in hand (with groups), and the sort's words; in the launch that sorts too, one after the other
    a.lds_keys = a.E;
    // (with groups a token's keys and where its groups that stay begin; the tokens of a wave 16 banks apart)
    a.key_stride = (a.E + a.groups + 47) / 64 * 64 + 16;
    const size_t key_words = a.E + (grouped ? (size_t)p.threads / p.lpt * a.key_stride : 0);
    const size_t words = a.place && p.blocks == 1 ? std::max(sort_words, key_words) : key_words;
    const double bytes = (double)a.T * a.E * (a.bf16 ? 2 : 4) + 8.0 * a.T * a.k;
    profile_before(kTagRoute, st, bytes);
    const size_t lds = words * 4;
    if (p.lpt == 16) {
        switch (p.vpl) {
            case 1: launch_route_as<16, 1>(a, p, lds, st); break;
            case 2: launch_route_as<16, 2>(a, p, lds, st); break;
            case 4: launch_route_as<16, 4>(a, p, lds, st); break;
            case 8: launch_route_as<16, 8>(a, p, lds, st); break;
            default: launch_route_as<16, 16>(a, p, lds, st); break;
        }
    } else {
        switch (p.vpl) {
            case 1: launch_route_as<64, 1>(a, p, lds, st); break;
            case 2: launch_route_as<64, 2>(a, p, lds, st); break;
            case 4: launch_route_as<64, 4>(a, p, lds, st); break;
            case 8: launch_route_as<64, 8>(a, p, lds, st); break;
            default: launch_route_as<64, 16>(a, p, lds, st); break;
        }
    }
    profile_after(st);
    if (!a.place || p.blocks == 1) return;
    profile_before(kTagDispatch, st, 12.0 * a.T * a.k + 4.0 * a.rows);
    hipLaunchKernelGGL(dispatch_kernel, dim3(p.blocks), dim3(kBlock), sort_words * 4, st, a, p.blocks);
    profile_after(st);
}

void launch_route_bwd(const RouteBwdArgs &a, hipStream_t st) {
    if (a.T == 0) return;
    const int64_t blocks = (a.T + kBwdTokens - 1) / kBwdTokens;
    const size_t lds = (size_t)kBwdTokens * a.E * 4;
    profile_before(kTagRouteBwd, st, (double)a.T * a.E * (a.bf16 ? 2 : 4));
    if (a.bf16) hipLaunchKernelGGL(route_bwd_kernel<true>, dim3((unsigned)blocks), dim3(kBwdThreads), lds, st, a);
    else hipLaunchKernelGGL(route_bwd_kernel<false>, dim3((unsigned)blocks), dim3(kBwdThreads), lds, st, a);
    profile_after(st);
}

void launch_combine(const CombineArgs &a, hipStream_t st) {
    if (a.T == 0) return;
    const int64_t blocks = (a.T * (a.d / 8) + 255) / 256;
    profile_before(kTagCombine, st, (a.k * (a.o_f32 ? 4.0 : 2.0) + (a.y_f32 ? 4.0 : 2.0)) * a.T * a.d);
    // as many rows at once as there are, up to 128 bytes a thread (k = 8: one at a time 29.4 us, eight 23.9; k = 2, 1041 tokens of 4096: two
    // 7.0, eight 8.7)
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid_of_many(blocks), dim3(256), 0, st, a); };
    if (a.y_f32) {
        if (a.k <= 2) go(combine_kernel<true, true, 2>);
        else go(combine_kernel<true, true, 4>);
    } else if (a.o_f32) {
        if (a.k <= 2) go(combine_kernel<true, false, 2>);
        else go(combine_kernel<true, false, 4>);
    } else {
        if (a.k <= 2) go(combine_kernel<false, false, 2>);
        else if (a.k <= 4) go(combine_kernel<false, false, 4>);
        else go(combine_kernel<false, false, 8>);
    }
    profile_after(st);
}

}  // namespace ssg
