// Host side of the operators on a served batch (include/td.h): argument checks and launches.
// Nothing is allocated and nothing synchronises.
#include <algorithm>
#include <atomic>
#include <cmath>
#include <utility>

#include "td_embed.cuh"
#include "td_logprob.cuh"
#include "td_policy.cuh"
#include "td_range.h"

using namespace td;

namespace {

constexpr uint64_t kMaxGrid = 0x7fffffffull;
constexpr uint32_t kIndexLimit = 1u << 31;

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline uint32_t size_of(int32_t dtype) { return dtype == TD_F32 ? 4u : 2u; }
inline bool float_type(int32_t dtype) { return dtype == TD_F32 || dtype == TD_BF16 || dtype == TD_F16; }
inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The call's device made current, and the caller's put back.
class DeviceGuard {
public:
    explicit DeviceGuard(int device) {
        ok_ = cudaGetDevice(&before_) == cudaSuccess;
        if (ok_ && before_ != device) {
            ok_ = cudaSetDevice(device) == cudaSuccess;
            changed_ = ok_;
        }
    }
    ~DeviceGuard() { if (changed_) cudaSetDevice(before_); }
    DeviceGuard(const DeviceGuard &) = delete;
    DeviceGuard &operator=(const DeviceGuard &) = delete;
    bool ok() const { return ok_; }
private:
    int before_ = 0;
    bool ok_ = false, changed_ = false;
};

// Launch that may be brought on while the kernel ahead of it in the stream drains; every kernel here
// waits for that one before it touches memory.  cluster: blocks per cluster.
template <typename... KArgs, typename... Args>
cudaError_t launch_smem(void (*kernel)(KArgs...), uint64_t grid, uint32_t block, size_t smem, cudaStream_t st, uint32_t cluster,
                        Args &&...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)grid);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    cfg.attrs = attr;
#ifndef TD_NO_PDL
    attr[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
#endif
    if (cluster > 1) {
        attr[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        attr[cfg.numAttrs].val.clusterDim.x = cluster;
        attr[cfg.numAttrs].val.clusterDim.y = attr[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    return cudaLaunchKernelEx(&cfg, kernel, KArgs(std::forward<Args>(args))...);
}

template <typename... KArgs, typename... Args>
cudaError_t launch(void (*kernel)(KArgs...), uint64_t grid, uint32_t block, cudaStream_t st, uint32_t cluster, Args &&...args) {
    return launch_smem(kernel, grid, block, 0, st, cluster, std::forward<Args>(args)...);
}


BatchView view_of(const td_batch *b) {
    if (!b) return BatchView{nullptr, nullptr, nullptr, 0u};
    return BatchView{b->cu_prompt, b->cu_response, b->result, b->max_samples};
}
bool batch_ok(const td_batch *b, bool need_prompt, bool need_response) {
    return b->max_samples < kIndexLimit && aligned(b->cu_prompt, 4) && aligned(b->cu_response, 4) && aligned(b->result, 8) &&
           (b->cu_prompt || !need_prompt) && (b->cu_response || !need_response);
}

// What the two log-probability calls share.
template <typename A>
int check_logprob(const A *a) {
    if (!a || !float_type(a->dtype) || a->vocab == 0 || a->vocab >= kIndexLimit) return TD_EINVAL;
    if (a->n_rows >= kIndexLimit || a->n_tokens >= kIndexLimit || a->logits_stride < 0) return TD_EINVAL;
    if (!(a->temperature > 0.0f) || !std::isfinite(a->temperature) || !std::isfinite(1.4426951f / a->temperature)) return TD_EINVAL;
    if (a->rows != TD_ROWS_TOKEN && a->rows != TD_ROWS_STREAM) return TD_EINVAL;
    if (a->rows == TD_ROWS_TOKEN && a->n_tokens > a->n_rows) return TD_EINVAL;
    if (a->rows == TD_ROWS_STREAM && !a->batch) return TD_EINVAL;
    if (a->batch && !batch_ok(a->batch, a->rows == TD_ROWS_STREAM, true)) return TD_EINVAL;
    if ((a->n_rows && !a->logits) || (a->n_tokens && !a->targets)) return TD_EINVAL;
    if (!aligned(a->logits, size_of(a->dtype)) || !aligned(a->targets, 4) || !aligned(a->status, 4)) return TD_EINVAL;
    return TD_OK;
}
template <typename A>
LogprobArgs logprob_args(const A *a) {
    LogprobArgs k{};
    k.logits = a->logits;
    k.stride = a->logits_stride;
    k.vocab = a->vocab;
    k.n_rows = a->n_rows;
    k.n_tokens = a->n_tokens;
    k.stream_rows = a->rows == TD_ROWS_STREAM;
    k.inv_tau = (float)(1.0 / (double)a->temperature);
    k.scale2 = (float)(1.4426950408889634 / (double)a->temperature);
    k.batch = view_of(a->batch);
    k.targets = a->targets;
    k.status = a->status;
    return k;
}

template <typename T>
cudaError_t run_logprob(const LogprobArgs &k, cudaStream_t st) {
    // Blocks per row (a cluster joins them) and threads per block, by the rows there are to fill 148 SMs with.
    // In us, bfloat16, a vocabulary of 129280: 1 row 4.1 on 8 x 256 threads, 5.0 on 4 x 128; 74 rows 7.8 on
    // 2 x 512, 8.6 on 1 x 512; 148 rows 9.8 on 1 x 512, 12.2 on 1 x 256; 500 rows 25.6 on 256, 26.5 on 512;
    // 1200 rows 54.4 on 256, 59.2 on 128; 8192 rows of 152064 405 on 128, 410 on 256.  Rows of fewer than 8192
    // vectors gain nothing from a second block (32003: 3.6 on one, 3.9 on two), and a block wants four
    // vectors per thread (4096: 2.3 on 128, 3.1 on 512).  float rows, with half the work per byte, go to 128
    // threads earlier (777 rows of 50021: 27.8, on 256 31.0).
    const uint32_t nvec = k.vocab / Elem<T>::kVec, rows = k.n_tokens;
    const bool entropy = k.entropy || k.entropy_bf16;
    auto go = [&](auto *with, auto *without, uint32_t threads, uint32_t parts) {
        return launch(entropy ? with : without, (uint64_t)rows * parts, threads, st, parts, k);
    };
    auto go128 = [&]() { return go(token_logprob_kernel<T, true, 128>, token_logprob_kernel<T, false, 128>, 128, 1); };
    auto go256 = [&](uint32_t parts) { return go(token_logprob_kernel<T, true, 256>, token_logprob_kernel<T, false, 256>, 256, parts); };
    auto go512 = [&](uint32_t parts) { return go(token_logprob_kernel<T, true, 512>, token_logprob_kernel<T, false, 512>, 512, parts); };
    // Short rows go a warp each, four to a block: 8000 rows of 1000 6.9 (a block each 22.0), of 6000 19.2 (29.1);
    // 2000 rows of 6000 9.6 both ways, 200 rows 3.5 (3.2).
    if (nvec < (rows >= 4096 ? 1024 : 512))
        return launch(entropy ? token_logprob_kernel<T, true, 32> : token_logprob_kernel<T, false, 32>, ((uint64_t)rows + 3) / 4, 128, st, 1u, k);
    if (nvec >= 8192 && rows <= 74) return rows <= 18 ? go256(8) : go512(rows <= 37 ? 4 : 2);
    if (nvec >= 2048 && rows <= 296) return go512(1);
    if (nvec >= 1024 && rows <= (sizeof(T) == 4 ? 592 : 1200)) return go256(1);
    return go128();
}
template <typename T>
cudaError_t run_logprob_grad(const LogprobArgs &k, cudaStream_t st) {
    const bool same = ((reinterpret_cast<uintptr_t>(k.logits) ^ reinterpret_cast<uintptr_t>(k.grad)) & 15u) == 0 &&
                      (k.stride - k.grad_stride) * (long long)sizeof(T) % 16 == 0;
    // Short rows go a warp each: 40000 rows of 1000 bfloat16 29 us (a block each 87), of 6000 154 (178); 2000 rows of
    // 4000 9.9 (9.4), of 1000 3.3 (5.4); 200 rows of 2000 2.9 (2.1).
    if (k.vocab / Elem<T>::kVec < (k.n_rows >= 4096 ? 1024u : k.n_rows >= 1024 ? 256u : 128u)) {
        constexpr uint32_t kRows = kGradThreads / 32;
        return launch(same ? token_logprob_grad_kernel<T, true, 32> : token_logprob_grad_kernel<T, false, 32>, ((uint64_t)k.n_rows + kRows - 1) / kRows,
                      kGradThreads, st, 1u, k);
    }
    return launch(same ? token_logprob_grad_kernel<T, true, kGradThreads> : token_logprob_grad_kernel<T, false, kGradThreads>,
                  (uint64_t)k.n_rows * k.chunks, kGradThreads, st, 1u, k);
}

uint32_t policy_blocks(uint64_t n_tokens) {
    const uint64_t want = (n_tokens + 4 * kPolicyThreads - 1) / (4 * kPolicyThreads);
    return (uint32_t)(want < 1 ? 1 : want < kPolicyMaxBlocks ? want : kPolicyMaxBlocks);
}

// The instance for a call: positions per access, the KL term's form, mask and entropy or none.
template <int kVec, int kKl, bool kMask, bool kEnt>
cudaError_t run_policy(const PolicyArgs &k, cudaStream_t st) {
    constexpr size_t smem = PolicyStage<kVec, kKl, kMask, kEnt>::kStages * PolicyStage<kVec, kKl, kMask, kEnt>::kBytes;
    if (smem > 40 * 1024) {                                  // with the fixed arrays, beyond the 48 KB a launch gets unasked
        const cudaError_t rc = cudaFuncSetAttribute(policy_loss_kernel<kVec, kKl, kMask, kEnt>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (rc != cudaSuccess) return rc;
    }
    return launch_smem(policy_loss_kernel<kVec, kKl, kMask, kEnt>, policy_blocks(k.n_tokens), kPolicyThreads, smem, st, 1u, k);
}
template <int kVec, int kKl>
cudaError_t run_policy(const PolicyArgs &k, cudaStream_t st) {
    if (k.mask) return k.entropy ? run_policy<kVec, kKl, true, true>(k, st) : run_policy<kVec, kKl, true, false>(k, st);
    return k.entropy ? run_policy<kVec, kKl, false, true>(k, st) : run_policy<kVec, kKl, false, false>(k, st);
}
template <int kVec>
cudaError_t run_policy(const PolicyArgs &k, int kl, cudaStream_t st) {
    return kl == kNoKl ? run_policy<kVec, kNoKl>(k, st) : kl == kKlExp ? run_policy<kVec, kKlExp>(k, st) : run_policy<kVec, kKlPoly>(k, st);
}

template <typename T>
cudaError_t run_embed(const EmbedArgs &k, bool whole, cudaStream_t st) {
    const uint32_t nvec = k.dim / Elem<T>::kVec + 1;
    uint32_t team = 2;                                       // lanes per row, as a power of two: a quarter of its vectors
    while (team < 5 && (kEmbedUnroll << team) < nvec) ++team;
    const uint32_t pieces = (nvec + (kEmbedUnroll << team) - 1) / (kEmbedUnroll << team), teams = kEmbedThreads >> team;
    const uint64_t grid = ((uint64_t)k.n_tokens * pieces + teams - 1) / teams;
    if (grid > kMaxGrid) return cudaErrorInvalidValue;
    return launch(whole ? embed_kernel<T, true> : embed_kernel<T, false>, grid, kEmbedThreads, st, 1u, k, team, pieces);
}

// Sorted positions per chunk of the segment sums: short chunks while there are few positions to spread over the
// machine, long ones later (a run cut by a border costs two float rows of extra traffic, and one warp joins
// its parts).  65536 positions x 8 slices: 295 us with 64, 327 with 32, 309 with 128.
constexpr uint32_t kMinChunk = 8, kMaxChunk = 512, kWantParts = 148 * 64;
uint32_t chunk_rows(uint32_t n_tokens, uint32_t slices) {
    uint32_t r = kMinChunk;
    while (r < kMaxChunk && (uint64_t)n_tokens * slices > (uint64_t)r * kWantParts) r *= 2;
    return r;
}
// The most (chunk, slice) pairs of a call of up to n_tokens positions and up to so many slices: with the shortest chunks
// ceil(n / 8) slices; with longer ones kWantParts and the last, partly filled chunk's, or ceil(n / 512) slices
// where even the longest chunks are more.
uint64_t most_parts(uint32_t n_tokens, uint32_t slices) {
    const uint64_t shortest = ((uint64_t)n_tokens + kMinChunk - 1) / kMinChunk * slices, longest = ((uint64_t)n_tokens + kMaxChunk - 1) / kMaxChunk * slices;
    return std::min<uint64_t>(shortest, std::max<uint64_t>((uint64_t)kWantParts + slices, longest));
}
constexpr uint32_t kFewTiles = 1u << 17;                     // positions up to which a tile of the sort is kSortThreads * 4, beyond * 16
uint32_t most_tiles(uint32_t n_tokens) {                     // of a call of up to n_tokens positions
    const uint32_t small = (std::min(n_tokens, kFewTiles) + kSortThreads * 4 - 1) / (kSortThreads * 4);
    return std::max(small, (uint32_t)(((uint64_t)n_tokens + kSortThreads * 16 - 1) / (kSortThreads * 16)));
}
struct EmbedGradLayout {
    size_t keys[2], pos[2], counts, present, arrived, partial, partial_stride, total;
    uint32_t n_tiles, n_chunks, rows_per_chunk, slices, passes;
    bool big_tiles;
};
// Areas have room for what any call with no more positions, vocabulary and columns would take, so that a workspace for the
// largest call holds for all.
EmbedGradLayout embed_layout(uint32_t n_tokens, uint32_t vocab, uint32_t dim) {
    EmbedGradLayout L{};
    int bits = 0;
    while (bits < 32 && (vocab >> bits) != 0) ++bits;        // the keys are 0 .. vocab
    L.passes = (uint32_t)((bits + kSortBits - 1) / kSortBits);
    L.big_tiles = n_tokens > kFewTiles;                      // every block reads all tiles' counts: few of them
    const uint32_t tile = kSortThreads * (L.big_tiles ? 16 : 4);
    L.n_tiles = (uint32_t)(((uint64_t)n_tokens + tile - 1) / tile);
    L.slices = (uint32_t)(((uint64_t)dim + kSumWarpCols - 1) / kSumWarpCols);
    L.rows_per_chunk = chunk_rows(n_tokens, L.slices);
    L.n_chunks = (uint32_t)(((uint64_t)n_tokens + L.rows_per_chunk - 1) / L.rows_per_chunk);
    L.partial_stride = (size_t)L.slices * kSumWarpCols;
    size_t p = 0;
    auto take = [&](size_t bytes) { const size_t at = p; p = round_up(p + bytes, 256); return at; };
    for (int k = 0; k < 2; ++k) { L.keys[k] = take((size_t)n_tokens * 4); L.pos[k] = take((size_t)n_tokens * 4); }
    const size_t parts = most_parts(n_tokens, L.slices);
    L.counts = take((size_t)L.passes * most_tiles(n_tokens) * kSortBins * 4);
    L.present = take(((size_t)vocab + 31) / 32 * 4);
    L.arrived = take(3 * parts * 4);
    L.partial = take(2 * parts * kSumWarpCols * 4);
    L.total = p;
    return L;
}

template <int kItems>
cudaError_t run_sort(EmbedArgs &k, const EmbedGradLayout &L, uint8_t *ws, cudaStream_t st) {
    SortPass s{};
    s.n_tiles = L.n_tiles;
    s.passes = L.passes;
    s.counts = reinterpret_cast<uint32_t *>(ws + L.counts);
    cudaError_t rc = launch(sort_count_kernel<kItems>, L.n_tiles, kSortThreads, st, 1u, k, s);
    for (uint32_t p = 0; p < L.passes && rc == cudaSuccess; ++p) {
        s.shift = p * kSortBits;
        s.first = p == 0;
        s.last = p + 1 == L.passes;
        s.keys_in = reinterpret_cast<uint32_t *>(ws + L.keys[(p + 1) & 1]);
        s.pos_in = reinterpret_cast<uint32_t *>(ws + L.pos[(p + 1) & 1]);
        s.keys_out = reinterpret_cast<uint32_t *>(ws + L.keys[p & 1]);
        s.pos_out = reinterpret_cast<uint32_t *>(ws + L.pos[p & 1]);
        rc = launch(sort_place_kernel<kItems>, L.n_tiles + (s.last ? k.zero_from : 0u), kSortThreads, st, 1u, k, s);
    }
    k.keys = s.keys_out;
    k.pos = s.pos_out;
    return rc;
}

template <typename T, typename G>
cudaError_t run_embed_grad(EmbedArgs k, const EmbedGradLayout &L, uint8_t *ws, bool wide, cudaStream_t st) {
    // Rows without a token are cleared by blocks behind those of the sums, 32 rows each or 32 kZeroWords.
    cudaError_t rc;
    const uint32_t per_block = (uint64_t)k.dim * sizeof(G) >= kLongRow ? 1u : kZeroWords;
    const uint32_t zeroing = k.accumulate ? 0u : (uint32_t)(((uint64_t)k.vocab + 32 * per_block - 1) / (32 * per_block));
    // Few positions need no sort.  Without / with one, in us, added into float rows: 300 of 40 columns 4.2 / 9.5, 2000 of 40
    // 13.9 / 14.6, 600 of 1001 11.2 / 13.9, 30 of 4096 3.3 / 8.3; but 1000 of 1001 18.6 / 15.3, 4000 of 40 34.6 / 19.5,
    // 300 of 4096 15.5 / 10.0.
    if ((uint64_t)k.n_tokens * L.slices <= 2400) {
        const uint32_t positions = k.n_tokens * L.slices;
        if (positions + zeroing == 0) return cudaSuccess;
        return launch(wide ? embed_few_kernel<T, G, true> : embed_few_kernel<T, G, false>, (uint64_t)positions + zeroing, kSumThreads, st, 1u, k, L.slices, positions);
    }
    k.arrived = reinterpret_cast<uint32_t *>(ws + L.arrived);
    k.n_arrived = 3 * L.n_chunks * L.slices;
    if (k.n_tokens <= kRankMax) {
        k.keys = reinterpret_cast<uint32_t *>(ws + L.keys[0]);
        k.pos = reinterpret_cast<uint32_t *>(ws + L.pos[0]);
        rc = launch(embed_rank_kernel, (k.n_tokens + 31) / 32, kRankThreads, st, 1u, k);
    } else {
        if (zeroing) {
            k.present = reinterpret_cast<uint32_t *>(ws + L.present);
            // the last of several placing kernels leaves most of the machine idle for 8 us: time to clear the first 30 MB
            const uint64_t early = (30ull << 20) / (32 * per_block * (uint64_t)k.dim * sizeof(G)) + 1;
            if (L.passes > 1) k.zero_from = early < zeroing ? (uint32_t)early : zeroing;
        }
        rc = L.big_tiles ? run_sort<16>(k, L, ws, st) : run_sort<4>(k, L, ws, st);
    }
    if (rc != cudaSuccess) return rc;
    const uint32_t sum_blocks = (uint32_t)(((uint64_t)L.n_chunks * L.slices + kSumThreads / 32 - 1) / (kSumThreads / 32));
    const uint32_t zero_blocks = zeroing - k.zero_from;
    if (sum_blocks + zero_blocks == 0) return cudaSuccess;
    const uint64_t grid = (uint64_t)sum_blocks + zero_blocks;
    const size_t smem = sum_blocks ? kSumWarps * (wide ? SumLayout<T, true>::kWarpBytes : SumLayout<T, false>::kWarpBytes) : 0;
    auto *kernel = wide ? embed_sum_kernel<T, G, true> : embed_sum_kernel<T, G, false>;
    if (smem > 48 * 1024 && (rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem)) != cudaSuccess) return rc;
    return launch_smem(kernel, grid, kSumThreads, smem, st, 1u, k, L.slices, sum_blocks);
}

}  // namespace

extern "C" {

int td_token_logprob(const td_logprob_args *a, void *stream) {
    TD_RANGE("td_token_logprob");
    const int chk = check_logprob(a);
    if (chk != TD_OK) return chk;
    if (a->n_tokens == 0) return TD_OK;
    if (!a->logprob || !aligned(a->logprob, 4) || !aligned(a->norm, 4) || !aligned(a->entropy, 4) || !aligned(a->entropy_bf16, 2))
        return TD_EINVAL;
    DeviceGuard dev(a->device);
    if (!dev.ok()) return TD_ECUDA;
    LogprobArgs k = logprob_args(a);
    k.logprob = a->logprob;
    k.norm = a->norm;
    k.entropy = a->entropy;
    k.entropy_bf16 = static_cast<__nv_bfloat16 *>(a->entropy_bf16);
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t rc = a->dtype == TD_F32 ? run_logprob<float>(k, st)
                         : a->dtype == TD_BF16 ? run_logprob<__nv_bfloat16>(k, st) : run_logprob<__half>(k, st);
    return rc == cudaSuccess ? TD_OK : TD_ECUDA;
}

int td_token_logprob_grad(const td_logprob_grad_args *a, void *stream) {
    TD_RANGE("td_token_logprob_grad");
    const int chk = check_logprob(a);
    if (chk != TD_OK) return chk;
    if (a->n_rows == 0) return TD_OK;
    if (!a->grad_logits || !aligned(a->grad_logits, size_of(a->dtype)) || a->grad_stride < (int64_t)a->vocab) return TD_EINVAL;
    if (a->grad_logits == a->logits && a->grad_stride != a->logits_stride) return TD_EINVAL;
    if (a->n_tokens && (!a->norm || (!a->grad_logprob && !a->grad_entropy) || (a->grad_entropy && !a->entropy))) return TD_EINVAL;
    if (!aligned(a->norm, 4) || !aligned(a->entropy, 4) || !aligned(a->grad_logprob, 4) || !aligned(a->grad_entropy, 4)) return TD_EINVAL;
    LogprobArgs k = logprob_args(a);
    k.norm_in = a->norm;
    k.entropy_in = a->entropy;
    k.grad_logprob = a->grad_logprob;
    k.grad_entropy = a->grad_entropy;
    k.grad = a->grad_logits;
    k.grad_stride = a->grad_stride;
    const uint32_t per_vec = 16u / size_of(a->dtype);
    const uint32_t nvec = (a->vocab + per_vec - 1) / per_vec;
    k.chunks = (nvec + kGradVectors - 1) / kGradVectors;
    if ((uint64_t)a->n_rows * k.chunks > kMaxGrid) return TD_EINVAL;
    DeviceGuard dev(a->device);
    if (!dev.ok()) return TD_ECUDA;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t rc = a->dtype == TD_F32 ? run_logprob_grad<float>(k, st)
                         : a->dtype == TD_BF16 ? run_logprob_grad<__nv_bfloat16>(k, st) : run_logprob_grad<__half>(k, st);
    return rc == cudaSuccess ? TD_OK : TD_ECUDA;
}

size_t td_policy_loss_workspace_bytes(uint32_t max_samples) {
    return round_up(256 + (size_t)kPolicyMaxBlocks * kPolicySums * 8 + (size_t)max_samples * 4, 256);
}

int td_policy_loss(const td_policy_args *a, void *stream) {
    TD_RANGE("td_policy_loss");
    if (!a || !a->batch || !batch_ok(a->batch, false, true)) return TD_EINVAL;
    if (a->row_width) {
        if (a->row_width >= kIndexLimit || a->n_tokens != (uint64_t)a->batch->max_samples * a->row_width || a->n_tokens >= 1ull << 40) return TD_EINVAL;
    } else if (a->n_tokens >= kIndexLimit) return TD_EINVAL;
    if (a->column_dtype != TD_F32 && a->column_dtype != TD_BF16) return TD_EINVAL;
    if (a->ref_logprob && (a->kl_kind < TD_KL_K1 || a->kl_kind > TD_KL_K3)) return TD_EINVAL;
    if (a->reduction != TD_MEAN_TOKENS && a->reduction != TD_MEAN_SAMPLES) return TD_EINVAL;
    if (!(a->clip_low >= 0.0f) || !(a->clip_low <= 1.0f) || !(a->clip_high >= 0.0f)) return TD_EINVAL;
    if (!(a->dual_clip == 0.0f || a->dual_clip > 1.0f) || !(a->norm >= 0.0f)) return TD_EINVAL;
    if (!std::isfinite(a->kl_coef) || !std::isfinite(a->entropy_coef) || !std::isfinite(a->norm) || !std::isfinite(a->grad_scale)) return TD_EINVAL;
    if (!a->stats || !aligned(a->stats, 4)) return TD_EINVAL;
    if (a->n_tokens && (!a->logprob || !a->advantages || !a->grad_logprob)) return TD_EINVAL;
    const size_t cs = size_of(a->column_dtype);
    if (!aligned(a->logprob, 4) || !aligned(a->old_logprob, cs) || !aligned(a->ref_logprob, cs) || !aligned(a->entropy, 4) ||
        !aligned(a->advantages, 4) || !aligned(a->grad_logprob, 4) || !aligned(a->grad_entropy, 4)) return TD_EINVAL;
    if (!a->workspace || !aligned(a->workspace, 256) || a->workspace_bytes < td_policy_loss_workspace_bytes(a->batch->max_samples))
        return TD_EWORKSPACE;
    DeviceGuard dev(a->device);
    if (!dev.ok()) return TD_ECUDA;

    PolicyArgs k{};
    k.batch = view_of(a->batch);
    k.n_tokens = a->n_tokens;
    k.row_width = a->row_width;
    k.bf16_columns = a->column_dtype == TD_BF16;
    k.kl_c1 = a->kl_kind == TD_KL_K1 ? -1.0f : 0.0f;
    k.kl_c2 = a->kl_kind == TD_KL_K2 ? 0.5f : 0.0f;
    k.mean_samples = a->reduction == TD_MEAN_SAMPLES;
    k.lo = 1.0f - a->clip_low;
    k.hi = 1.0f + a->clip_high;
    k.dual_clip = a->dual_clip > 0.0f ? a->dual_clip : INFINITY;
    k.kl_coef = a->ref_logprob ? a->kl_coef : 0.0f;
    k.entropy_coef = a->entropy ? a->entropy_coef : 0.0f;
    k.norm = a->norm;
    k.grad_scale = a->grad_scale;
    k.logprob = a->logprob;
    k.old_logprob = a->old_logprob;
    k.ref_logprob = a->ref_logprob;
    k.entropy = a->entropy;
    k.mask = a->mask;
    k.advantages = a->advantages;
    k.grad_logprob = a->grad_logprob;
    k.grad_entropy = a->grad_entropy;
    k.stats = a->stats;
    uint8_t *ws = static_cast<uint8_t *>(a->workspace);
    k.ticket = reinterpret_cast<uint32_t *>(ws);
    k.partials = reinterpret_cast<double *>(ws + 256);
    k.counts = reinterpret_cast<int32_t *>(ws + 256 + (size_t)kPolicyMaxBlocks * kPolicySums * 8);
    k.need_counts = k.mean_samples ? a->mask != nullptr : a->norm == 0.0f && (a->mask || a->row_width);
    cudaStream_t st = (cudaStream_t)stream;
    if (k.need_counts && a->batch->max_samples) {
        const uint32_t per = kPolicyThreads / 32;
        if (launch(policy_count_kernel, (a->batch->max_samples + per - 1) / per, kPolicyThreads, st, 1u, k) != cudaSuccess) return TD_ECUDA;
    }
    // four positions per access where every array allows it
    const bool wide = aligned(k.logprob, 16) && aligned(k.old_logprob, 4 * cs) && aligned(k.ref_logprob, 4 * cs) &&
                      aligned(k.entropy, 16) && aligned(k.mask, 4) && aligned(k.grad_logprob, 16) && aligned(k.grad_entropy, 16);
    const int kl = !a->ref_logprob ? kNoKl : a->kl_kind == TD_KL_K3 ? kKlExp : kKlPoly;
    const cudaError_t rc = wide ? run_policy<4>(k, kl, st) : run_policy<1>(k, kl, st);
    return rc == cudaSuccess ? TD_OK : TD_ECUDA;
}

int td_embed(const td_embed_args *a, void *stream) {
    TD_RANGE("td_embed");
    if (!a || !float_type(a->dtype) || a->vocab == 0 || a->vocab >= kIndexLimit || a->dim == 0 || a->dim >= kIndexLimit) return TD_EINVAL;
    if (a->n_tokens >= kIndexLimit || a->table_stride < (int64_t)a->dim || a->out_stride < (int64_t)a->dim) return TD_EINVAL;
    if (a->batch && (a->tokens < TD_TOKENS_PROMPT || a->tokens > TD_TOKENS_SEQ ||
                     !batch_ok(a->batch, a->tokens & TD_TOKENS_PROMPT, a->tokens & TD_TOKENS_RESPONSE))) return TD_EINVAL;
    if (a->n_tokens == 0) return TD_OK;
    const uint32_t es = size_of(a->dtype);
    if (!a->ids || !a->table || !a->out || !aligned(a->ids, 4) || !aligned(a->table, es) || !aligned(a->out, es) || !aligned(a->status, 4))
        return TD_EINVAL;
    // rows of both sides start on 16-byte boundaries
    const bool whole = aligned(a->table, 16) && aligned(a->out, 16) && a->table_stride * es % 16 == 0 && a->out_stride * es % 16 == 0;
    DeviceGuard dev(a->device);
    if (!dev.ok()) return TD_ECUDA;
    EmbedArgs k{};
    k.ids = a->ids;
    k.n_tokens = a->n_tokens;
    k.vocab = a->vocab;
    k.dim = a->dim;
    k.tokens = (uint32_t)a->tokens;
    k.scale = a->scale;
    k.batch = view_of(a->batch);
    k.status = a->status;
    k.table = a->table;
    k.out = a->out;
    k.table_stride = a->table_stride;
    k.out_stride = a->out_stride;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t rc = a->dtype == TD_F32 ? run_embed<float>(k, whole, st)
                         : a->dtype == TD_BF16 ? run_embed<__nv_bfloat16>(k, whole, st) : run_embed<__half>(k, whole, st);
    if (rc == cudaErrorInvalidValue) return TD_EINVAL;
    return rc == cudaSuccess ? TD_OK : TD_ECUDA;
}

size_t td_embed_grad_workspace_bytes(uint32_t n_tokens, uint32_t vocab, uint32_t dim) {
    return n_tokens < kIndexLimit && vocab < kIndexLimit && dim < kIndexLimit ? embed_layout(n_tokens, vocab, dim).total : 0;
}

int td_embed_grad(const td_embed_grad_args *a, void *stream) {
    TD_RANGE("td_embed_grad");
    if (!a || !float_type(a->dtype) || a->vocab == 0 || a->vocab >= kIndexLimit || a->dim == 0 || a->dim >= kIndexLimit) return TD_EINVAL;
    if (a->grad_dtype != TD_F32 && a->grad_dtype != a->dtype) return TD_EINVAL;
    if (a->n_tokens >= kIndexLimit || a->table_stride < (int64_t)a->dim || a->out_stride < 0) return TD_EINVAL;
    if (a->accumulate != 0 && a->accumulate != 1) return TD_EINVAL;
    if (a->batch && (a->tokens < TD_TOKENS_PROMPT || a->tokens > TD_TOKENS_SEQ ||
                     !batch_ok(a->batch, a->tokens & TD_TOKENS_PROMPT, a->tokens & TD_TOKENS_RESPONSE))) return TD_EINVAL;
    const uint32_t es = size_of(a->dtype), gs = size_of(a->grad_dtype);
    if (!a->grad_table || !aligned(a->grad_table, gs) || !aligned(a->status, 4)) return TD_EINVAL;
    if (a->n_tokens && (!a->ids || !a->grad_out || !aligned(a->ids, 4) || !aligned(a->grad_out, es))) return TD_EINVAL;
    const EmbedGradLayout L = embed_layout(a->n_tokens, a->vocab, a->dim);
    if (!a->workspace || !aligned(a->workspace, 256) || a->workspace_bytes < L.total) return TD_EWORKSPACE;
    if (3 * (uint64_t)L.n_chunks * L.slices + (uint64_t)a->vocab / 32 >= kMaxGrid) return TD_EINVAL;          // also keeps n_arrived in 32 bits
    DeviceGuard dev(a->device);
    if (!dev.ok()) return TD_ECUDA;
    EmbedArgs k{};
    k.ids = a->ids;
    k.n_tokens = a->n_tokens;
    k.vocab = a->vocab;
    k.dim = a->dim;
    k.tokens = (uint32_t)a->tokens;
    k.scale = a->scale;
    k.batch = view_of(a->batch);
    k.status = a->status;
    k.grad_out = a->grad_out;
    k.out_stride = a->out_stride;
    k.grad_table = a->grad_table;
    k.table_stride = a->table_stride;
    k.accumulate = (uint32_t)a->accumulate;
    k.grad_size = gs;
    k.rows_per_chunk = L.rows_per_chunk;
    k.n_chunks = L.n_chunks;
    uint8_t *ws = static_cast<uint8_t *>(a->workspace);
    k.partial = reinterpret_cast<float *>(ws + L.partial);
    k.partial_stride = L.partial_stride;
    // rows of both sides start on 16-byte boundaries and are whole lanes' columns
    const bool wide = a->dim % kSumCols == 0 && aligned(a->grad_out, 16) && a->out_stride * es % 16 == 0 && aligned(a->grad_table, 16) &&
                      a->table_stride * gs % 16 == 0;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t rc;
    if (a->dtype == TD_F32) rc = run_embed_grad<float, float>(k, L, ws, wide, st);
    else if (a->dtype == TD_BF16)
        rc = a->grad_dtype == TD_F32 ? run_embed_grad<__nv_bfloat16, float>(k, L, ws, wide, st)
                                     : run_embed_grad<__nv_bfloat16, __nv_bfloat16>(k, L, ws, wide, st);
    else
        rc = a->grad_dtype == TD_F32 ? run_embed_grad<__half, float>(k, L, ws, wide, st)
                                     : run_embed_grad<__half, __half>(k, L, ws, wide, st);
    return rc == cudaSuccess ? TD_OK : TD_ECUDA;
}

}  // extern "C"
