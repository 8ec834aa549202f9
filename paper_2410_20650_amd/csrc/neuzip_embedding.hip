// Embedding on a compressed table: host side of the C ABI (see include/neuzip.h).

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "neuzip.h"

#include "neuzip_embedding_kernels.h"
#include "neuzip_host.h"

using namespace nz;

namespace {

inline bool valid_table(uint64_t rows, uint64_t features)
{
    return rows > 0 && features > 0 && features % kRun == 0 && rows < (1ull << 32) && features < (1ull << 32) &&
           rows * features < (1ull << 32);
}

// Gradient: up to which tokens one launch does it all, with any table (us, three launches / one: 64 tokens, 5003 x 520 7.9 / 4.2, 50257 x 768
// 15.3 / 13.1, 128256 x 4096 158.6 / 151.7; all of one row, 5003 x 520, 9.8 / 9.0), and with one of at most 8 MB, whose zeros then leave at a quarter of
// the rate (333 tokens, 2048 x 512 12.0 / 5.9, 5003 x 520 12.6 / 8.1, 1040 x 3648, 7.6 MB, 13.7 / 11.8, but 12936 x 856, 22 MB, 13.7 / 18.6; 512 of one
// row, 5003 x 520, 14.7 / 15.7).
constexpr uint32_t kFewTokens = 64, kSomeTokens = 512;
constexpr uint64_t kSomePieces = 1ull << 19;

// Tables up to which the sort has workgroups of 1024 threads, which count a run sooner; the zeros of larger ones, which hide it, leave
// faster from smaller ones (us, 256 / 1024 threads: 4096 tokens, 5003 x 520, 11.4 / 7.2; 2048, 32000 x 2048, 18.3 / 18.4; 4096, 128256 x 4096, 155 / 171).
constexpr uint64_t kSortWidePieces = 1ull << 23;
template <uint32_t THREADS>
void launch_sort(const EmbeddingGradArgs &a, hipStream_t stream)
{
    const uint64_t fill_wgs = (static_cast<uint64_t>(a.rows) * a.row_pieces.by + THREADS - 1) / THREADS;
    hipLaunchKernelGGL(embedding_sort_kernel<THREADS>, dim3(static_cast<uint32_t>(static_cast<uint64_t>(a.sort_wgs) * a.n_runs + fill_wgs)), dim3(THREADS), 0,
                       stream, a);
}

// how many parts the tokens are looked over in, 0: not in one launch
inline uint32_t few_parts(uint64_t count, uint64_t rows, uint64_t features)
{
    return count == 0 ? 0u : count <= kFewTokens ? 1u : count <= kSomeTokens && rows * features / kRun <= kSomePieces ? 4u : 0u;
}

template <int PARTS>
void launch_few(const EmbeddingGradArgs &a, hipStream_t stream)
{
    constexpr uint32_t kWide = kGradThreads / PARTS;
    const uint32_t pieces = a.rows * a.row_pieces.by;
    hipLaunchKernelGGL(embedding_few_kernel<PARTS>, dim3((pieces + kWide - 1) / kWide), dim3(kGradThreads), 0, stream, a);
}

template <int KB, bool NORM>
void launch_embedding(const EmbeddingArgs &a, hipStream_t stream)
{
    // Few units: workgroups of four waves, and the step without a branch, as long as a CU has one or two of them.
    constexpr uint32_t kFew = 256, kMany = 512;
    const uint32_t wgs = (a.units + kFew / kStates - 1) / (kFew / kStates);
    if (wgs <= 512)
        hipLaunchKernelGGL((embedding_kernel<KB, NORM, true, kFew>), dim3(wgs), dim3(kFew), 0, stream, a);
    else
        hipLaunchKernelGGL((embedding_kernel<KB, NORM, false, kMany>), dim3((a.units + kMany / kStates - 1) / (kMany / kStates)), dim3(kMany), 0,
                           stream, a);
}

}  // namespace

extern "C" {

int neuzip_embedding(const neuzip_blob *table, uint64_t rows, uint64_t features, const int64_t *d_tokens, uint64_t count, float scale,
                     void *d_out, void *hip_stream)
{
    if (!is_blob(table) || !table->has_table || !on_current_device(table) || !valid_table(rows, features) || rows * features != table->n)
        return NEUZIP_EINVAL;
    if (table->elem != NEUZIP_BF16)
        return NEUZIP_EUNSUPPORTED;
    if (count == 0)
        return NEUZIP_OK;
    if (!d_tokens || !d_out || (reinterpret_cast<uintptr_t>(d_tokens) & 7u) || (reinterpret_cast<uintptr_t>(d_out) & 15u))
        return NEUZIP_EINVAL;
    // units of a token: as many as a row's elements can touch
    const uint64_t unit = has_entry_points(table->n_chunks) ? kMidTurn * kTurn : kChunk;
    const uint64_t per_token = unit % features == 0 ? 1 : (features % unit == 0 ? features / unit : (features - 1) / unit + 2);
    if (count >= (1ull << 27) || count * per_token >= (1ull << 27))  // (16 threads to each, of fewer than 2^32)
        return NEUZIP_EUNSUPPORTED;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const int behind = follow(table, stream);
    if (behind != NEUZIP_OK)
        return behind;
    EmbeddingArgs a;
    std::memset(&a, 0, sizeof(a));
    a.tb = table_of(table);
    a.offsets = offsets_of(table);
    a.states = states_of(table);
    a.lens = lens_of(table);
    a.mid_states = mid_states_of(table);
    a.mid_lens = mid_lens_of(table);
    a.words = reinterpret_cast<const uint16_t *>(table->words);
    a.sm = sm_of(table);
    a.coef = coef_of(table);
    while (table->block && (1u << a.block_shift) < table->block)
        ++a.block_shift;
    a.n_chunks = table->n_chunks;
    a.status = table_of(table)->status;
    a.tokens = d_tokens;
    a.out = static_cast<uint16_t *>(d_out);
    a.rows = static_cast<uint32_t>(rows);
    a.features = static_cast<uint32_t>(features);
    a.per_token.set(static_cast<uint32_t>(per_token));
    a.units = static_cast<uint32_t>(count * per_token);
    a.scale = scale;
    if (table->block) {
        switch (table->k) {
        case 3: launch_embedding<3, true>(a, stream); break;
        case 1: launch_embedding<1, true>(a, stream); break;
        default: launch_embedding<0, true>(a, stream); break;
        }
    } else {
        switch (table->k) {
        case 7: launch_embedding<7, false>(a, stream); break;
        case 3: launch_embedding<3, false>(a, stream); break;
        case 1: launch_embedding<1, false>(a, stream); break;
        default: launch_embedding<0, false>(a, stream); break;
        }
    }
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

uint64_t neuzip_embedding_grad_scratch_bytes(uint64_t count, uint64_t rows, uint64_t features)
{
    if (!valid_table(rows, features) || count >= (1ull << 31) || few_parts(count, rows, features))
        return 0;
    const uint64_t runs = (count + kSortRun - 1) / kSortRun;
    return runs * (sizeof(SortedRun) + kPieces * features * sizeof(float));
}

int neuzip_embedding_grad(const int64_t *d_tokens, uint64_t count, const void *d_grad_out, uint64_t rows, uint64_t features, float scale,
                          void *d_grad, void *d_scratch, uint64_t scratch_bytes, void *hip_stream)
{
    if (!valid_table(rows, features) || !d_grad || (reinterpret_cast<uintptr_t>(d_grad) & 15u))
        return NEUZIP_EINVAL;
    if (count >= (1ull << 31))
        return NEUZIP_EUNSUPPORTED;
    if (count > 0 && (!d_tokens || !d_grad_out || (reinterpret_cast<uintptr_t>(d_tokens) & 7u) || (reinterpret_cast<uintptr_t>(d_grad_out) & 15u)))
        return NEUZIP_EINVAL;
    const uint64_t needed = neuzip_embedding_grad_scratch_bytes(count, rows, features);
    if (needed > 0 && (!d_scratch || (reinterpret_cast<uintptr_t>(d_scratch) & 15u) || scratch_bytes < needed))
        return NEUZIP_EINVAL;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    EmbeddingGradArgs a;
    std::memset(&a, 0, sizeof(a));
    a.tokens = d_tokens;
    a.count = count;
    a.grad_out = static_cast<const uint16_t *>(d_grad_out);
    a.grad = static_cast<uint16_t *>(d_grad);
    a.runs = static_cast<SortedRun *>(d_scratch);
    a.n_runs = static_cast<uint32_t>((count + kSortRun - 1) / kSortRun);
    a.partial = reinterpret_cast<float *>(a.runs + a.n_runs);
    a.rows = static_cast<uint32_t>(rows);
    a.features = static_cast<uint32_t>(features);
    while (((rows - 1) >> a.range_shift) >= kSortRanges)
        ++a.range_shift;
    a.row_pieces.set(static_cast<uint32_t>(features / kRun));
    a.scale = scale;
    if (a.n_runs > 65535)
        return NEUZIP_EUNSUPPORTED;
    const uint32_t most = count < kSortRun ? static_cast<uint32_t>(count) : kSortRun;  // tokens of a run
    a.sort_wgs = count > 0 ? (most + kSortRanges + kSortQueries) / kSortQueries : 0u;
    const uint32_t strips = (a.row_pieces.by + kGradThreads - 1) / kGradThreads;
    if (strips > 65535)
        return NEUZIP_EUNSUPPORTED;
    if (const uint32_t parts = few_parts(count, rows, features)) {
        if (parts == 1)
            launch_few<1>(a, stream);
        else
            launch_few<4>(a, stream);
        return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
    }
    if (rows * a.row_pieces.by <= kSortWidePieces && a.n_runs <= 64)  // (more runs have every CU at work anyway, and a launch fewer than 2^32 threads)
        launch_sort<1024>(a, stream);
    else
        launch_sort<256>(a, stream);
    if (count > 0) {
        hipLaunchKernelGGL(embedding_pieces_kernel, dim3(kPieces, a.n_runs, strips), dim3(kGradThreads), 0, stream, a);
        hipLaunchKernelGGL(embedding_rows_kernel, dim3(most, a.n_runs, strips), dim3(kGradThreads), 0, stream, a);
    }
    return hip_ok(hipGetLastError()) ? NEUZIP_OK : NEUZIP_EHIP;
}

}  // extern "C"
