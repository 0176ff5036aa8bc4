// C entry points of the words' log probabilities and their gradient.
#include "entry.hpp"
#include "score.hpp"

using namespace tl;

namespace {

constexpr int WIDE = 512, NARROW = 256;         // threads of a row's workgroup

// Logits that are read past the caches: those of a list of words, which nothing reads again, and those that are too many to be there when the gradient
// reads them (256 MB hold them, and what it writes).  Measured (us, kept / past): 512 x 131072 bf16 with a list 55 / 48, with gradients 4096 x 50000 bf16 237 / 209, 813 x
// 20000 fp32 36 / 40.
bool once(const ScoreArgs &a, int size) { return a.top > 0 || (double)a.n_rows * a.vocab * size > 1.3e8; }

bool check(int dtype, int n_rows, int vocab, const void *logits, long long row)
{
    return is_dtype(dtype) && n_rows >= 0 && vocab >= 1 && vocab <= (1 << 30) && check_matrix(logits, row, dtype, n_rows, vocab, false);
}

bool word_pointer(const void *p) { return ((uintptr_t)p & 3) == 0; }

// Parts that a row is cut into: few rows are divided among workgroups where a row is long enough to pay for the second launch, which joins them.  Measured (us,
// whole / in parts of 16384 words): 1 x 50000 bf16 with 5 words 11.0 / 12.6, 1 x 131072 fp32 18.0 / 15.0, 64 x 131072 bf16 18.7 / 17.4, without words 18.4 / 13.0, 128 x 131072
// fp32 with 20 words 23 / 28; parts of 4096: 1 x 20000 fp32 8.3 / 10.6, 1 x 131072 22.0.
int parts_of(long long rows, long long vocab)
{
    if (rows == 0 || rows > 1024 || vocab < 4 * 16384) return 1;        // (asking for the units takes more than a microsecond)
    const long long units = compute_units();
    if (4 * rows > units) return 1;
    const long long n = units / rows < vocab / 16384 ? units / rows : vocab / 16384;
    return (int)(n > 64 ? 64 : n);
}

long long workspace(long long rows, int parts, int top) { return parts == 1 ? 0 : round16(rows * parts * (16 + (top > 0 ? 8ll * SCO_TOP : 0))); }

template <typename T, bool TOP, bool ONCE> void launch_rows(const ScoreArgs &a, unsigned blocks, bool wide, hipStream_t st)
{
    if (wide) hipLaunchKernelGGL((k_score<T, WIDE, TOP, ONCE>), dim3(blocks), dim3(WIDE), 0, st, a);
    else hipLaunchKernelGGL((k_score<T, NARROW, TOP, ONCE>), dim3(blocks), dim3(NARROW), 0, st, a);
}

template <typename T, bool TOP> hipError_t forward_of(ScoreArgs a, hipStream_t st)
{
    // (narrow workgroups for short rows and parts: their waves have more than a round of pieces each)
    const bool wide = a.parts == 1 && (long long)a.vocab * sizeof(T) >= 32768;
    const long long most = most_blocks(wide ? WIDE : NARROW) / a.parts;
    for (long long left = a.n_rows; left > 0; left -= most, a.first += most) {
        const unsigned n = (unsigned)((left < most ? left : most) * a.parts);
        if (once(a, sizeof(T))) launch_rows<T, TOP, true>(a, n, wide, st);
        else launch_rows<T, TOP, TOP>(a, n, wide, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.parts > 1) hipLaunchKernelGGL((k_score_join<T, TOP>), dim3((unsigned)((a.n_rows + 3) / 4)), dim3(256), 0, st, a);
    return hipGetLastError();
}

template <typename T> hipError_t forward(const ScoreArgs &a, hipStream_t st) { return a.top > 0 ? forward_of<T, true>(a, st) : forward_of<T, false>(a, st); }

template <typename T> hipError_t backward(ScoreArgs a, hipStream_t st)
{
    constexpr int WORDS = SCO_BACK_THREADS * SCO_BACK_PIECES * 16 / (int)sizeof(T);
    a.parts = (a.vocab + WORDS - 1) / WORDS;
    const long long most = most_blocks(SCO_BACK_THREADS) / a.parts;
    for (long long left = a.n_rows; left > 0; left -= most, a.first += most) {
        const dim3 grid((unsigned)((left < most ? left : most) * a.parts));
        if (once(a, sizeof(T))) hipLaunchKernelGGL((k_score_back<T, true>), grid, dim3(SCO_BACK_THREADS), 0, st, a);
        else hipLaunchKernelGGL((k_score_back<T, false>), grid, dim3(SCO_BACK_THREADS), 0, st, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

extern "C" {

int tl_score_workspace(int dtype, int n_rows, int vocab, int n_top, int64_t *bytes)
{
    if (!bytes || !is_dtype(dtype) || n_rows < 0 || vocab < 1 || vocab > (1 << 30) || n_top < 0 || n_top > SCO_TOP) return TL_EINVAL;
    *bytes = workspace(n_rows, parts_of(n_rows, vocab), n_top);
    return TL_OK;
}

int tl_score(int dtype, int n_rows, int vocab, const void *logits, int64_t row, const int32_t *word, int n_top, float *logprob, float *stats,
             int32_t *top_word, float *top_logprob, void *workspace_p, int64_t workspace_bytes, void *hip_stream)
{
    if (!check(dtype, n_rows, vocab, logits, row) || n_top < 0 || n_top > SCO_TOP) return TL_EINVAL;
    if (n_rows == 0) return TL_OK;
    if ((logprob && !word) || (n_top > 0 && (!top_word || !top_logprob))) return TL_EINVAL;
    for (const void *p : {(const void *)word, (const void *)logprob, (const void *)stats, (const void *)top_word, (const void *)top_logprob})
        if (!word_pointer(p)) return TL_EINVAL;
    ScoreArgs a = {};
    a.parts = parts_of(n_rows, vocab);
    const long long need = workspace(n_rows, a.parts, n_top);
    if (need > workspace_bytes) return TL_ELIMIT;
    if (need > 0 && (!workspace_p || ((uintptr_t)workspace_p & 15))) return TL_EINVAL;
    a.logits = logits;
    a.row = row;
    a.word = word;
    a.logprob = logprob;
    a.stats = stats;
    a.top_word = top_word;
    a.top_logprob = top_logprob;
    a.part = static_cast<float *>(workspace_p);
    a.n_rows = n_rows;
    a.vocab = vocab;
    a.top = n_top;
    const hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = dtype == TL_DT_F32 ? forward<float>(a, st) : dtype == TL_DT_BF16 ? forward<bf16_t>(a, st) : forward<f16_t>(a, st);
    return e == hipSuccess ? TL_OK : TL_EHIP;
}

int tl_score_backward(int dtype, int n_rows, int vocab, const void *logits, int64_t row, const int32_t *word, const float *stats, const float *d_logprob,
                      const float *d_entropy, void *d_logits, int64_t d_row, void *hip_stream)
{
    if (!check(dtype, n_rows, vocab, logits, row) || !check_matrix(d_logits, d_row, dtype, n_rows, vocab, true)) return TL_EINVAL;
    if (n_rows == 0) return TL_OK;
    if (!stats || (d_logprob && !word) || (d_logits == logits && d_row != row && n_rows > 1)) return TL_EINVAL;
    for (const void *p : {(const void *)word, (const void *)stats, (const void *)d_logprob, (const void *)d_entropy})
        if (!word_pointer(p)) return TL_EINVAL;
    ScoreArgs a = {};
    a.logits = logits;
    a.row = row;
    a.word = word;
    a.stats = const_cast<float *>(stats);
    a.n_rows = n_rows;
    a.vocab = vocab;
    a.d_logprob = d_logprob;
    a.d_entropy = d_entropy;
    a.d_logits = d_logits;
    a.d_row = d_row;
    const hipStream_t st = (hipStream_t)hip_stream;
    const hipError_t e = dtype == TL_DT_F32 ? backward<float>(a, st) : dtype == TL_DT_BF16 ? backward<bf16_t>(a, st) : backward<f16_t>(a, st);
    return e == hipSuccess ? TL_OK : TL_EHIP;
}

}  // extern "C"
