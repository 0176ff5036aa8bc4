// C entry points of the recurrence along sentences.
#include "entry.hpp"
#include "recur.hpp"

using namespace tl;

namespace {

// Waves of a workgroup and words that each takes at a time: whole sentences forwards (F) and backwards (B), many brief ones (FB, BB), parts (FC, BC) and large
// parts (FL, BL) of cut ones.  A lane has 4 bytes of a row.
constexpr int F_WAVES = 4, F_WORDS = 8;
constexpr int B_WAVES = 4, B_WORDS = 16;
constexpr int FB_WAVES = 4, FB_WORDS = 8, BB_WAVES = 4, BB_WORDS = 16;
constexpr int FC_WAVES = 8, FC_WORDS = 16, FL_WAVES = 8, FL_WORDS = 32;
constexpr int BC_WAVES = 8, BC_WORDS = 8, BL_WAVES = 8, BL_WORDS = 16;
constexpr int LANE_BYTES = 4;

// (as many words as a state's place and the block behind the last word can be counted in 32 bits with)
constexpr int MOST_ROWS = INT32_MAX - 65536;

constexpr int log_2(int n) { return n > 1 ? 1 + log_2(n / 2) : 0; }

bool check(const tl_recurrence *r)
{
    if (!r || !is_dtype(r->dtype) || (r->gate != TL_GATE_SIGMOID && r->gate != TL_GATE_GIVEN)) return false;
    if (r->n_trees < 0 || r->n_rows < 0 || r->n_rows > MOST_ROWS || r->channels < 1 || r->channels > (1 << 20)) return false;
    if (r->n_trees == 0) return r->n_rows == 0;
    return r->off && check_matrix(r->g, r->g_row, r->dtype, r->n_rows, r->channels, false) && check_matrix(r->x, r->x_row, r->dtype, r->n_rows, r->channels, false);
}

struct Plan {
    int V, slices, shift, slots;
    bool narrow, single, brief, cut, large;                  // a wave per sentence; sentences of a block or two; parts
    long long blocks, pairs, states, parts, copy;               // bytes of the workspace's parts
    long long workspace() const { return pairs + states + parts + copy + (cut ? 16 : 0); }
};

// Whether sentences are cut into parts, by their words on average (the host sees no lengths, and a batch with one sentence much longer than the
// others waits for it).  A whole sentence is a chain of blocks, a part waits for others, for its number, and needs a launch more.  Measured (us, whole / cut, states alone, then gradients
// less the states; words x channels, bf16): 20 sentences of 165 x 512 15.4 / 12.5, 20.7 / 17.0; 25 of 200 x 150 fp32 13.1 / 10.8, 17.8 / 13.7, of 125 8.8 / 9.6, 10.7 / 11.4; 40 of 165 16.0 / 16.4,
// 21.9 / 25.6; 40 of 400 32.2 / 24.6, 45.7 / 38.3; 60 of 400 32.6 / 32.9, 46.7 / 48.8; 100 of 400 41.5 / 46.1, 62.0 / 70.1, of 900 88.0 / 84.6, 144 / 151; 200 of 650 107 / 117, 201 / 215.
// Sentences that end within a block, more of them than the chip holds at once, need no registers for the block after it (brief).  Measured (us, states, then gradients, with
// those registers / without): 2000 sentences of 15 words x 256 bf16 20.1 / 16.4, 63 / 36; 1024 of 15 x 256 fp32 14.3 / 13.0, 32.6 / 28.0; 256 of 27 x 512 bf16 7.4 / 8.1, 18.4 / 15.4.
// Large parts have half as many pairs to be taken, small ones fill the chip with fewer words and waste less of a sentence's last part.  Measured (us, large / small, bf16): states
// of 2 sentences of 13 000 words x 2048 99 / 107, 8 of 1800 x 1024 34.5 / 37.0, 2 of 5000 x 2048 47.0 / 48.2, 60 of 1000 x 512 65 / 59, 4 of 1500 x 256 18.2 / 13.7; gradients
// (less the states): 8 of 1800 x 1024 52 / 57, one of 8000 x 1024 42 / 50, one of 4000 x 1024 25 / 30, 4 of 1500 x 256 20 / 17.
// (All as graphs of ten calls.)
bool plan(const tl_recurrence *r, bool back, Plan *p)
{
    const long long rows = r->n_rows, trees = r->n_trees;
    p->V = LANE_BYTES / element_size(r->dtype);
    p->narrow = r->channels < p->V;             // fewer channels than a lane would have: one each
    if (p->narrow) p->V = 1;
    p->slices = (r->channels + 64 * p->V - 1) / (64 * p->V);
    const long long workgroups = trees * p->slices;
    p->cut = rows > 96 * trees && rows / trees > 2 * workgroups;
    p->single = !back && !p->cut && rows <= 8 * trees;
    p->brief = !p->cut && rows <= 32 * trees && workgroups >= 1024 && workgroups >= 8 * compute_units();      // (asking for the units takes more than a microsecond)
    p->large = false;
    p->shift = REC_WHOLE;
    if (p->cut) {
        const int words = log_2(back ? BL_WAVES * BL_WORDS : FL_WAVES * FL_WORDS);
        const long long blocks = ((rows >> words) + trees) * p->slices, units = compute_units();
        p->large = back ? blocks >= units - units / 8 : 2 * blocks >= 3 * units && rows >= 1500 * trees;
        p->shift = p->large ? words : log_2(back ? BC_WAVES * BC_WORDS : FC_WAVES * FC_WORDS);
    }
    const long long slots = (rows >> p->shift) + trees;
    p->blocks = slots * p->slices;
    p->slots = (int)slots;
    p->pairs = p->cut ? round16(8 * slots * r->channels) : 0;
    p->states = p->cut ? round16(4 * ((slots / REC_GROUP + 1) * r->channels + REC_LINE * p->slices)) : 0;
    p->parts = p->cut ? 16 * slots : 0;
    p->copy = p->cut && !back ? round16(4 * trees * r->channels) : 0;
    return p->blocks <= most_blocks(64 * 16);
}

RecurArgs arguments(const tl_recurrence *r, const Plan &p)
{
    RecurArgs a = {};
    a.g = r->g;
    a.g_row = r->g_row;
    a.x = r->x;
    a.x_row = r->x_row;
    a.off = r->off;
    a.n_trees = r->n_trees;
    a.n_rows = r->n_rows;
    a.C = r->channels;
    a.slices = p.slices;
    a.slots = p.slots;
    a.shift = p.shift;
    a.polls = r->spin_limit == 0 || r->spin_limit > REC_POLLS ? REC_POLLS : r->spin_limit > 0 ? r->spin_limit : 0;
    return a;
}

void lay_out(const Plan &p, void *workspace, RecurArgs *a)
{
    if (!p.cut) return;
    char *const base = static_cast<char *>(workspace);
    a->pairs = reinterpret_cast<uint64_t *>(base);
    a->states = reinterpret_cast<uint32_t *>(base + p.pairs);
    a->taken = a->states + (p.slots / REC_GROUP + 1ll) * a->C;
    a->parts = reinterpret_cast<int4 *>(base + p.pairs + p.states);
    a->broken = reinterpret_cast<uint32_t *>(base + p.pairs + p.states + p.parts + p.copy);
    if (p.copy && a->h0) a->copy = reinterpret_cast<float *>(base + p.pairs + p.states + p.parts);
}

template <auto KERNEL> hipError_t start(const RecurArgs &a, const Plan &p, int waves, hipStream_t st)
{
    hipLaunchKernelGGL(KERNEL, dim3((unsigned)p.blocks), dim3(64 * waves), 0, st, a);
    return hipGetLastError();
}

template <typename T, int V, int GATE, bool ONCE> hipError_t cut_of(const RecurArgs &a, const Plan &p, hipStream_t st)
{
    return p.large ? start<k_recur<T, V, FL_WAVES, FL_WORDS, GATE, true, ONCE, false>>(a, p, FL_WAVES, st)
                   : start<k_recur<T, V, FC_WAVES, FC_WORDS, GATE, true, ONCE, false>>(a, p, FC_WAVES, st);
}

template <typename T, int V, int GATE> hipError_t forward_of(const RecurArgs &a, const Plan &p, hipStream_t st)
{
    if (p.cut) return a.tape ? cut_of<T, V, GATE, false>(a, p, st) : cut_of<T, V, GATE, true>(a, p, st);
    if (p.single) return start<k_recur<T, V, 1, F_WORDS, GATE, false, false, true>>(a, p, 1, st);
    if (p.brief) return start<k_recur<T, V, FB_WAVES, FB_WORDS, GATE, false, false, false>>(a, p, FB_WAVES, st);
    if (!a.tape) return start<k_recur<T, V, F_WAVES, F_WORDS, GATE, false, true, true>>(a, p, F_WAVES, st);
    return start<k_recur<T, V, F_WAVES, F_WORDS, GATE, false, false, true>>(a, p, F_WAVES, st);
}

template <typename T, int V, int GATE> hipError_t backward_of(const RecurArgs &a, const Plan &p, hipStream_t st)
{
    if (p.cut && p.large) return start<k_recur_back<T, V, BL_WAVES, BL_WORDS, GATE, true, false>>(a, p, BL_WAVES, st);
    if (p.cut) return start<k_recur_back<T, V, BC_WAVES, BC_WORDS, GATE, true, false>>(a, p, BC_WAVES, st);
    if (p.brief) return start<k_recur_back<T, V, BB_WAVES, BB_WORDS, GATE, false, false>>(a, p, BB_WAVES, st);
    return start<k_recur_back<T, V, B_WAVES, B_WORDS, GATE, false, true>>(a, p, B_WAVES, st);
}

template <typename T, int V, int GATE> hipError_t launch_of(const RecurArgs &a, const Plan &p, bool back, hipStream_t st)
{
    return back ? backward_of<T, V, GATE>(a, p, st) : forward_of<T, V, GATE>(a, p, st);
}

template <typename T, int GATE> hipError_t launch_at(const RecurArgs &a, const Plan &p, bool back, hipStream_t st)
{
    if (p.cut) {
        const long long words = (p.pairs + p.states) / 8, copies = (long long)a.n_trees * a.C, most = 4ll * compute_units();
        const long long blocks = ((words > copies ? words : copies) + 255) / 256;
        hipLaunchKernelGGL(k_recur_prepare, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a, words, copies);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if constexpr (sizeof(T) < LANE_BYTES)
        if (p.narrow) return launch_of<T, 1, GATE>(a, p, back, st);
    return launch_of<T, LANE_BYTES / sizeof(T), GATE>(a, p, back, st);
}

template <typename T> hipError_t launch_for(const RecurArgs &a, int gate, const Plan &p, bool back, hipStream_t st)
{
    return gate == TL_GATE_SIGMOID ? launch_at<T, TL_GATE_SIGMOID>(a, p, back, st) : launch_at<T, TL_GATE_GIVEN>(a, p, back, st);
}

int launch(const tl_recurrence *r, const RecurArgs &a, const Plan &p, bool back, void *stream)
{
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = r->dtype == TL_DT_F32    ? launch_for<float>(a, r->gate, p, back, st)
                         : r->dtype == TL_DT_BF16 ? launch_for<bf16_t>(a, r->gate, p, back, st)
                                                  : launch_for<f16_t>(a, r->gate, p, back, st);
    return e == hipSuccess ? TL_OK : TL_EHIP;
}

bool float_pointer(const void *p) { return ((uintptr_t)p & 3) == 0; }

}  // namespace

extern "C" {

int tl_recur_workspace(const tl_recurrence *r, int backward, int64_t *bytes)
{
    Plan p;
    if (!bytes || !check(r)) return TL_EINVAL;
    *bytes = 0;
    if (r->n_trees == 0) return TL_OK;
    if (!plan(r, backward != 0, &p)) return TL_EINVAL;
    *bytes = p.workspace();
    return TL_OK;
}

int tl_recur(const tl_recurrence *r, const float *h0, void *h, int64_t h_row, float *h_last, float *tape, void *workspace_p, int64_t workspace_bytes, void *hip_stream)
{
    if (!check(r) || !check_matrix(h, h_row, r->dtype, r->n_rows, r->channels, true)) return TL_EINVAL;
    if (!float_pointer(h0) || !float_pointer(h_last) || !float_pointer(tape)) return TL_EINVAL;
    if (r->n_trees == 0) return TL_OK;
    if (r->n_rows > 0 && (h == r->g || h == r->x)) return TL_EINVAL;         // (words that have to be walked are read a second time)
    Plan p;
    if (!plan(r, false, &p)) return TL_EINVAL;
    const long long need = p.workspace();
    if (need > workspace_bytes) return TL_ELIMIT;
    if (need > 0 && (!workspace_p || ((uintptr_t)workspace_p & 15))) return TL_EINVAL;
    RecurArgs a = arguments(r, p);
    a.h = h;
    a.h_row = h_row;
    a.h0 = h0;
    a.h_last = h_last;
    a.tape = tape;
    lay_out(p, workspace_p, &a);
    return launch(r, a, p, false, hip_stream);
}

int tl_recur_backward(const tl_recurrence *r, const float *tape, const void *d_h, int64_t d_h_row, const float *d_last, void *d_g, int64_t d_g_row, void *d_x,
                      int64_t d_x_row, float *d_h0, void *workspace_p, int64_t workspace_bytes, void *hip_stream)
{
    if (!check(r) || (d_h && !check_matrix(d_h, d_h_row, r->dtype, r->n_rows, r->channels, false))) return TL_EINVAL;
    if (!check_matrix(d_g, d_g_row, r->dtype, r->n_rows, r->channels, true) || !check_matrix(d_x, d_x_row, r->dtype, r->n_rows, r->channels, true)) return TL_EINVAL;
    if (!float_pointer(tape) || !float_pointer(d_last) || !float_pointer(d_h0) || (r->n_rows > 0 && !tape)) return TL_EINVAL;
    if (r->n_trees == 0) return TL_OK;
    if (d_h0 && d_h0 == d_last) return TL_EINVAL;
    for (const void *out : {d_g, d_x})
        if (r->n_rows > 0 && (out == r->g || out == r->x || out == d_h)) return TL_EINVAL;
    if (r->n_rows > 0 && d_g == d_x) return TL_EINVAL;
    Plan p;
    if (!plan(r, true, &p)) return TL_EINVAL;
    const long long need = p.workspace();
    if (need > workspace_bytes) return TL_ELIMIT;
    if (need > 0 && (!workspace_p || ((uintptr_t)workspace_p & 15))) return TL_EINVAL;
    RecurArgs a = arguments(r, p);
    a.tape = const_cast<float *>(tape);
    a.d_h = d_h;
    a.d_h_row = d_h_row;
    a.d_last = d_last;
    a.d_g = d_g;
    a.d_g_row = d_g_row;
    a.d_x = d_x;
    a.d_x_row = d_x_row;
    a.d_h0 = d_h0;
    lay_out(p, workspace_p, &a);
    return launch(r, a, p, true, hip_stream);
}

}  // extern "C"
