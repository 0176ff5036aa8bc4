// C entry points of the recurrence along sentences.
#include "entry.hpp"
#include "recur.hpp"

using namespace tl;

namespace {

// Waves of a workgroup, words that each takes at a time and bytes of a row that a lane has: of whole sentences, and of parts of cut ones.
constexpr int F_WAVES = 4, F_WORDS = 8, F_BYTES = 4;
constexpr int B_WAVES = 4, B_WORDS = 16, B_BYTES = 4;
constexpr int FB_WAVES = 4, FB_WORDS = 8, BB_WAVES = 4, BB_WORDS = 16;
constexpr int FC_WAVES = 8, FC_WORDS = 32, FC_BYTES = 4;
constexpr int BC_WAVES = 8, BC_WORDS = 16, BC_BYTES = 4;

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
    bool single, brief, cut;                    // a wave per sentence; sentences of a block or two; parts
    long long blocks, pairs, states, parts, copy;               // bytes of the workspace's parts
    long long workspace() const { return pairs + states + parts + copy + (cut ? 16 : 0); }
};

// Whether sentences are cut into parts, by their words on average (the host does not know the lengths, and a batch with one sentence much longer than the
// others waits for it).  A whole sentence is a chain of blocks, a part waits for others and needs a launch more.  Measured (us, whole / cut, states
// alone; words x channels, bf16): 40 sentences of 100 x 512 12.1 / 13.0, 60 of 400 34.8 / 34.3, 60 of 1000 72 / 60, 100 of 400 44 / 47, 100 of 1000 98 / 88, 256 of 750 151 / 161,
// 4 of 1500 x 256 116 / 17; with gradients 30 / 34, 85 / 82, 179 / 159, 112 / 119, 253 / 244, 409 / 449, 287 / 37.
// Sentences that end within a block, more of them than the chip holds at once, need no registers for the block after it (brief).  Measured (us, with gradients, with
// those registers / without): 2000 sentences of 15 words x 256 bf16 71 / 49, 1024 of 15 x 256 fp32 42 / 38, 256 of 27 x 512 bf16 29.5 / 30.2.
bool plan(const tl_recurrence *r, bool back, Plan *p)
{
    const long long rows = r->n_rows, trees = r->n_trees;
    const int size = element_size(r->dtype);
    const int whole_V = (back ? B_BYTES : F_BYTES) / size;
    const long long workgroups = trees * ((r->channels + 64 * whole_V - 1) / (64 * whole_V));
    p->cut = rows > 128 * trees && rows / trees > 2 * workgroups;
    p->single = !back && !p->cut && rows <= 8 * trees;
    p->brief = !p->cut && rows <= 32 * trees && workgroups >= 1024 && workgroups >= 8 * compute_units();      // (asking for the units takes more than a microsecond)
    p->V = p->cut ? (back ? BC_BYTES : FC_BYTES) / size : whole_V;
    if (r->channels < p->V) p->V = 1;
    p->slices = (r->channels + 64 * p->V - 1) / (64 * p->V);
    p->shift = !p->cut ? REC_WHOLE : back ? log_2(BC_WAVES * BC_WORDS) : log_2(FC_WAVES * FC_WORDS);
    const long long slots = (rows >> p->shift) + trees;
    p->blocks = slots * p->slices;
    p->slots = (int)slots;
    p->pairs = p->cut ? round16(8 * slots * r->channels) : 0;
    p->states = p->cut ? round16(4 * (slots / REC_GROUP + 1) * r->channels) : 0;
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
    return a;
}

void lay_out(const Plan &p, void *workspace, RecurArgs *a)
{
    if (!p.cut) return;
    char *const base = static_cast<char *>(workspace);
    a->pairs = reinterpret_cast<uint64_t *>(base);
    a->states = reinterpret_cast<uint32_t *>(base + p.pairs);
    a->parts = reinterpret_cast<int4 *>(base + p.pairs + p.states);
    a->broken = reinterpret_cast<uint32_t *>(base + p.pairs + p.states + p.parts + p.copy);
    if (p.copy && a->h0) a->copy = reinterpret_cast<float *>(base + p.pairs + p.states + p.parts);
}

template <auto KERNEL> hipError_t start(const RecurArgs &a, const Plan &p, int waves, hipStream_t st)
{
    hipLaunchKernelGGL(KERNEL, dim3((unsigned)p.blocks), dim3(64 * waves), 0, st, a);
    return hipGetLastError();
}

template <typename T, int V, int GATE> hipError_t forward_of(const RecurArgs &a, const Plan &p, hipStream_t st)
{
    if (p.cut && !a.tape) return start<k_recur<T, V, FC_WAVES, FC_WORDS, GATE, true, true, false>>(a, p, FC_WAVES, st);
    if (p.cut) return start<k_recur<T, V, FC_WAVES, FC_WORDS, GATE, true, false, false>>(a, p, FC_WAVES, st);
    if (p.single) return start<k_recur<T, V, 1, F_WORDS, GATE, false, false, true>>(a, p, 1, st);
    if (p.brief) return start<k_recur<T, V, FB_WAVES, FB_WORDS, GATE, false, false, false>>(a, p, FB_WAVES, st);
    if (!a.tape) return start<k_recur<T, V, F_WAVES, F_WORDS, GATE, false, true, true>>(a, p, F_WAVES, st);
    return start<k_recur<T, V, F_WAVES, F_WORDS, GATE, false, false, true>>(a, p, F_WAVES, st);
}

template <typename T, int V, int GATE> hipError_t backward_of(const RecurArgs &a, const Plan &p, hipStream_t st)
{
    if (p.cut) return start<k_recur_back<T, V, BC_WAVES, BC_WORDS, GATE, true, false>>(a, p, BC_WAVES, st);
    if (p.brief) return start<k_recur_back<T, V, BB_WAVES, BB_WORDS, GATE, false, false>>(a, p, BB_WAVES, st);
    return start<k_recur_back<T, V, B_WAVES, B_WORDS, GATE, false, true>>(a, p, B_WAVES, st);
}

template <typename T, int GATE> hipError_t launch_at(const RecurArgs &a, const Plan &p, bool back, hipStream_t st)
{
    constexpr int V = 4 / sizeof(T);
    static_assert(F_BYTES == 4 && B_BYTES == 4 && FC_BYTES == 4 && BC_BYTES == 4, "a lane's channels");
    if (p.cut) {
        const long long words = (p.pairs + p.states) / 8, copies = (long long)a.n_trees * a.C, most = 4ll * compute_units();
        const long long blocks = ((words > copies ? words : copies) + 255) / 256;
        hipLaunchKernelGGL(k_recur_prepare, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, st, a, words, copies);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (back) return p.V == 1 ? backward_of<T, 1, GATE>(a, p, st) : backward_of<T, V, GATE>(a, p, st);
    return p.V == 1 ? forward_of<T, 1, GATE>(a, p, st) : forward_of<T, V, GATE>(a, p, st);
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
