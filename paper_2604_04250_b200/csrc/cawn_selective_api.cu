// Selective scan: argument checks, workspaces and the order of launches.
#include "cawn_selective.cuh"

namespace cawn {
namespace {

int check(const cawn_scan_params *p)
{
    if (p == nullptr) return CAWN_ERR_NULL_POINTER;
    if (p->struct_size != sizeof(cawn_scan_params)) return CAWN_ERR_INVALID_ARG;
    if (p->B < 1 || p->L < 0 || p->D < 1 || p->N < 1 || p->G < 1 || p->D % p->G != 0 || p->rows < 0 || !storage_flags_ok(p->flags) ||
        (p->softplus != 0 && p->softplus != 1) || p->reserved != 0)
        return CAWN_ERR_INVALID_ARG;
    const int64_t bc = (int64_t)p->G * p->N;
    for (int64_t stride : {p->x_stride, p->dt_stride, p->z_stride})
        if (stride != 0 && stride < p->D) return CAWN_ERR_INVALID_ARG;
    for (int64_t stride : {p->b_stride, p->c_stride})
        if (stride != 0 && stride < bc) return CAWN_ERR_INVALID_ARG;
    if (p->N > 64 || p->D > (1 << 22) || p->G > 65535) return CAWN_ERR_UNSUPPORTED;
    int64_t wide = most(p->D, bc);
    for (int64_t stride : {p->x_stride, p->dt_stride, p->z_stride, p->b_stride, p->c_stride}) wide = most(wide, stride);
    const double rows = p->rows > 0 ? (double)p->rows : (double)p->B * (double)p->L;
    if (rows * (double)wide > 1.0e17) return CAWN_ERR_UNSUPPORTED;
    if ((double)p->B * (p->D / kScanChannels + p->G) * 16.0 > 2.0e9 || (double)p->B * ((double)p->L / kTile + 1) > 2.0e9) return CAWN_ERR_UNSUPPORTED;
    return CAWN_OK;
}

int64_t blocks_of(const cawn_scan_params *p) { return p->G * ceil_div(p->D / p->G, kScanChannels); }
int64_t rows_of(const cawn_scan_params *p) { return p->rows > 0 ? p->rows : (int64_t)p->B * p->L; }

// Segments of the time axis, none shorter than 128 tokens.  Where the blocks of whole sequences leave multiprocessors idle, as many
// segments as are resident at once; otherwise none: 2048 tokens of 16 states take 112 us with one block a multiprocessor, 131 with
// two and 233 with four, and the pass before it half as much again (74 blocks: 112 us whole, 67 in four segments; 148 blocks of 32
// states: 125 us whole, 164 in two).
// The backward's pass is an eighth of its walk: two segments pay as soon as they are resident, with 9 to 16 states up to seven tenths of
// the places (1024 tokens of 16 states, float: 288 blocks 669 us whole, 575 in two, 352 blocks 692 and 687, 384 blocks 694 and 742; bfloat16:
// 416 blocks 709 and 679, 448 blocks 729 and 781; with 8 states, float, 320 blocks 669 and 687, with 24 224 blocks 742 and 790).
// Packed sequences count by their rows, as so many of the longest one's length: blocks of short ones end early.
constexpr int kShortest = 128, kMostSegments = 64;
int64_t slots_of(const cawn_scan_params *p, bool bwd)
{
    const Shape s = shape_of(p->N);
    return (int64_t)sm_count() * (bwd ? s.resident_bwd(p->flags != 0) : s.resident());
}
// The most blocks that the backward takes in two segments each.
int64_t most_in_two(const cawn_scan_params *p) { return shape_of(p->N).nl == 4 ? slots_of(p, true) * 7 / 10 : slots_of(p, true) / 2; }
int64_t segments_of(const cawn_scan_params *p, bool bwd)
{
    const int64_t sequences = p->rows > 0 && p->L > 0 && p->rows / p->L < p->B ? p->rows / p->L + 1 : p->B;
    const int64_t whole = sequences * blocks_of(p), room = slots_of(p, bwd) / whole, longest = most(p->L / kShortest, 1);
    const int64_t cut = bwd && whole <= most_in_two(p) ? most(room, 2) : room;
    if (cut < (bwd ? 2 : 3) || (!bwd && whole > sm_count())) return 1;
    const int64_t s = cut < longest ? cut : longest;
    return s < kMostSegments ? s : kMostSegments;
}
// For a size query: the most segments of one sequence, and of all sequences together (counted by the rows where they are packed: see
// carve_segments), in any call with up to this B, L and rows.
struct Most { int64_t of_one, of_all; };
Most most_segments(const cawn_scan_params *p, bool bwd)
{
    const int64_t room = most(slots_of(p, bwd) / blocks_of(p), 1), longest = most(p->L / kShortest, 1);
    const int64_t each = bwd ? most(room, 2 * (most_in_two(p) / blocks_of(p))) : room, of_one = each < longest ? each : longest;
    const int64_t whole = p->rows > 0 ? p->rows / kShortest : p->B * longest;
    return {of_one < kMostSegments ? of_one : kMostSegments, each < whole ? each : whole};
}

// A workspace in its parts, each on a 256-byte boundary.
struct Carver {
    unsigned char *base;
    size_t used = 0;
    float *floats(int64_t n)
    {
        float *p = base != nullptr ? reinterpret_cast<float *>(base + used) : nullptr;
        used += ((size_t)n * sizeof(float) + 255) / 256 * 256;
        return p;
    }
};

// The parts of a call whose time axis is cut.  All segments of a sequence but one keep an end.  These are numbered by sequences or, where
// that are fewer (packed, many sequences shorter than L), by rows: a sequence of n rows from row r has floor((n - 1) / per) of them from
// floor(r / per) on, so those of two sequences never meet, and all lie below rows / per.  That is no more than what is resident at once: by
// segments_of, rows / L sequences of S segments are, and per >= L / S.
// `sized`: for any call up to this one (the size query) instead of for this very call.
void carve_segments(Carver &c, SelectiveParams &P, const cawn_scan_params *p, bool bwd, bool sized)
{
    const Most m = most_segments(p, bwd);
    if ((sized ? m.of_one : P.S) < 2) return;
    const int64_t by_sequence = p->B * ((sized ? m.of_one : P.S) - 1);
    const int64_t by_rows = sized ? m.of_all : P.seq.offsets != nullptr ? P.seq.rows / P.per : by_sequence;
    P.by_rows = by_rows < by_sequence;
    const int64_t ends = (bwd ? 2 : 1) * (P.by_rows ? by_rows : by_sequence);       // the backward may have one per half
    P.seg_state = c.floats(ends * p->D * p->N);
    P.seg_time = c.floats(ends * p->D);
    if (!bwd) P.first = c.floats((int64_t)p->B * p->D * p->N);
}
// Partial sums of grad_A, grad_skip and grad_dt_bias: rows that begin on 16 bytes, one a segment, numbered as the ends are with one more for
// each sequence.
int64_t param_cols(const cawn_scan_params *p) { return ceil_div((int64_t)p->D * (p->N + 2), 4) * 4; }
void carve_bwd(Carver &c, SelectiveParams &P, const cawn_scan_params *p, bool sized)
{
    carve_segments(c, P, p, true, sized);
    P.part_bc = c.floats(blocks_of(p) * rows_of(p) * 2 * p->N);
    const Most m = most_segments(p, true);
    P.param_rows = P.by_rows ? p->B + (sized ? m.of_all : P.seq.rows / P.per) : p->B * (sized ? m.of_one : P.S);
    P.part_param = c.floats(P.param_rows * param_cols(p));
}
int64_t checkpoint_rows(const cawn_scan_params *p) { return rows_of(p) / kTile + p->B + 1; }

// The time axis in segments, for one direction.
void cut(SelectiveParams &P, const cawn_scan_params *p, bool bwd)
{
    P.S = (int)segments_of(p, bwd);
    P.per = most(ceil_div(ceil_div(p->L, P.S), kTile), 1) * kTile;
    P.per_inverse = 1.0 / (double)P.per;
    P.halves = bwd && 2 * (P.S - 1) * p->B * blocks_of(p) <= slots_of(p, false) ? 2 : 1;
}

SelectiveParams fill(const cawn_scan_params *p, const int64_t *offsets, const void *x, const void *dt, const void *z, const void *b, const void *c)
{
    SelectiveParams P = {};
    const int per = p->flags != 0 ? 8 : 4;
    P.seq = {reinterpret_cast<const long long *>(offsets), p->L, rows_of(p), p->B};
    P.D = p->D; P.N = p->N; P.G = p->G; P.Dg = p->D / p->G;
    P.blocks = (int)ceil_div(P.Dg, kScanChannels);
    auto stride = [](int64_t s, int64_t dense) { return s != 0 ? s : dense; };
    P.xs = stride(p->x_stride, p->D); P.dts = stride(p->dt_stride, p->D); P.zs = stride(p->z_stride, p->D);
    P.bs = stride(p->b_stride, (int64_t)p->G * p->N); P.cs = stride(p->c_stride, (int64_t)p->G * p->N);
    const bool eights = P.Dg % 8 == 0;          // a block's channels begin on a word
    P.x = x; P.dt = dt; P.z = z; P.bm = b; P.cm = c;
    P.whole_x = eights && P.xs % per == 0 && begins_on(x, 16);
    P.whole_dt = eights && P.dts % per == 0 && begins_on(dt, 16);
    P.whole_z = eights && P.zs % per == 0 && begins_on(z, 16);
    P.whole_d = eights && p->D % per == 0;
    const uintptr_t quad = p->flags != 0 ? 8 : 16;
    P.whole_b = p->N % 4 == 0 && P.bs % 4 == 0 && begins_on(b, quad);
    P.whole_c = p->N % 4 == 0 && P.cs % 4 == 0 && begins_on(c, quad);
    P.whole = P.whole_x && P.whole_dt && P.whole_z && P.whole_d && P.whole_b && P.whole_c;
    P.softplus = p->softplus;
    P.param_cols = param_cols(p);
    return P;
}

}  // namespace
}  // namespace cawn

extern "C" int cawn_selective_scan_workspace_bytes(const cawn_scan_params *params, int op, size_t *bytes)
{
    using namespace cawn;
    const int rc = check(params);
    if (rc != CAWN_OK) return rc;
    if (bytes == nullptr) return CAWN_ERR_NULL_POINTER;
    SelectiveParams P = {};
    Carver c = {nullptr};
    switch (op) {
    case CAWN_SCAN_FWD: carve_segments(c, P, params, false, true); break;
    case CAWN_SCAN_BWD: carve_bwd(c, P, params, true); break;
    case CAWN_SCAN_BWD_RECOMPUTE:
        carve_bwd(c, P, params, true);
        c.floats(checkpoint_rows(params) * params->D * params->N);
        carve_segments(c, P, params, false, true);
        break;
    case CAWN_SCAN_CHECKPOINTS: c.floats(checkpoint_rows(params) * params->D * params->N); break;
    default: return CAWN_ERR_INVALID_ARG;
    }
    *bytes = c.used;
    return CAWN_OK;
}

extern "C" int cawn_selective_scan_fwd(const cawn_scan_params *params, const void *x, const void *dt, const float *A, const void *B,
                                       const void *C, const float *skip, const float *dt_bias, const void *z, const float *state_in,
                                       const int64_t *offsets, void *y, float *state_out, float *checkpoints,
                                       void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace cawn;
    int rc = check(params);
    if (rc == CAWN_OK) rc = check_offsets(offsets, params->B, params->L, params->rows);
    if (rc != CAWN_OK) return rc;
    if (A == nullptr || (params->L > 0 && (x == nullptr || dt == nullptr || B == nullptr || C == nullptr || y == nullptr))) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(A, skip, dt_bias, state_in, y, state_out, checkpoints, workspace) || !elements_aligned(params->flags, x, dt, z, B, C))
        return CAWN_ERR_MISALIGNED;
    SelectiveParams P = fill(params, offsets, x, dt, z, B, C);
    cut(P, params, false);
    Carver c = {static_cast<unsigned char *>(workspace)};
    carve_segments(c, P, params, false, false);
    if (c.used > 0 && workspace == nullptr) return CAWN_ERR_NULL_POINTER;
    if (c.used > workspace_bytes) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    P.A = A; P.skip = skip; P.dt_bias = dt_bias;
    P.state_in = state_in; P.y = y; P.state_out = state_out; P.checkpoints = checkpoints;
    const Shape s = shape_of(params->N);
    const bool half = params->flags != 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (P.S > 1) rc = launch_selective_fwd(P, s, half, true, st);
    return rc != CAWN_OK ? rc : launch_selective_fwd(P, s, half, false, st);
}

extern "C" int cawn_selective_scan_step(const cawn_scan_params *params, const void *x, const void *dt, const float *A, const void *B,
                                        const void *C, const float *skip, const float *dt_bias, const void *z, const float *state_in,
                                        void *y, float *state_out, void *cuda_stream)
{
    using namespace cawn;
    int rc = check(params);
    if (rc == CAWN_OK) rc = check_offsets(nullptr, params->B, params->L, params->rows);
    if (rc != CAWN_OK) return rc;
    if (A == nullptr || (params->L > 0 && (x == nullptr || dt == nullptr || B == nullptr || C == nullptr || y == nullptr))) return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(A, skip, dt_bias, state_in, y, state_out) || !elements_aligned(params->flags, x, dt, z, B, C)) return CAWN_ERR_MISALIGNED;
    SelectiveParams P = fill(params, nullptr, x, dt, z, B, C);
    P.A = A; P.skip = skip; P.dt_bias = dt_bias;
    P.state_in = state_in; P.y = y; P.state_out = state_out;
    return launch_selective_step(P, params->flags != 0, static_cast<cudaStream_t>(cuda_stream));
}

extern "C" int cawn_selective_scan_bwd(const cawn_scan_params *params, const void *x, const void *dt, const float *A, const void *B,
                                       const void *C, const float *skip, const float *dt_bias, const void *z, const float *state_in,
                                       const int64_t *offsets, const float *checkpoints, const void *grad_y, const float *grad_state_out,
                                       void *grad_x, void *grad_dt, float *grad_A, void *grad_B, void *grad_C, float *grad_skip,
                                       float *grad_dt_bias, void *grad_z, float *grad_state_in,
                                       void *workspace, size_t workspace_bytes, void *cuda_stream)
{
    using namespace cawn;
    int rc = check(params);
    if (rc == CAWN_OK) rc = check_offsets(offsets, params->B, params->L, params->rows);
    if (rc != CAWN_OK) return rc;
    if (z == nullptr && grad_z != nullptr) return CAWN_ERR_INVALID_ARG;
    if (A == nullptr || grad_A == nullptr || workspace == nullptr) return CAWN_ERR_NULL_POINTER;
    if (params->L > 0 && (x == nullptr || dt == nullptr || B == nullptr || C == nullptr || grad_y == nullptr || grad_x == nullptr || grad_dt == nullptr ||
                          grad_B == nullptr || grad_C == nullptr || (z != nullptr && grad_z == nullptr)))
        return CAWN_ERR_NULL_POINTER;
    if (!all_aligned16(A, skip, dt_bias, state_in, checkpoints, grad_y, grad_state_out, grad_x, grad_dt, grad_A, grad_B, grad_C, grad_skip,
                       grad_dt_bias, grad_z, grad_state_in, workspace) || !elements_aligned(params->flags, x, dt, z, B, C))
        return CAWN_ERR_MISALIGNED;
    SelectiveParams P = fill(params, offsets, x, dt, z, B, C);
    Carver c = {static_cast<unsigned char *>(workspace)};
    cut(P, params, true);
    carve_bwd(c, P, params, false);
    P.A = A; P.skip = skip; P.dt_bias = dt_bias; P.state_in = state_in;
    const Shape s = shape_of(params->N);
    const bool half = params->flags != 0, again = checkpoints == nullptr && params->L > 0;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    P.checkpoints = const_cast<float *>(checkpoints);
    SelectiveParams F = P;          // the forward's walk once more, for its states alone
    if (again) {
        P.checkpoints = F.checkpoints = c.floats(checkpoint_rows(params) * params->D * params->N);
        cut(F, params, false);
        carve_segments(c, F, params, false, false);
    }
    if (c.used > workspace_bytes) return CAWN_ERR_WORKSPACE_TOO_SMALL;
    P.gy = grad_y; P.gstate_out = grad_state_out; P.gx = grad_x; P.gdt = grad_dt; P.gz = grad_z; P.gstate_in = grad_state_in;
    if (again && F.S > 1) rc = launch_selective_fwd(F, s, half, true, st);
    if (rc == CAWN_OK && again) rc = launch_selective_fwd(F, s, half, false, st);
    if (rc == CAWN_OK && P.S > 1) rc = launch_selective_bwd(P, s, half, true, st);
    if (rc == CAWN_OK) rc = launch_selective_bwd(P, s, half, false, st);
    if (rc == CAWN_OK && params->L > 0) rc = launch_selective_bc(P, half, grad_B, grad_C, st);
    if (rc != CAWN_OK) return rc;
    const long long D = params->D;
    PartialSums sums = {P.part_param, P.param_rows, P.param_cols, {grad_A, grad_skip, grad_dt_bias}, {D * params->N, D, D}};
    return sum_partials(sums, st);
}
